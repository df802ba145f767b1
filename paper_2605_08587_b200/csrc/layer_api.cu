// extern "C" boundary of the operators around a mixer: argument validation, dispatch, error codes.
#include <cmath>

#include "layer_ops.h"

namespace kla {

static bool aligned(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 15u) return false;
    return true;
}

// fp32 parameters and steps are read one by one
static bool aligned4(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return false;
    return true;
}

// Sequences and rows of a call; as the chunk forward's checks.
static kla_status check_rows(const kla_desc *d, int64_t *rows)
{
    if (!d) return KLA_ERR_NULL;
    if (d->io_dtype != KLA_F32 && d->io_dtype != KLA_BF16) return KLA_ERR_DTYPE;
    if (d->B < 1 || d->T < 0) return KLA_ERR_SHAPE;
    if (d->status_word && (reinterpret_cast<uintptr_t>(d->status_word) & 3u)) return KLA_ERR_ALIGN;
    *rows = (int64_t)d->B * d->T;
    return *rows < ((int64_t)1 << 31) - (1 << 21) ? KLA_OK : KLA_ERR_SHAPE;   // (room for the strides of loops over rows)
}
static kla_status check_sequences(const kla_desc *d)
{
    if (!d->cu_seqlens) return d->n_seq == d->B ? KLA_OK : KLA_ERR_SHAPE;
    if (!d->host_seqlens) return KLA_ERR_NULL;
    if (d->B != 1 || d->n_seq < 1) return KLA_ERR_SHAPE;
    if (d->host_seqlens[0] != 0 || d->host_seqlens[d->n_seq] != d->T) return KLA_ERR_SEQLENS;
    for (int i = 0; i < d->n_seq; ++i)
        if (d->host_seqlens[i + 1] < d->host_seqlens[i]) return KLA_ERR_SEQLENS;
    return reinterpret_cast<uintptr_t>(d->cu_seqlens) & 3u ? KLA_ERR_ALIGN : KLA_OK;
}
static kla_status check_step(const kla_desc *d) { return d->T == 1 && !d->cu_seqlens ? KLA_OK : KLA_ERR_SHAPE; }
static kla_status check_workspace(const kla_desc *d, size_t need)
{
    if (need && (!d->workspace || d->workspace_bytes < need)) return KLA_ERR_WORKSPACE;
    return aligned({d->workspace}) ? KLA_OK : KLA_ERR_ALIGN;
}
static kla_status launched(cudaError_t e) { return e == cudaSuccess ? KLA_OK : KLA_ERR_LAUNCH; }

#define CHECK(expr)                         \
    do {                                    \
        const kla_status st_ = (expr);      \
        if (st_ != KLA_OK) return st_;      \
    } while (0)

// ---- convolution ----------------------------------------------------------------------------------------------------------------
static kla_status conv_args(const kla_desc *d, int32_t channels, int32_t taps, const void *x, int64_t x_stride, const float *weight, const float *bias,
                            ConvParams *p)
{
    int64_t rows = 0;
    CHECK(check_rows(d, &rows));
    if ((!x && rows) || !weight) return KLA_ERR_NULL;   // (a call without tokens has no arrays of them)
    if (channels < 1 || taps < 2 || taps > 4 || x_stride < channels) return KLA_ERR_SHAPE;
    if (!aligned({x}) || !aligned4({weight, bias})) return KLA_ERR_ALIGN;
    *p = ConvParams{};
    p->x = x;
    p->weight = weight;
    p->bias = bias;
    p->cu_seqlens = d->cu_seqlens;
    p->x_stride = x_stride;
    p->rows = (int32_t)rows;
    p->C = channels;
    p->taps = taps;
    p->T = d->T;
    p->n_seq = d->n_seq;
    p->silu = !(d->flags & KLA_FLAG_CONV_LINEAR);
    return KLA_OK;
}

// ---- scan -------------------------------------------------------------------------------------------------------------------------
static bool ssm_widths(const kla_desc *d, int32_t groups)
{
    return d->H >= 1 && groups >= 1 && d->H % groups == 0 && d->d_k >= 8 && d->d_k <= 256 && d->d_k % 8 == 0 && d->d_v >= 8 && d->d_v <= 256 && d->d_v % 8 == 0;
}
static kla_status ssm_args(const kla_desc *d, int32_t groups, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                           int64_t v_stride, const float *dt, const float *a, const float *d_skip, SsmParams *p)
{
    int64_t rows = 0;
    CHECK(check_rows(d, &rows));
    if (d->out_dtype != KLA_F32 && d->out_dtype != KLA_BF16) return KLA_ERR_DTYPE;
    if (((!q || !k || !v || !dt) && rows) || !a) return KLA_ERR_NULL;
    if (!ssm_widths(d, groups)) return KLA_ERR_SHAPE;
    if (q_stride < (int64_t)groups * d->d_k || k_stride < (int64_t)groups * d->d_k || v_stride < (int64_t)d->H * d->d_v) return KLA_ERR_SHAPE;
    if ((int64_t)(d->n_seq > d->B ? d->n_seq : d->B) * d->H * 16 >= (int64_t)1 << 31) return KLA_ERR_SHAPE;
    const int64_t unit = d->io_dtype == KLA_BF16 ? 8 : 4;   // elements of 16 bytes
    if (q_stride % unit || k_stride % unit || v_stride % unit) return KLA_ERR_ALIGN;
    if (!aligned({q, k, v}) || !aligned4({dt, a, d_skip})) return KLA_ERR_ALIGN;
    *p = SsmParams{};
    p->q = q;
    p->k = k;
    p->v = v;
    p->dt = dt;
    p->a = a;
    p->skip = d_skip;
    p->cu_seqlens = d->cu_seqlens;
    p->host_seqlens = d->cu_seqlens ? d->host_seqlens : nullptr;
    p->whole = (d->flags & KLA_FLAG_NO_SEGMENTS) != 0;
    p->q_stride = q_stride;
    p->k_stride = k_stride;
    p->v_stride = v_stride;
    p->rows = (int32_t)rows;
    p->T = d->T;
    p->n_seq = d->n_seq;
    p->H = d->H;
    p->G = groups;
    p->N = d->d_k;
    p->P = d->d_v;
    p->status_word = d->status_word;
    p->test_timeout = (d->flags & KLA_INTERNAL_FLAG_TEST_TIMEOUT) ? 1 : 0;
    p->workspace = d->workspace;
    return KLA_OK;
}

// ---- norms ------------------------------------------------------------------------------------------------------------------------
static kla_status norm_args(const kla_desc *d, int32_t width, int32_t group, const void *x, int64_t x_stride, const void *residual, int32_t residual_dtype,
                            const float *scale, const void *gate, int64_t gate_stride, const float *weight, float eps, NormParams *p)
{
    int64_t rows = 0;
    CHECK(check_rows(d, &rows));
    if ((!x && rows) || !weight) return KLA_ERR_NULL;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return KLA_ERR_EPS;
    if (width < 1 || group < 1 || width % group || x_stride < width) return KLA_ERR_SHAPE;
    if (gate && (residual || gate_stride < width)) return KLA_ERR_SHAPE;
    if (scale && !residual && rows) return KLA_ERR_SHAPE;   // (without rows the residual has no address)
    if (residual && residual_dtype != KLA_F32 && residual_dtype != d->io_dtype) return KLA_ERR_DTYPE;
    if (rows * (width / group) >= (int64_t)1 << 31) return KLA_ERR_SHAPE;
    if (!aligned({x, residual, gate}) || !aligned4({scale, weight})) return KLA_ERR_ALIGN;
    *p = NormParams{};
    p->x = x;
    p->gate = gate;
    p->residual = residual;
    p->scale = scale;
    p->weight = weight;
    p->x_stride = x_stride;
    p->gate_stride = gate_stride;
    p->rows = (int32_t)rows;
    p->width = width;
    p->group = group;
    p->eps = eps;
    p->gate_first = (d->flags & KLA_FLAG_GATE_FIRST) != 0;
    return KLA_OK;
}

}  // namespace kla

using namespace kla;

extern "C" {

kla_status kla_conv_fwd(const kla_desc *desc, int32_t channels, int32_t taps, const void *x, int64_t x_stride, const float *weight, const float *bias,
                        const void *init_state, void *out, void *final_state)
{
    ConvParams p;
    CHECK(conv_args(desc, channels, taps, x, x_stride, weight, bias, &p));
    CHECK(check_sequences(desc));
    if (!out && p.rows) return KLA_ERR_NULL;
    if (!aligned({init_state, out, final_state})) return KLA_ERR_ALIGN;
    CHECK(check_arch());
    p.init_state = init_state;
    p.out = out;
    p.final_state = final_state;
    return launched(launch_conv_fwd(p, desc->io_dtype, (cudaStream_t)desc->stream));
}

kla_status kla_conv_step(const kla_desc *desc, int32_t channels, int32_t taps, const void *x, int64_t x_stride, const float *weight, const float *bias,
                         void *state_inout, void *out)
{
    ConvParams p;
    CHECK(conv_args(desc, channels, taps, x, x_stride, weight, bias, &p));
    CHECK(check_step(desc));
    if (!state_inout || !out) return KLA_ERR_NULL;
    if (!aligned({state_inout, out})) return KLA_ERR_ALIGN;
    CHECK(check_arch());
    p.out = out;
    p.final_state = state_inout;
    return launched(launch_conv_step(p, desc->io_dtype, (cudaStream_t)desc->stream));
}

size_t kla_conv_bwd_workspace_bytes(const kla_desc *desc, int32_t channels, int32_t taps)
{
    int64_t rows = 0;
    if (check_rows(desc, &rows) != KLA_OK || channels < 1 || taps < 2 || taps > 4) return 0;
    return conv_bwd_workspace_bytes(channels, taps, (int)rows);
}

kla_status kla_conv_bwd(const kla_desc *desc, int32_t channels, int32_t taps, const void *x, int64_t x_stride, const float *weight, const float *bias,
                        const void *init_state, const void *d_out, const void *d_final_state, void *dx, float *dweight, float *dbias,
                        void *dinit_state)
{
    ConvParams p;
    CHECK(conv_args(desc, channels, taps, x, x_stride, weight, bias, &p));
    CHECK(check_sequences(desc));
    if (((!d_out || !dx) && p.rows) || !dweight) return KLA_ERR_NULL;
    if (!aligned({init_state, d_out, d_final_state, dx, dweight, dbias, dinit_state})) return KLA_ERR_ALIGN;
    CHECK(check_workspace(desc, kla_conv_bwd_workspace_bytes(desc, channels, taps)));
    CHECK(check_arch());
    p.init_state = init_state;
    p.d_out = d_out;
    p.d_final = d_final_state;
    p.dx = dx;
    p.dweight = dweight;
    p.dbias = dbias;
    p.dinit = dinit_state;
    p.partial = static_cast<float *>(desc->workspace);
    return launched(launch_conv_bwd(p, desc->io_dtype, (cudaStream_t)desc->stream));
}

// The sizes alone
static SsmParams ssm_sizes(const kla_desc *d, int64_t rows, int32_t groups)
{
    SsmParams p = {};
    p.rows = (int32_t)rows;
    p.T = d->T;
    p.n_seq = d->n_seq;
    p.host_seqlens = d->cu_seqlens ? d->host_seqlens : nullptr;
    p.H = d->H;
    p.G = groups;
    p.N = d->d_k;
    p.P = d->d_v;
    p.whole = (d->flags & KLA_FLAG_NO_SEGMENTS) != 0;
    return p;
}
static bool on_tensor_cores(const kla_desc *d, const SsmParams &p)
{
    return ssm_chunk_supported(d->io_dtype, p.N, p.P, p.rows) && !(d->flags & KLA_FLAG_FORCE_SIMT);
}

size_t kla_ssm_fwd_workspace_bytes(const kla_desc *desc, int32_t groups)
{
    int64_t rows = 0;
    if (check_rows(desc, &rows) != KLA_OK || check_sequences(desc) != KLA_OK || !ssm_widths(desc, groups)) return 0;
    const SsmParams p = ssm_sizes(desc, rows, groups);
    return on_tensor_cores(desc, p) ? ssm_chunk_workspace_bytes(p) : 0;
}

kla_status kla_ssm_fwd(const kla_desc *desc, int32_t groups, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, const float *dt, const float *a, const float *d_skip, const float *init_state, void *out, float *final_state)
{
    SsmParams p;
    CHECK(ssm_args(desc, groups, q, q_stride, k, k_stride, v, v_stride, dt, a, d_skip, &p));
    CHECK(check_sequences(desc));
    if (!out && p.rows) return KLA_ERR_NULL;
    if (!aligned({init_state, out, final_state})) return KLA_ERR_ALIGN;
    CHECK(check_workspace(desc, kla_ssm_fwd_workspace_bytes(desc, groups)));
    CHECK(check_arch());
    p.init_state = init_state;
    p.out = out;
    p.final_state = final_state;
    if (on_tensor_cores(desc, p)) return launched(launch_ssm_chunk(p, desc->out_dtype, (cudaStream_t)desc->stream));
    return launched(launch_ssm_scan(p, desc->io_dtype, desc->out_dtype, (cudaStream_t)desc->stream));
}

kla_status kla_ssm_step(const kla_desc *desc, int32_t groups, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                        int64_t v_stride, const float *dt, const float *a, const float *d_skip, float *state_inout, void *out)
{
    SsmParams p;
    CHECK(ssm_args(desc, groups, q, q_stride, k, k_stride, v, v_stride, dt, a, d_skip, &p));
    CHECK(check_step(desc));
    if (!state_inout || !out) return KLA_ERR_NULL;
    if (!aligned({state_inout, out})) return KLA_ERR_ALIGN;
    CHECK(check_arch());
    p.final_state = state_inout;
    p.out = out;
    return launched(launch_ssm_step(p, desc->io_dtype, desc->out_dtype, (cudaStream_t)desc->stream));
}

size_t kla_ssm_bwd_workspace_bytes(const kla_desc *desc, int32_t groups)
{
    int64_t rows = 0;
    if (check_rows(desc, &rows) != KLA_OK || check_sequences(desc) != KLA_OK || !ssm_widths(desc, groups)) return 0;
    const SsmParams p = ssm_sizes(desc, rows, groups);
    return on_tensor_cores(desc, p) ? ssm_bwd_chunk_workspace_bytes(p) : ssm_bwd_workspace_bytes((int)rows, desc->n_seq, desc->H, groups, desc->d_k, desc->d_v);
}

kla_status kla_ssm_bwd(const kla_desc *desc, int32_t groups, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, const float *dt, const float *a, const float *d_skip, const float *init_state, const void *d_out,
                       const float *d_final_state, void *dq, void *dk, void *dv, float *ddt, float *da, float *dd, float *dinit_state)
{
    SsmParams p;
    CHECK(ssm_args(desc, groups, q, q_stride, k, k_stride, v, v_stride, dt, a, d_skip, &p));
    CHECK(check_sequences(desc));
    if (((!d_out || !dq || !dk || !dv || !ddt) && p.rows) || !da) return KLA_ERR_NULL;
    if (!aligned({init_state, d_out, d_final_state, dq, dk, dv, ddt, da, dd, dinit_state})) return KLA_ERR_ALIGN;
    CHECK(check_workspace(desc, kla_ssm_bwd_workspace_bytes(desc, groups)));
    CHECK(check_arch());
    p.init_state = init_state;
    p.d_out = d_out;
    p.d_final = d_final_state;
    p.dq = dq;
    p.dk = dk;
    p.dv = dv;
    p.ddt = ddt;
    p.da = da;
    p.dd = dd;
    p.dinit = dinit_state;
    if (on_tensor_cores(desc, p)) return launched(launch_ssm_bwd_chunk(p, (cudaStream_t)desc->stream));
    return launched(launch_ssm_bwd(p, desc->io_dtype, (cudaStream_t)desc->stream));
}

kla_status kla_norm_fwd(const kla_desc *desc, int32_t width, int32_t group, const void *x, int64_t x_stride, const void *residual, int32_t residual_dtype,
                        const float *scale, const void *gate, int64_t gate_stride, const float *weight, float eps, void *out, void *residual_out)
{
    NormParams p;
    CHECK(norm_args(desc, width, group, x, x_stride, residual, residual_dtype, scale, gate, gate_stride, weight, eps, &p));
    if (p.rows && (!out || (residual && !residual_out))) return KLA_ERR_NULL;
    if (!aligned({out, residual_out})) return KLA_ERR_ALIGN;
    CHECK(check_arch());
    p.out = out;
    p.residual_out = residual_out;
    return launched(launch_norm_fwd(p, desc->io_dtype, residual ? residual_dtype : desc->io_dtype, (cudaStream_t)desc->stream));
}

size_t kla_norm_bwd_workspace_bytes(const kla_desc *desc, int32_t width, int32_t group)
{
    int64_t rows = 0;
    if (check_rows(desc, &rows) != KLA_OK || width < 1 || group < 1 || width % group) return 0;
    return norm_bwd_workspace_bytes((int)rows, width, group);
}

kla_status kla_norm_bwd(const kla_desc *desc, int32_t width, int32_t group, const void *x, int64_t x_stride, const void *residual, int32_t residual_dtype,
                        const float *scale, const void *gate, int64_t gate_stride, const float *weight, float eps, const void *d_out,
                        const void *d_residual_out, void *dx, void *dresidual, float *dscale, void *dgate, float *dweight)
{
    NormParams p;
    CHECK(norm_args(desc, width, group, x, x_stride, residual, residual_dtype, scale, gate, gate_stride, weight, eps, &p));
    if ((p.rows && (!d_out || !dx || (residual && !dresidual) || (gate && !dgate))) || !dweight) return KLA_ERR_NULL;
    if (!aligned({d_out, d_residual_out, dx, dresidual, dscale, dgate, dweight})) return KLA_ERR_ALIGN;
    CHECK(check_workspace(desc, kla_norm_bwd_workspace_bytes(desc, width, group)));
    CHECK(check_arch());
    p.d_out = d_out;
    p.d_residual_out = residual ? d_residual_out : nullptr;
    p.dx = dx;
    p.dresidual = dresidual;
    p.dscale = residual || !p.rows ? dscale : nullptr;
    p.dgate = dgate;
    p.dweight = dweight;
    p.partial = static_cast<float *>(desc->workspace);
    return launched(launch_norm_bwd(p, desc->io_dtype, residual ? residual_dtype : desc->io_dtype, (cudaStream_t)desc->stream));
}

}  // extern "C"
