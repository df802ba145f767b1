// RMS norms before and after a block, forward and backward, over groups of L channels (L = width: the whole row):
//
//   before   u = residual + scale o x,  y = u r o w,             r = 1 / sqrt(mean(u^2) + eps)     u is the new residual
//   after    u = x,                     y = u r o w o silu(z)     (a gate z), or, gate first, u = x o silu(z), y = u r o w
//
// Backward, with g the gradient of u r:  du = r (g - u r c),  c = mean(g o u r);  dw = sum over rows of (dy o act) o u r.  Both sums a row
// needs, of u^2 and of g o u, are known before r is, so they are formed together.
//
// Memory-bound: every array passes once.  8 x 4096 rows, bf16, residual fp32, width 1024: 69 us, 5.8 TB/s; gated backward, width 2048 in groups of 128: 139 us, 4.8 TB/s
// (bound by registers: with two rows requested ahead 137 us, but spills for the longest rows; three blocks of 256 threads per SM 152 us).  A thread owns eight neighbouring channels (16 bytes of bf16) of every row its block
// takes, so weights are loaded once and the sums over rows (dw, dscale) stay in its registers; the next row's operands are
// requested before the current row's sums are exchanged.  Groups of up to 32 threads exchange by shuffles; longer ones also
// through shared memory, behind one barrier (two buffers in turn).  The norm is of the sum in fp32, before u is rounded to the residual's type.
//
// Rows of more than 8192 channels, odd widths and groups that are neither a power of two up to 256 nor a multiple of 256
// take plain two-pass kernels, one block per group.
#include "layer_ops.h"
#include "layer_pieces.cuh"

namespace kla {

enum { NORM_PLAIN = 0, NORM_ADD = 1, NORM_GATE = 2, NORM_GATE_FIRST = 3 };

// Where a thread stands: TX threads to a row, TY rows to a block; `lanes` threads (a power of two) exchange by shuffles, then `warps`
// warps through shared memory.
struct NormShape {
    int tx, ty, lanes, warps;
};

template <int N>
__device__ __forceinline__ void group_sums(float (&x)[N], const NormShape &s, float (*red)[N], int &turn)
{
    for (int o = s.lanes >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    if (s.warps > 1) {
        float (*buf)[N] = red + 32 * turn;
        turn ^= 1;
        const int warp = threadIdx.x >> 5, first = warp - (threadIdx.x % s.tx >> 5) % s.warps;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[warp][i] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = 0.f;
        for (int k = 0; k < s.warps; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += buf[first + k][i];
    }
}

template <typename IO, typename RES, int MODE>
__global__ void __launch_bounds__(1024) norm_fwd_kernel(NormParams p, NormShape s)
{
    __shared__ float red[64][1];
    int turn = 0;
    const int c = (threadIdx.x % s.tx) * 8, ry = threadIdx.x / s.tx;
    const bool col = c < p.width;
    float w[8], sc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = col ? p.weight[c + e] : 0.f;
        sc[e] = MODE == NORM_ADD && col && p.scale ? p.scale[c + e] : 1.f;
    }
    Pack<IO, 8> x, z;
    Pack<RES, 8> res;
    auto request = [&](int r) {
        if (r >= p.rows || !col) return;
        x.load(static_cast<const IO *>(p.x) + (size_t)r * p.x_stride + c);
        if (MODE >= NORM_GATE) z.load(static_cast<const IO *>(p.gate) + (size_t)r * p.gate_stride + c);
        if (MODE == NORM_ADD) res.load(static_cast<const RES *>(p.residual) + (size_t)r * p.width + c);
    };
    x.zero();
    z.zero();
    res.zero();
    const int step = gridDim.x * s.ty;
    request(blockIdx.x * s.ty + ry);
    for (int base = blockIdx.x * s.ty; base < p.rows; base += step) {
        const int r = base + ry;
        const bool on = r < p.rows && col;
        float u[8], act[8], sum[1] = {0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = on ? x.get(e) : 0.f;
            act[e] = 1.f;
            if (MODE == NORM_ADD) u[e] = fmaf(sc[e], u[e], on ? res.get(e) : 0.f);
            if (MODE >= NORM_GATE) {
                const float zz = z.get(e);
                act[e] = zz * sigmoid(zz);
                if (MODE == NORM_GATE_FIRST && on) u[e] *= act[e];
            }
            sum[0] = fmaf(u[e], u[e], sum[0]);
        }
        request(r + step);
        group_sums(sum, s, red, turn);
        if (on) {
            const float rr = rsqrtf(sum[0] / p.group + p.eps);
            if (MODE == NORM_ADD) {
                Pack<RES, 8> o;
                o.set(u);
                o.store(static_cast<RES *>(p.residual_out) + (size_t)r * p.width + c);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] *= rr * w[e];
                if (MODE == NORM_GATE) u[e] *= act[e];
            }
            Pack<IO, 8> o;
            o.set(u);
            o.store(static_cast<IO *>(p.out) + (size_t)r * p.width + c);
        }
    }
}

template <typename IO, typename RES, int MODE, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_bwd_kernel(NormParams p, NormShape s)
{
    __shared__ float red[64][2];
    extern __shared__ float rows_sums[];   // [ty][tx 8]
    int turn = 0;
    const int c = (threadIdx.x % s.tx) * 8, ry = threadIdx.x / s.tx;
    const bool col = c < p.width;
    float w[8], sc[8], dw[8], ds[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = col ? p.weight[c + e] : 0.f;
        sc[e] = MODE == NORM_ADD && col && p.scale ? p.scale[c + e] : 1.f;
        dw[e] = ds[e] = 0.f;
    }
    Pack<IO, 8> x, z, g;
    Pack<RES, 8> res, dres;
    auto request = [&](int r) {
        if (r >= p.rows || !col) return;
        x.load(static_cast<const IO *>(p.x) + (size_t)r * p.x_stride + c);
        g.load(static_cast<const IO *>(p.d_out) + (size_t)r * p.width + c);
        if (MODE >= NORM_GATE) z.load(static_cast<const IO *>(p.gate) + (size_t)r * p.gate_stride + c);
        if (MODE == NORM_ADD) {
            res.load(static_cast<const RES *>(p.residual) + (size_t)r * p.width + c);
            if (p.d_residual_out) dres.load(static_cast<const RES *>(p.d_residual_out) + (size_t)r * p.width + c);
        }
    };
    x.zero();
    g.zero();
    z.zero();
    res.zero();
    dres.zero();
    const int step = gridDim.x * s.ty;
    request(blockIdx.x * s.ty + ry);
    for (int base = blockIdx.x * s.ty; base < p.rows; base += step) {
        const int r = base + ry;
        const bool on = r < p.rows && col;
        // xin: x; u: what is normed; gw: gradient of (u r o w) / w;  act, dact: the gate and its derivative
        float xin[8], u[8], gw[8], act[8], dact[8], dr[8], sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            xin[e] = on ? x.get(e) : 0.f;
            gw[e] = on ? g.get(e) : 0.f;
            u[e] = xin[e];
            if (MODE == NORM_ADD) {
                u[e] = fmaf(sc[e], xin[e], on ? res.get(e) : 0.f);
                dr[e] = on ? dres.get(e) : 0.f;
            }
            if (MODE >= NORM_GATE) {
                const float zz = on ? z.get(e) : 0.f, sig = sigmoid(zz);
                act[e] = zz * sig;
                dact[e] = sig * fmaf(zz, 1.f - sig, 1.f);
                if (MODE == NORM_GATE_FIRST) u[e] *= act[e];
                else {
                    dact[e] *= gw[e];   // dy o act'
                    gw[e] *= act[e];
                }
            }
            sum[0] = fmaf(u[e], u[e], sum[0]);
            sum[1] = fmaf(gw[e] * w[e], u[e], sum[1]);
        }
        request(r + step);
        group_sums(sum, s, red, turn);
        if (on) {
            const float rr = rsqrtf(sum[0] / p.group + p.eps), cc = rr * rr * sum[1] / p.group;   // c over r: u r c = u r (r cc')
            float du[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = u[e] * rr;
                dw[e] = fmaf(gw[e], y, dw[e]);
                du[e] = rr * (gw[e] * w[e] - u[e] * cc);
                if (MODE == NORM_GATE) dact[e] *= y * w[e];
                if (MODE == NORM_GATE_FIRST) {
                    dact[e] *= du[e] * xin[e];
                    du[e] *= act[e];
                }
                if (MODE == NORM_ADD) {
                    dr[e] += du[e];
                    ds[e] = fmaf(dr[e], xin[e], ds[e]);
                    du[e] = dr[e] * sc[e];
                }
            }
            Pack<IO, 8> o;
            o.set(du);
            o.store(static_cast<IO *>(p.dx) + (size_t)r * p.width + c);
            if (MODE >= NORM_GATE) {
                o.set(dact);
                o.store(static_cast<IO *>(p.dgate) + (size_t)r * p.width + c);
            }
            if (MODE == NORM_ADD) {
                Pack<RES, 8> q;
                q.set(dr);
                q.store(static_cast<RES *>(p.dresidual) + (size_t)r * p.width + c);
            }
        }
    }
    // sums over the rows of the block: over its ty threads of a column, then one partial [2][width]
#pragma unroll
    for (int k = 0; k < (MODE == NORM_ADD ? 2 : 1); ++k) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) rows_sums[(size_t)ry * s.tx * 8 + c + e] = k ? ds[e] : dw[e];
        __syncthreads();
        for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
            float t = 0.f;
            for (int y = 0; y < s.ty; ++y) t += rows_sums[(size_t)y * s.tx * 8 + i];
            p.partial[((size_t)blockIdx.x * 2 + k) * p.width + i] = t;
        }
    }
}

// partial [n][2][width] -> dweight, dscale
__global__ void __launch_bounds__(512) norm_reduce_kernel(const float *partial, int n, int width, float *dweight, float *dscale)
{
    sum_partials(partial, n, 2 * width, [&](int i, float s) {
        if (i < width) dweight[i] = s;
        else if (dscale) dscale[i - width] = s;
    });
}

// ---- any width ------------------------------------------------------------------------------------------------------------------
// The operands of one element.
template <typename IO, typename RES>
struct NormElement {
    float x, u, act, dact, dr;
    __device__ __forceinline__ NormElement(const NormParams &p, int r, int c, int mode)
    {
        x = u = to_f32(static_cast<const IO *>(p.x)[(size_t)r * p.x_stride + c]);
        act = 1.f;
        dact = dr = 0.f;
        if (mode == NORM_ADD) {
            u = fmaf(p.scale ? p.scale[c] : 1.f, x, to_f32(static_cast<const RES *>(p.residual)[(size_t)r * p.width + c]));
            if (p.d_residual_out) dr = to_f32(static_cast<const RES *>(p.d_residual_out)[(size_t)r * p.width + c]);
        }
        if (mode >= NORM_GATE) {
            const float z = to_f32(static_cast<const IO *>(p.gate)[(size_t)r * p.gate_stride + c]), sig = sigmoid(z);
            act = z * sig;
            dact = sig * fmaf(z, 1.f - sig, 1.f);
            if (mode == NORM_GATE_FIRST) u *= act;
        }
    }
};

template <int N>
__device__ __forceinline__ void block_sums(float (&x)[N])
{
    __shared__ float red[8][N];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) red[threadIdx.x >> 5][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
        for (int k = 0; k < 8; ++k) x[i] += red[k][i];
    }
    __syncthreads();
}

// One block of 256 threads to a group of a row.
template <typename IO, typename RES>
__global__ void __launch_bounds__(256) norm_fwd_any_kernel(NormParams p, int mode)
{
    const int groups = p.width / p.group, r = blockIdx.x / groups, c0 = blockIdx.x % groups * p.group;
    float sum[1] = {0.f};
    for (int i = threadIdx.x; i < p.group; i += 256) {
        const NormElement<IO, RES> e(p, r, c0 + i, mode);
        sum[0] = fmaf(e.u, e.u, sum[0]);
    }
    block_sums(sum);
    const float rr = rsqrtf(sum[0] / p.group + p.eps);
    for (int i = threadIdx.x; i < p.group; i += 256) {
        const NormElement<IO, RES> e(p, r, c0 + i, mode);
        const size_t at = (size_t)r * p.width + c0 + i;
        if (mode == NORM_ADD) static_cast<RES *>(p.residual_out)[at] = from_f32<RES>(e.u);
        static_cast<IO *>(p.out)[at] = from_f32<IO>(e.u * rr * p.weight[c0 + i] * (mode == NORM_GATE ? e.act : 1.f));
    }
}

// Gradients of the inputs; r and c r^2 of each group go to `stats` for the sums over rows.
template <typename IO, typename RES>
__global__ void __launch_bounds__(256) norm_bwd_any_kernel(NormParams p, int mode, float2 *stats)
{
    const int groups = p.width / p.group, r = blockIdx.x / groups, c0 = blockIdx.x % groups * p.group;
    const IO *dy = static_cast<const IO *>(p.d_out) + (size_t)r * p.width;
    float sum[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < p.group; i += 256) {
        const NormElement<IO, RES> e(p, r, c0 + i, mode);
        const float gw = to_f32(dy[c0 + i]) * (mode == NORM_GATE ? e.act : 1.f);
        sum[0] = fmaf(e.u, e.u, sum[0]);
        sum[1] = fmaf(gw * p.weight[c0 + i], e.u, sum[1]);
    }
    block_sums(sum);
    const float rr = rsqrtf(sum[0] / p.group + p.eps), cc = rr * rr * sum[1] / p.group;
    if (threadIdx.x == 0) stats[blockIdx.x] = make_float2(rr, cc);
    for (int i = threadIdx.x; i < p.group; i += 256) {
        const int c = c0 + i;
        const NormElement<IO, RES> e(p, r, c, mode);
        const size_t at = (size_t)r * p.width + c;
        const float g = to_f32(dy[c]), gw = g * (mode == NORM_GATE ? e.act : 1.f);
        float du = rr * (gw * p.weight[c] - e.u * cc);
        if (mode == NORM_GATE) static_cast<IO *>(p.dgate)[at] = from_f32<IO>(e.dact * g * e.u * rr * p.weight[c]);
        if (mode == NORM_GATE_FIRST) {
            static_cast<IO *>(p.dgate)[at] = from_f32<IO>(e.dact * du * e.x);
            du *= e.act;
        }
        if (mode == NORM_ADD) {
            du += e.dr;
            static_cast<RES *>(p.dresidual)[at] = from_f32<RES>(du);
            if (p.scale) du *= p.scale[c];
        }
        static_cast<IO *>(p.dx)[at] = from_f32<IO>(du);
    }
}

// Sums over rows: a thread owns a column, a block row of the grid a run of rows.
template <typename IO, typename RES>
__global__ void __launch_bounds__(256) norm_cols_any_kernel(NormParams p, int mode, const float2 *stats, int rows_per)
{
    const int c = blockIdx.x * 256 + threadIdx.x, groups = p.width / p.group;
    if (c >= p.width) return;
    float dw = 0.f, ds = 0.f;
    const int r1 = min(p.rows, (int)(blockIdx.y + 1) * rows_per);
    for (int r = blockIdx.y * rows_per; r < r1; ++r) {
        const NormElement<IO, RES> e(p, r, c, mode);
        const float2 st = stats[(size_t)r * groups + c / p.group];
        const float gw = to_f32(static_cast<const IO *>(p.d_out)[(size_t)r * p.width + c]) * (mode == NORM_GATE ? e.act : 1.f);
        dw = fmaf(gw, e.u * st.x, dw);
        ds = fmaf(st.x * (gw * p.weight[c] - e.u * st.y) + e.dr, e.x, ds);
    }
    p.partial[((size_t)blockIdx.y * 2) * p.width + c] = dw;
    p.partial[((size_t)blockIdx.y * 2 + 1) * p.width + c] = ds;
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
static int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
static bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

// Whether the kernels with whole packs take this shape, and how.
static bool norm_shape(int width, int group, NormShape &s)
{
    if (width % 8 || width > 8192) return false;
    const int packs = width / 8;
    if (group == width) {
        if (packs <= 32) {   // a part of a warp to a row
            s.lanes = 1;
            while (s.lanes < packs) s.lanes *= 2;
            s.tx = s.lanes;
            s.warps = 1;
        } else {
            s.lanes = 32;
            s.tx = (packs + 31) / 32 * 32;
            s.warps = s.tx / 32;
        }
    } else if (group % 8 == 0 && pow2(group / 8) && group <= 256) {
        s.lanes = group / 8;
        s.warps = 1;
        s.tx = packs <= 32 && pow2(packs) ? packs : (packs + 31) / 32 * 32;
    } else if (group % 256 == 0) {   // (then so is width)
        s.lanes = 32;
        s.warps = group / 256;
        s.tx = packs;
    } else {
        return false;
    }
    s.ty = s.tx >= 256 ? 1 : 256 / s.tx;
    return true;
}
static bool whole_rows(const NormParams &p, int io_dtype)
{
    const int bytes = io_dtype == KLA_BF16 ? 2 : 4;
    return (size_t)p.x_stride * bytes % 16 == 0 && (!p.gate || (size_t)p.gate_stride * bytes % 16 == 0);
}
// (without rows a residual may be null, and the sums over rows are wanted all the same)
static int norm_mode(const NormParams &p) { return p.residual || p.dscale ? NORM_ADD : p.gate ? (p.gate_first ? NORM_GATE_FIRST : NORM_GATE) : NORM_PLAIN; }

// Blocks of the backward's persistent grid (each leaves one partial), and the row runs of the column sums of any width.
static int bwd_blocks(int rows, const NormShape &s)
{
    const int per_sm = 512 / (s.tx * s.ty) > 0 ? 512 / (s.tx * s.ty) : 1;   // (as many as are resident: fewer partial sums)
    const int need = ceil_div(rows, s.ty), most = per_sm * sm_count();
    return need < 1 ? 1 : need < most ? need : most;
}
static int any_runs(int rows, int width)
{
    const int cols = ceil_div(width, 256), most = ceil_div(rows, 32);
    const int n = ceil_div(8LL * sm_count(), cols);
    return most < 1 ? 1 : n < most ? n : most;
}
static size_t stats_bytes(int rows, int width, int group) { return ((size_t)rows * (width / group) * sizeof(float2) + 255) / 256 * 256; }

template <typename IO, typename RES>
static cudaError_t norm_fwd_t(const NormParams &p, int io_dtype, cudaStream_t stream)
{
    if (p.rows == 0) return cudaSuccess;
    const int mode = norm_mode(p);
    NormShape s;
    if (!norm_shape(p.width, p.group, s) || !whole_rows(p, io_dtype)) {
        norm_fwd_any_kernel<IO, RES><<<p.rows * (p.width / p.group), 256, 0, stream>>>(p, mode);
    } else {
        const int threads = s.tx * s.ty, most = sm_count() * (2048 / threads) * 2, need = ceil_div(p.rows, s.ty);
        const int blocks = need < most ? need : most;
        switch (mode) {
            case NORM_PLAIN: norm_fwd_kernel<IO, RES, NORM_PLAIN><<<blocks, threads, 0, stream>>>(p, s); break;
            case NORM_ADD: norm_fwd_kernel<IO, RES, NORM_ADD><<<blocks, threads, 0, stream>>>(p, s); break;
            case NORM_GATE: norm_fwd_kernel<IO, RES, NORM_GATE><<<blocks, threads, 0, stream>>>(p, s); break;
            default: norm_fwd_kernel<IO, RES, NORM_GATE_FIRST><<<blocks, threads, 0, stream>>>(p, s); break;
        }
    }
    count_launch(1);
    return cudaGetLastError();
}

template <typename IO, typename RES>
static cudaError_t norm_bwd_t(NormParams p, int io_dtype, cudaStream_t stream)
{
    const int mode = norm_mode(p);
    NormShape s;
    int n;
    if (!norm_shape(p.width, p.group, s) || !whole_rows(p, io_dtype)) {
        float2 *stats = reinterpret_cast<float2 *>(p.partial);
        p.partial += stats_bytes(p.rows, p.width, p.group) / sizeof(float);
        n = any_runs(p.rows, p.width);
        if (p.rows) {
            norm_bwd_any_kernel<IO, RES><<<p.rows * (p.width / p.group), 256, 0, stream>>>(p, mode, stats);
            count_launch(1);
        }
        norm_cols_any_kernel<IO, RES><<<dim3((unsigned)ceil_div(p.width, 256), (unsigned)n), 256, 0, stream>>>(p, mode, stats, ceil_div(p.rows, n));
    } else {
        n = bwd_blocks(p.rows, s);
        const int threads = s.tx * s.ty;
        const size_t smem = (size_t)threads * 8 * sizeof(float);   // at most 32 KB
        // (two sizes of block: 1024 threads leave 64 registers each, which spills)
        auto launch = [&](auto T) {
            switch (mode) {
                case NORM_PLAIN: norm_bwd_kernel<IO, RES, NORM_PLAIN, T()><<<n, threads, smem, stream>>>(p, s); break;
                case NORM_ADD: norm_bwd_kernel<IO, RES, NORM_ADD, T()><<<n, threads, smem, stream>>>(p, s); break;
                case NORM_GATE: norm_bwd_kernel<IO, RES, NORM_GATE, T()><<<n, threads, smem, stream>>>(p, s); break;
                default: norm_bwd_kernel<IO, RES, NORM_GATE_FIRST, T()><<<n, threads, smem, stream>>>(p, s); break;
            }
        };
        if (threads <= 512) launch(std::integral_constant<int, 512>());
        else launch(std::integral_constant<int, 1024>());
    }
    norm_reduce_kernel<<<ceil_div((mode == NORM_ADD ? 2LL : 1LL) * p.width, 32), 512, 0, stream>>>(p.partial, n, p.width, p.dweight, p.dscale);
    count_launch(2);
    return cudaGetLastError();
}

size_t norm_bwd_workspace_bytes(int rows, int width, int group)
{
    NormShape s;
    const size_t any = stats_bytes(rows, width, group) + (size_t)any_runs(rows, width) * 2 * width * sizeof(float);
    const size_t packs = norm_shape(width, group, s) ? (size_t)bwd_blocks(rows, s) * 2 * width * sizeof(float) : 0;
    return any > packs ? any : packs;
}
cudaError_t launch_norm_fwd(const NormParams &p, int io_dtype, int res_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_F32) return norm_fwd_t<float, float>(p, io_dtype, stream);
    return res_dtype == KLA_F32 ? norm_fwd_t<__nv_bfloat16, float>(p, io_dtype, stream) : norm_fwd_t<__nv_bfloat16, __nv_bfloat16>(p, io_dtype, stream);
}
cudaError_t launch_norm_bwd(const NormParams &p, int io_dtype, int res_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_F32) return norm_bwd_t<float, float>(p, io_dtype, stream);
    return res_dtype == KLA_F32 ? norm_bwd_t<__nv_bfloat16, float>(p, io_dtype, stream) : norm_bwd_t<__nv_bfloat16, __nv_bfloat16>(p, io_dtype, stream);
}

}  // namespace kla
