// Selective state space scan: per sequence and head a state S of N x P (N = d_k, P = d_v), one decay per token and head,
//
//     S_t = exp(dt_t a) S_{t-1} + dt_t k_t v_t^T,     o_t = S_t^T q_t + d v_t,
//
// q and k shared by the H / G heads of a group.  This file: the recurrence in fp32 on CUDA cores for any N and P (multiples of 8 up to
// 256), one token of it, and the reverse mode by chunks.  bf16 calls with N of 64 or 128 and P a multiple of 64 go to ssm_chunk.cu and ssm_bwd.cu.
//
// Reverse mode of one chunk of tokens (l_i: sum of dt a up to and with token i, l_Q of the whole chunk; S: the state before the
// chunk; G: the gradient of the state behind it; L_ij = exp(l_i - l_j) for j <= i):
//
//     dv_j = sum_i L_ij dt_j (q_i . k_j) do_i + dt_j e^{l_Q - l_j} G^T k_j + d do_j
//     dq_i = sum_j L_ij dt_j (do_i . v_j) k_j + e^{l_i} S do_i
//     dk_j = sum_i L_ij dt_j (do_i . v_j) q_i + dt_j e^{l_Q - l_j} G v_j              (dq, dk: summed over the heads of a group)
//
// and with R_ij = L_ij dt_j (q_i . k_j)(do_i . v_j), x_i = e^{l_i} q_i^T S do_i, z_j = dt_j e^{l_Q - l_j} k_j^T G v_j
//
//     dL/d(dt_t a) = F_t = sum_{i >= t > j} R_ij + sum_{i >= t} x_i + sum_{j < t} z_j + e^{l_Q} <S, G>
//     ddt_t = (sum_i R_it + z_t) / dt_t (formed without the division) + a F_t;   da = sum_t dt_t F_t;   dd = sum_t do_t . v_t.
#include "layer_ops.h"
#include "layer_pieces.cuh"

namespace kla {

// Rows of the state are dealt out in fours: thread part p of 8 holds rows 32 m + 4 p + e, so that the parts of a warp read 128
// consecutive bytes of a vector in shared memory.
constexpr int TT = 16;   // tokens staged at a time

// Forward.  A warp: 4 columns of the state x 8 parts of its rows, R rows to a thread; a block: 16 columns.  Bound by the latency of one token after another
// and of a warp's sums over the parts: 8 packed sequences of up to 1024 tokens, 8 heads, N = P = 64, fp32: 78 us (a token at a time 176; four, but
// with operands converted as they arrive, 129).
template <typename IO, typename OUT, int R>
__global__ void __launch_bounds__(128) ssm_scan_kernel(SsmParams p, Sequences seqs)
{
    __shared__ __align__(16) float ks[TT][8 * R], qs[TT][8 * R];
    __shared__ float vs[TT][16], xs[TT][16], al[TT];   // xs: dt v
    const int cols = (p.P + 15) / 16;
    const int cb = blockIdx.x % cols, h = blockIdx.x / cols % p.H, n = blockIdx.x / cols / p.H, g = h / (p.H / p.G);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane >> 2, cc = warp * 4 + (lane & 3), col = cb * 16 + cc;
    const int start = seqs.start(n), end = seqs.start(n + 1);
    const size_t unit = ((size_t)n * p.H + h) * p.N * p.P;
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = (r >> 2) * 32 + part * 4 + (r & 3);
        s[r] = p.init_state && row < p.N && col < p.P ? p.init_state[unit + (size_t)row * p.P + col] : 0.f;
    }
    const IO *q = static_cast<const IO *>(p.q) + g * p.N, *k = static_cast<const IO *>(p.k) + g * p.N, *v = static_cast<const IO *>(p.v) + h * p.P;
    OUT *out = static_cast<OUT *>(p.out) + h * p.P + col;
    const float a = p.a[h], skip = p.skip ? p.skip[h] : 0.f;
    // The next tile's operands wait in registers, as loaded, while this one's tokens run (a conversion or a product would wait for the load).
    IO nq[R], nk[R], nv[2];
    float nd = 0.f, ndv[2];
    auto fetch = [&](int t0) {
        const int m = end - t0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int i = threadIdx.x + 128 * j, t = i / (8 * R), x = i % (8 * R);
            nq[j] = nk[j] = from_f32<IO>(0.f);
            if (t < m && x < p.N) {
                nq[j] = q[(size_t)(t0 + t) * p.q_stride + x];
                nk[j] = k[(size_t)(t0 + t) * p.k_stride + x];
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = threadIdx.x + 128 * j, t = i >> 4, c = cb * 16 + (i & 15);
            nv[j] = from_f32<IO>(0.f);
            ndv[j] = 0.f;
            if (t < m && c < p.P) {
                nv[j] = v[(size_t)(t0 + t) * p.v_stride + c];
                ndv[j] = p.dt[(size_t)(t0 + t) * p.H + h];
            }
        }
        if (threadIdx.x < TT) nd = threadIdx.x < m ? p.dt[(size_t)(t0 + threadIdx.x) * p.H + h] : 0.f;
    };
    if (start < end) fetch(start);
    for (int t0 = start; t0 < end; t0 += TT) {
        const int m = min(TT, end - t0);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int i = threadIdx.x + 128 * j;
            qs[i / (8 * R)][i % (8 * R)] = to_f32(nq[j]);
            ks[i / (8 * R)][i % (8 * R)] = to_f32(nk[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float x = to_f32(nv[j]);
            vs[(threadIdx.x + 128 * j) >> 4][threadIdx.x & 15] = x;
            xs[(threadIdx.x + 128 * j) >> 4][threadIdx.x & 15] = ndv[j] * x;
        }
        if (threadIdx.x < TT) al[threadIdx.x] = expf(nd * a);
        __syncthreads();
        if (t0 + TT < end) fetch(t0 + TT);
        // Four tokens at a time: their vectors are fetched and their read-outs summed over the parts together (rows behind the tile's end are
        // tokens of step 0 that write nothing).
#pragma unroll 1
        for (int t0i = 0; t0i < m; t0i += 4) {
            float y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = t0i + u;
                const float x = xs[t][cc], d = al[t];
                float y0 = 0.f, y1 = 0.f;
#pragma unroll
                for (int r = 0; r < R; r += 4) {
                    const float4 kk = *reinterpret_cast<const float4 *>(&ks[t][(r >> 2) * 32 + part * 4]);
                    const float4 qq = *reinterpret_cast<const float4 *>(&qs[t][(r >> 2) * 32 + part * 4]);
                    s[r] = fmaf(kk.x, x, d * s[r]);
                    s[r + 1] = fmaf(kk.y, x, d * s[r + 1]);
                    s[r + 2] = fmaf(kk.z, x, d * s[r + 2]);
                    s[r + 3] = fmaf(kk.w, x, d * s[r + 3]);
                    y0 = fmaf(qq.x, s[r], y0);
                    y1 = fmaf(qq.y, s[r + 1], y1);
                    y0 = fmaf(qq.z, s[r + 2], y0);
                    y1 = fmaf(qq.w, s[r + 3], y1);
                }
                y[u] = y0 + y1;
            }
            // lane bits 4 and 3 choose the token, bit 2 is summed over
            const bool b4 = lane & 16, b3 = lane & 8;
            const float z0 = (b4 ? y[2] : y[0]) + __shfl_xor_sync(0xffffffffu, b4 ? y[0] : y[2], 16);
            const float z1 = (b4 ? y[3] : y[1]) + __shfl_xor_sync(0xffffffffu, b4 ? y[1] : y[3], 16);
            float z = (b3 ? z1 : z0) + __shfl_xor_sync(0xffffffffu, b3 ? z0 : z1, 8);
            z += __shfl_xor_sync(0xffffffffu, z, 4);
            const int t = t0i + (b4 ? 2 : 0) + (b3 ? 1 : 0);
            if (!(lane & 4) && t < m && col < p.P) out[(size_t)(t0 + t) * p.H * p.P] = from_f32<OUT>(fmaf(skip, vs[t][cc], z));
        }
    }
    if (p.final_state)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = (r >> 2) * 32 + part * 4 + (r & 3);
            if (row < p.N && col < p.P) p.final_state[unit + (size_t)row * p.P + col] = s[r];
        }
}

// One token.  Bound by memory: 512 sequences of 32 heads, N 128, P 64, 1.08 GB: 158 us, 6.8 TB/s.  A warp owns 16 columns of one head's state, a lane 4 of them over R rows (a run of them: part p holds rows p R ..), read once and
// written once; the read-out needs the new state, so its sums come from the registers that are being stored.
template <typename IO, typename OUT, int R>
__global__ void __launch_bounds__(128) ssm_step_kernel(SsmParams p)
{
    const int cols = (p.P + 15) / 16;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    asm volatile("griddepcontrol.wait;" ::: "memory");   // what the previous kernel on the stream wrote may be read here
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (unit >= (long long)p.rows * p.H * cols) return;
    const int lane = threadIdx.x & 31, part = lane >> 2, col = (int)(unit % cols) * 16 + (lane & 3) * 4;
    const long long bh = unit / cols;
    const int h = (int)(bh % p.H), g = h / (p.H / p.G), row0 = part * R;
    const size_t b = (size_t)(bh / p.H);
    float *sp = p.final_state + (size_t)bh * p.N * p.P + (size_t)row0 * p.P + col;
    const bool on = col < p.P;
    float4 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = on && row0 + r < p.N ? load4(sp + (size_t)r * p.P) : make_float4(0.f, 0.f, 0.f, 0.f);
    const IO *qp = static_cast<const IO *>(p.q) + b * p.q_stride + g * p.N + row0, *kp = static_cast<const IO *>(p.k) + b * p.k_stride + g * p.N + row0;
    float kr[R], qr[R];
#pragma unroll
    for (int r = 0; r < R; r += 4) {
        Pack<IO, 4> x, y;
        x.zero();
        y.zero();
        if (row0 + r < p.N) {   // (N is a multiple of 8: four rows are all inside or all outside)
            x.load(kp + r);
            y.load(qp + r);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            kr[r + e] = x.get(e);
            qr[r + e] = y.get(e);
        }
    }
    const float dt = p.dt[bh], al = expf(dt * p.a[h]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (on) v = load4(static_cast<const IO *>(p.v) + b * p.v_stride + (size_t)h * p.P + col);
    const float4 dv = make_float4(dt * v.x, dt * v.y, dt * v.z, dt * v.w);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        s[r].x = fmaf(kr[r], dv.x, al * s[r].x);
        s[r].y = fmaf(kr[r], dv.y, al * s[r].y);
        s[r].z = fmaf(kr[r], dv.z, al * s[r].z);
        s[r].w = fmaf(kr[r], dv.w, al * s[r].w);
        y.x = fmaf(qr[r], s[r].x, y.x);
        y.y = fmaf(qr[r], s[r].y, y.y);
        y.z = fmaf(qr[r], s[r].z, y.z);
        y.w = fmaf(qr[r], s[r].w, y.w);
        if (on && row0 + r < p.N) store4(sp + (size_t)r * p.P, s[r]);
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        y.x += __shfl_xor_sync(0xffffffffu, y.x, o);
        y.y += __shfl_xor_sync(0xffffffffu, y.y, o);
        y.z += __shfl_xor_sync(0xffffffffu, y.z, o);
        y.w += __shfl_xor_sync(0xffffffffu, y.w, o);
    }
    if (part == 0 && on) {
        const float d = p.skip ? p.skip[h] : 0.f;
        store4(static_cast<OUT *>(p.out) + (size_t)bh * p.P + col, make_float4(fmaf(d, v.x, y.x), fmaf(d, v.y, y.y), fmaf(d, v.z, y.z), fmaf(d, v.w, y.w)));
    }
}

// ---- reverse mode ------------------------------------------------------------------------------------------------------------
// Chunks of QB tokens, counted per sequence from its first token.  Chunk c of sequence n has slot start(n) / QB + n + c: slots of different sequences
// do not meet, and there are at most rows / QB + n_seq of them.
constexpr int QB = 32;
static_assert(QB == 2 * TT, "whole tiles to a chunk");

// The state before every chunk (REV false) or the gradient of the state behind it (REV true: from the last chunk to the first,
// G <- exp(dt a) (G + q do^T)), at [slot][H][N][P].  Layout of threads as in the forward.
template <typename IO, int R, bool REV>
__global__ void __launch_bounds__(128) ssm_states_kernel(SsmParams p, Sequences seqs, float *states)
{
    __shared__ __align__(16) float ks[TT][8 * R];
    __shared__ float xs[TT][16], al[TT];   // xs: dt v (REV: do)
    const int cols = (p.P + 15) / 16;
    const int cb = blockIdx.x % cols, h = blockIdx.x / cols % p.H, n = blockIdx.x / cols / p.H, g = h / (p.H / p.G);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane >> 2, cc = warp * 4 + (lane & 3), col = cb * 16 + cc;
    const int start = seqs.start(n), end = seqs.start(n + 1), tiles = (end - start + TT - 1) / TT;
    const size_t unit = ((size_t)n * p.H + h) * p.N * p.P, slot0 = (size_t)(start / QB) + n;
    const float *from = REV ? p.d_final : p.init_state;
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = (r >> 2) * 32 + part * 4 + (r & 3);
        s[r] = from && row < p.N && col < p.P ? from[unit + (size_t)row * p.P + col] : 0.f;
    }
    const IO *k = static_cast<const IO *>(REV ? p.q : p.k) + g * p.N, *v = static_cast<const IO *>(REV ? p.d_out : p.v) + h * p.P;
    const int64_t ks_stride = REV ? p.q_stride : p.k_stride, vs_stride = REV ? (int64_t)p.H * p.P : p.v_stride;
    const float a = p.a[h];
    auto put = [&](float *to) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = (r >> 2) * 32 + part * 4 + (r & 3);
            if (row < p.N && col < p.P) to[(size_t)row * p.P + col] = s[r];
        }
    };
    auto first = [&](int u) { return (REV ? tiles - 1 - u : u) * TT; };   // of the u-th tile in order, from the sequence's start
    IO nk[R], nv[2];   // the next tile's, as loaded
    float nd = 0.f, ndv[2];
    auto fetch = [&](int u) {
        const int t0 = start + first(u), m = end - t0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int i = threadIdx.x + 128 * j, t = i / (8 * R), x = i % (8 * R);
            nk[j] = t < m && x < p.N ? k[(size_t)(t0 + t) * ks_stride + x] : from_f32<IO>(0.f);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = threadIdx.x + 128 * j, t = i >> 4, c = cb * 16 + (i & 15);
            nv[j] = from_f32<IO>(0.f);
            ndv[j] = 1.f;
            if (t < m && c < p.P) {
                nv[j] = v[(size_t)(t0 + t) * vs_stride + c];
                if (!REV) ndv[j] = p.dt[(size_t)(t0 + t) * p.H + h];
            }
        }
        if (threadIdx.x < TT) nd = threadIdx.x < m ? p.dt[(size_t)(t0 + threadIdx.x) * p.H + h] : 0.f;
    };
    if (tiles > 0) fetch(0);
    for (int u = 0; u < tiles; ++u) {
        const int t0 = first(u), m = min(TT, end - start - t0);
        if (REV ? u == 0 || t0 % QB == QB - TT : t0 % QB == 0) put(states + ((slot0 + t0 / QB) * p.H + h) * p.N * p.P);   // a chunk begins
        __syncthreads();
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int i = threadIdx.x + 128 * j;
            ks[i / (8 * R)][i % (8 * R)] = to_f32(nk[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) xs[(threadIdx.x + 128 * j) >> 4][threadIdx.x & 15] = ndv[j] * to_f32(nv[j]);
        if (threadIdx.x < TT) al[threadIdx.x] = expf(nd * a);
        __syncthreads();
        if (u + 1 < tiles) fetch(u + 1);
        for (int i = 0; i < m; ++i) {
            const int t = REV ? m - 1 - i : i;
            const float x = xs[t][cc], d = al[t];
#pragma unroll
            for (int r = 0; r < R; r += 4) {
                const float4 kk = *reinterpret_cast<const float4 *>(&ks[t][(r >> 2) * 32 + part * 4]);
                const float w[4] = {kk.x, kk.y, kk.z, kk.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r + e] = REV ? d * fmaf(w[e], x, s[r + e]) : fmaf(w[e], x, d * s[r + e]);
            }
        }
    }
    if (REV && p.dinit) put(p.dinit + unit);
}

// For every N and P and for fp32, on CUDA cores and for that not fast (4 x 1024 fp32 tokens of 8 heads in as many groups, N = P = 64:
// 339 us; a case of that size took 332 for 1 027 with rows a multiple of 32 words apart in shared memory and states read by rows from L1).
// One block of 256 threads to a chunk and a group; its heads one after another, dq and dk summed in shared memory in that order.
// A warp owns four tokens of each product, its lanes run along the channels.  da and dd leave as one partial per chunk and head.
template <typename IO>
__global__ void __launch_bounds__(256) ssm_grads_kernel(SsmParams p, Sequences seqs, const float *states, const float *dstates, float *part_a, float *part_d)
{
    extern __shared__ float smem[];
    const int N = p.N, P = p.P, N1 = N + 1, P1 = P + 1 /* rows in shared memory, read across by lanes */, per = p.H / p.G, g = blockIdx.x % p.G, slot = blockIdx.x / p.G;
    int n = 0, hi = p.n_seq;   // the sequence whose first slot is the last one at or before this
    while (hi - n > 1) {
        const int mid = (n + hi) >> 1;
        if (seqs.start(mid) / QB + mid <= slot) n = mid;
        else hi = mid;
    }
    const int first = seqs.start(n), end = seqs.start(n + 1), c = slot - (first / QB + n), start = first + c * QB, m = min(QB, end - start);
    if (m <= 0) {
        for (int i = threadIdx.x; i < per; i += 256) part_a[(size_t)slot * p.H + g * per + i] = part_d[(size_t)slot * p.H + g * per + i] = 0.f;
        return;
    }
    float *qs = smem, *ks = qs + QB * N1, *dqs = ks + QB * N1, *dks = dqs + QB * N1, *vs = dks + QB * N1, *gs = vs + QB * P1;
    float *cb = gs + QB * P1;               // q_i . k_j             [QB][QB + 1]
    float *m1 = cb + QB * (QB + 1);        // L_ij dt_j (q_i . k_j)
    float *m2 = m1 + QB * (QB + 1);        // L_ij dt_j (do_i . v_j)
    float *rr = m2 + QB * (QB + 1);        // L_ij (q_i . k_j)(do_i . v_j)
    __shared__ float tS[32][33], tG[32][33];   // 32 x 32 of S and G: read by rows of lanes, which in memory would be a line per lane
    __shared__ double l[QB];
    __shared__ float dts[QB], ei[QB], ej[QB], xs[QB], zs[QB], red[8][2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < QB * N; i += 256) {
        const int t = i / N, x = i % N;
        qs[t * N1 + x] = t < m ? to_f32(static_cast<const IO *>(p.q)[(size_t)(start + t) * p.q_stride + g * N + x]) : 0.f;
        ks[t * N1 + x] = t < m ? to_f32(static_cast<const IO *>(p.k)[(size_t)(start + t) * p.k_stride + g * N + x]) : 0.f;
        dqs[t * N1 + x] = dks[t * N1 + x] = 0.f;
    }
    __syncthreads();
    for (int x = tid; x < QB * QB; x += 256) {
        const int i = x / QB, j = x % QB;
        float t = 0.f;
        for (int e = 0; e < N; ++e) t = fmaf(qs[i * N1 + e], ks[j * N1 + e], t);
        cb[i * (QB + 1) + j] = t;
    }
    for (int hh = 0; hh < per; ++hh) {
        const int h = g * per + hh;
        const float a = p.a[h], skip = p.skip ? p.skip[h] : 0.f;
        const float *S = states + ((size_t)slot * p.H + h) * N * P, *G = dstates + ((size_t)slot * p.H + h) * N * P;
        __syncthreads();
        if (warp == 0) {   // sums of log decays, in 64 bits: their differences are what counts
            const float d = lane < m ? p.dt[(size_t)(start + lane) * p.H + h] : 0.f;
            double s = (double)d * (double)a;
            if (s < -1e4) s = -1e4;   // (zero in fp32 all the same; a larger one would take the others' digits from the sums)
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += t;
            }
            const double all = __shfl_sync(0xffffffffu, s, 31);
            l[lane] = s;
            dts[lane] = d;
            ei[lane] = expf((float)s);
            ej[lane] = expf((float)(all - s));
        }
        float dd = 0.f;
        for (int i = tid; i < QB * P; i += 256) {
            const int t = i / P, x = i % P;
            const float vv = t < m ? to_f32(static_cast<const IO *>(p.v)[(size_t)(start + t) * p.v_stride + h * P + x]) : 0.f;
            const float go = t < m ? to_f32(static_cast<const IO *>(p.d_out)[((size_t)(start + t) * p.H + h) * P + x]) : 0.f;
            vs[t * P1 + x] = vv;
            gs[t * P1 + x] = go;
            dd = fmaf(vv, go, dd);
        }
        __syncthreads();
        for (int x = tid; x < QB * QB; x += 256) {
            const int i = x / QB, j = x % QB, at = i * (QB + 1) + j;
            float t = 0.f, e = 0.f;
            if (j <= i) {
                for (int y = 0; y < P; ++y) t = fmaf(gs[i * P1 + y], vs[j * P1 + y], t);
                e = expf((float)(l[i] - l[j]));
            }
            m1[at] = j <= i ? e * dts[j] * cb[at] : 0.f;   // (what lies above the diagonal may not be finite)
            m2[at] = e * dts[j] * t;
            rr[at] = j <= i ? e * cb[at] * t : 0.f;
        }
        __syncthreads();
        float sg = 0.f;   // <S, G>
        for (int i = tid; i < N * P; i += 256) sg = fmaf(S[i], G[i], sg);
        const int t0 = warp * 4;
        {   // dv, and k^T G v
            float z[4] = {0.f, 0.f, 0.f, 0.f};
            for (int x = lane; x < P; x += 32) {
                float u[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
                for (int e = 0; e < N; ++e) {
                    const float gg = G[(size_t)e * P + x];
#pragma unroll
                    for (int j = 0; j < 4; ++j) u[j] = fmaf(ks[(t0 + j) * N1 + e], gg, u[j]);
                }
                for (int i = t0; i < m; ++i) {
                    const float go = gs[i * P1 + x];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = fmaf(m1[i * (QB + 1) + t0 + j], go, w[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = t0 + j;
                    u[j] *= ej[t];
                    z[j] = fmaf(u[j], vs[t * P1 + x], z[j]);
                    if (t < m)
                        static_cast<IO *>(p.dv)[((size_t)(start + t) * p.H + h) * P + x] = from_f32<IO>(fmaf(skip, gs[t * P1 + x], fmaf(dts[t], u[j], w[j])));
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                for (int o = 16; o > 0; o >>= 1) z[j] += __shfl_xor_sync(0xffffffffu, z[j], o);
                if (lane == 0) zs[t0 + j] = z[j];   // z_j / dt_j
            }
        }
        {   // dq, dk, and q^T S do
            float z[4] = {0.f, 0.f, 0.f, 0.f};
            for (int x0 = 0; x0 < N; x0 += 32) {
                const int x = x0 + lane;
                float u[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f}, dq[4] = {0.f, 0.f, 0.f, 0.f}, dk[4] = {0.f, 0.f, 0.f, 0.f};
                for (int e0 = 0; e0 < P; e0 += 32) {
                    const int ne = min(32, P - e0);
                    __syncthreads();
                    for (int r = warp; r < 32; r += 8) {
                        const bool in = x0 + r < N && lane < ne;
                        tS[r][lane] = in ? S[(size_t)(x0 + r) * P + e0 + lane] : 0.f;
                        tG[r][lane] = in ? G[(size_t)(x0 + r) * P + e0 + lane] : 0.f;
                    }
                    __syncthreads();
                    for (int e = 0; e < ne; ++e) {
                        const float ss = tS[lane][e], gg = tG[lane][e];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            u[j] = fmaf(ss, gs[(t0 + j) * P1 + e0 + e], u[j]);
                            w[j] = fmaf(gg, vs[(t0 + j) * P1 + e0 + e], w[j]);
                        }
                    }
                }
                if (x >= N) continue;
                for (int i = 0; i < m; ++i) {
                    const float qq = qs[i * N1 + x], kk = ks[i * N1 + x];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (i >= t0 + j) dk[j] = fmaf(m2[i * (QB + 1) + t0 + j], qq, dk[j]);
                        if (i <= t0 + j) dq[j] = fmaf(m2[(t0 + j) * (QB + 1) + i], kk, dq[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = t0 + j;
                    u[j] *= ei[t];
                    z[j] = fmaf(u[j], qs[t * N1 + x], z[j]);
                    dqs[t * N1 + x] += u[j] + dq[j];
                    dks[t * N1 + x] += fmaf(dts[t] * ej[t], w[j], dk[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                for (int o = 16; o > 0; o >>= 1) z[j] += __shfl_xor_sync(0xffffffffu, z[j], o);
                if (lane == 0) xs[t0 + j] = z[j];
            }
        }
        for (int o = 16; o > 0; o >>= 1) {
            sg += __shfl_xor_sync(0xffffffffu, sg, o);
            dd += __shfl_xor_sync(0xffffffffu, dd, o);
        }
        if (lane == 0) {
            red[warp][0] = sg;
            red[warp][1] = dd;
        }
        __syncthreads();
        if (warp == 0) {   // a lane to a token
            sg = lane < 8 ? red[lane & 7][0] : 0.f;
            dd = lane < 8 ? red[lane & 7][1] : 0.f;
            for (int o = 4; o > 0; o >>= 1) {
                sg += __shfl_xor_sync(0xffffffffu, sg, o);
                dd += __shfl_xor_sync(0xffffffffu, dd, o);
            }
            sg = __shfl_sync(0xffffffffu, sg, 0);
            const float d = dts[lane];
            // F of a token is a sum of the terms that span it, i >= t > j, and of no others.  (Row sums less column sums come to the same, but in every
            // token before a large step that step's would have to cancel: with a step of 1e6 nothing is left of ddt there.)  So column j
            // becomes its sums from row i down, and a token adds up its row.
            float below = 0.f, span = 0.f;
            for (int i = QB - 1; i > 0; --i)
                if (i > lane) {
                    below += rr[i * (QB + 1) + lane];
                    rr[i * (QB + 1) + lane] = below;
                }
            __syncwarp();
            for (int j = 0; j < QB - 1; ++j)
                if (j < lane) span = fmaf(dts[j], rr[lane * (QB + 1) + j], span);
            const float direct = below + rr[lane * (QB + 1) + lane] + zs[lane];
            float suffix = xs[lane], before = d * zs[lane];
            for (int o = 1; o < 32; o <<= 1) {
                const float t = __shfl_down_sync(0xffffffffu, suffix, o), u = __shfl_up_sync(0xffffffffu, before, o);
                if (lane + o < 32) suffix += t;
                if (lane >= o) before += u;
            }
            before = __shfl_up_sync(0xffffffffu, before, 1);   // (of the tokens before this one alone)
            const float f = span + suffix + (lane ? before : 0.f) + expf((float)l[QB - 1]) * sg;
            if (lane < m) p.ddt[(size_t)(start + lane) * p.H + h] = fmaf(a, f, direct);
            float da = lane < m ? d * f : 0.f;
            for (int o = 16; o > 0; o >>= 1) da += __shfl_xor_sync(0xffffffffu, da, o);
            if (lane == 0) {
                part_a[(size_t)slot * p.H + h] = da;
                part_d[(size_t)slot * p.H + h] = dd;
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < m * N; i += 256) {
        const size_t at = ((size_t)(start + i / N) * p.G + g) * N + i % N;
        static_cast<IO *>(p.dq)[at] = from_f32<IO>(dqs[i / N * N1 + i % N]);
        static_cast<IO *>(p.dk)[at] = from_f32<IO>(dks[i / N * N1 + i % N]);
    }
}

__global__ void __launch_bounds__(512) ssm_reduce_kernel(const float *part_a, const float *part_d, int n, int H, float *da, float *dd)
{
    const bool second = blockIdx.y != 0;
    sum_partials(second ? part_d : part_a, n, H, [&](int i, float s) {
        if (!second) da[i] = s;
        else if (dd) dd[i] = s;
    });
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
static int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

template <typename F>
static cudaError_t with_rows(int N, F f)
{
    if (N <= 32) return f(std::integral_constant<int, 4>());
    if (N <= 64) return f(std::integral_constant<int, 8>());
    if (N <= 128) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

template <typename IO, typename OUT>
static cudaError_t ssm_scan_t(const SsmParams &p, cudaStream_t stream)
{
    const Sequences seqs = {p.cu_seqlens, p.T, p.n_seq};
    return with_rows(p.N, [&](auto R) {
        ssm_scan_kernel<IO, OUT, R()><<<(unsigned)p.n_seq * p.H * ceil_div(p.P, 16), 128, 0, stream>>>(p, seqs);
        count_launch(1);
        return cudaGetLastError();
    });
}
cudaError_t launch_ssm_scan(const SsmParams &p, int io_dtype, int out_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_F32) return out_dtype == KLA_F32 ? ssm_scan_t<float, float>(p, stream) : ssm_scan_t<float, __nv_bfloat16>(p, stream);
    return out_dtype == KLA_F32 ? ssm_scan_t<__nv_bfloat16, float>(p, stream) : ssm_scan_t<__nv_bfloat16, __nv_bfloat16>(p, stream);
}

template <typename IO, typename OUT>
static cudaError_t ssm_step_t(const SsmParams &p, cudaStream_t stream)
{
    return with_rows(p.N, [&](auto R) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)ceil_div((long long)p.rows * p.H * ceil_div(p.P, 16), 4));
        cfg.blockDim = dim3(128);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t err = cudaLaunchKernelEx(&cfg, ssm_step_kernel<IO, OUT, R()>, p);
        count_launch(1);
        return err != cudaSuccess ? err : cudaGetLastError();
    });
}
cudaError_t launch_ssm_step(const SsmParams &p, int io_dtype, int out_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_F32) return out_dtype == KLA_F32 ? ssm_step_t<float, float>(p, stream) : ssm_step_t<float, __nv_bfloat16>(p, stream);
    return out_dtype == KLA_F32 ? ssm_step_t<__nv_bfloat16, float>(p, stream) : ssm_step_t<__nv_bfloat16, __nv_bfloat16>(p, stream);
}

size_t ssm_bwd_workspace_bytes(int rows, int n_seq, int H, int G, int N, int P)
{
    const size_t slots = (size_t)rows / QB + n_seq;
    return slots * H * ((size_t)2 * N * P + 2) * sizeof(float);
}

cudaError_t launch_ssm_sums(const float *part_a, const float *part_d, int n, int H, float *da, float *dd, cudaStream_t stream)
{
    ssm_reduce_kernel<<<dim3((unsigned)ceil_div(H, 32), 2), 512, 0, stream>>>(part_a, part_d, n, H, da, dd);
    count_launch(1);
    return cudaGetLastError();
}

static size_t grads_smem(int N, int P) { return ((size_t)QB * (4 * (N + 1) + 2 * (P + 1)) + 4 * QB * (QB + 1)) * sizeof(float); }

template <typename IO>
static cudaError_t ssm_bwd_t(const SsmParams &p, cudaStream_t stream)
{
    const Sequences seqs = {p.cu_seqlens, p.T, p.n_seq};
    const size_t slots = (size_t)p.rows / QB + p.n_seq, units = slots * p.H * p.N * p.P;
    float *states = static_cast<float *>(p.workspace), *dstates = states + units, *part_a = dstates + units, *part_d = part_a + slots * p.H;
    cudaError_t err = with_rows(p.N, [&](auto R) {
        const unsigned grid = (unsigned)p.n_seq * p.H * ceil_div(p.P, 16);
        ssm_states_kernel<IO, R(), false><<<grid, 128, 0, stream>>>(p, seqs, states);
        ssm_states_kernel<IO, R(), true><<<grid, 128, 0, stream>>>(p, seqs, dstates);
        count_launch(2);
        return cudaGetLastError();
    });
    if (err != cudaSuccess) return err;
    // (the limit is the function's, not the call's: always that of the largest widths, so that a call on another host thread finds it high enough)
    err = cudaFuncSetAttribute(ssm_grads_kernel<IO>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)grads_smem(256, 256));
    if (err != cudaSuccess) return err;
    ssm_grads_kernel<IO><<<(unsigned)(slots * p.G), 256, grads_smem(p.N, p.P), stream>>>(p, seqs, states, dstates, part_a, part_d);
    count_launch(1);
    return launch_ssm_sums(part_a, part_d, (int)slots, p.H, p.da, p.dd, stream);
}
cudaError_t launch_ssm_bwd(const SsmParams &p, int io_dtype, cudaStream_t stream)
{
    return io_dtype == KLA_F32 ? ssm_bwd_t<float>(p, stream) : ssm_bwd_t<__nv_bfloat16>(p, stream);
}

}  // namespace kla
