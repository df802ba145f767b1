// Short causal depthwise convolution over packed or fixed-length sequences, with SiLU: forward, backward and one token.
//
//   p_t[c] = b[c] + sum_{i < W} w[c][i] x_{t-W+1+i}[c]     (inputs before a sequence's first token: its state, else zeros)
//   y_t = p_t sigmoid(p_t)                                  (KLA_FLAG_CONV_LINEAR: y_t = p_t)
//
// Backward, with g_t = dy_t act'(p_t):   dx_t = sum_i w[i] g_{t+W-1-i} (tokens of the same sequence), plus the final state's gradient
// for the last W - 1 tokens;  dw[c][i] = sum_t g_t x_{t-W+1+i};  db = sum_t g_t.
//
// 8 x 4096 tokens of 2304 channels, 4 taps, bf16: 82 us, 3.7 TB/s (46 us by its bytes); backward of 16 packed sequences, 363 MB: 123 us.  Forward: bound by
// the wait for loads, of which three blocks of 80 registers hold too few in flight (instructions issue in 43 % of the cycles, 7 of 12 stalled warps of
// an issue wait for memory; the exponential and the reciprocal of a value keep their unit 45 % busy, 34 us of 75 M values).  Backward: by the latency of
// arithmetic on four warps per scheduler (issue 55 %, 0.5 waiting for memory); its SMs work 79 % of the time (594 blocks for 592 places of two rounds).
// A thread owns four neighbouring channels as two pairs (packed arithmetic) and walks a run of tokens with the window in registers, so a value is loaded
// once, but for the W - 1 before (backward: and behind) its run; eight rows (backward: four) are in flight while the last ones are worked on.
// Rows between a sequence's border and a run's end take a loop of their own, so that the others' code is straight.
#include "layer_ops.h"
#include "layer_pieces.cuh"
#include "scan_pieces.cuh"

namespace kla {

__device__ __forceinline__ float2 sigmoid2(float2 x)
{
    const float2 t = mul2(x, f2(-1.4426950408889634f));
    const float2 d = add2(f2(exp2_fast(t.x), exp2_fast(t.y)), f2(1.f));
    return f2(rcp_fast(d.x), rcp_fast(d.y));
}

template <typename IO, int VEC>
__device__ __forceinline__ void load_or_zero(Pack<IO, VEC> &x, const IO *p)
{
    if (p) x.load(p);
    else x.zero();
}

// Row `pos` of a sequence as the window sees it: pos >= 0 a token, pos < 0 a row of its state.
template <typename IO, int VEC>
__device__ __forceinline__ void window_row(Pack<IO, VEC> &x, const ConvParams &p, int seq, int start, int pos, int c)
{
    const IO *init = static_cast<const IO *>(p.init_state);
    const int W1 = p.taps - 1;
    load_or_zero(x, pos >= 0 ? static_cast<const IO *>(p.x) + (size_t)(start + pos) * p.x_stride + c
                   : init    ? init + ((size_t)seq * W1 + W1 + pos) * p.C + c
                             : nullptr);
}

// The last W - 1 rows of sequence n's window, whatever its length.  (final_state may be init_state: row i is written after row i + len is read.)
template <typename IO, int W, int VEC>
__device__ __forceinline__ void last_rows(const ConvParams &p, const Sequences &seqs, int n, int c)
{
    const int start = seqs.start(n), len = seqs.start(n + 1) - start;
    Pack<IO, VEC> x;
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
        window_row<IO, VEC>(x, p, n, start, len - (W - 1) + i, c);
        x.store(static_cast<IO *>(p.final_state) + ((size_t)n * (W - 1) + i) * p.C + c);
    }
}

// Any number of channels, any stride: a thread to a channel.  Units of work: (run of tokens, channel), then, where a final state is wanted,
// (sequence, channel).
template <typename IO, int W, bool SILU>
__global__ void __launch_bounds__(256) conv_fwd1_kernel(ConvParams p, Sequences seqs, int run, int n_runs)
{
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x, job = unit / p.C;
    const int c = (int)(unit % p.C);
    if (job >= n_runs) {
        if (p.final_state && job - n_runs < p.n_seq) last_rows<IO, W, 1>(p, seqs, (int)(job - n_runs), c);
        return;
    }
    const int r0 = (int)job * run, r1 = min(p.rows, r0 + run);
    float w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = p.weight[(size_t)c * W + i];
    const float b = p.bias ? p.bias[c] : 0.f;
    int seq = seqs.of_row(r0), start = seqs.start(seq), end = seqs.start(seq + 1);
    float win[W - 1];
    auto fill = [&](int pos) {   // the window before token `pos`
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            Pack<IO, 1> x;
            window_row<IO, 1>(x, p, seq, start, pos - (W - 1) + i, c);
            win[i] = x.get(0);
        }
    };
    fill(r0 - start);
    const IO *xp = static_cast<const IO *>(p.x) + c;
    IO *yp = static_cast<IO *>(p.out) + c;
    constexpr int AHEAD = 8;   // rows in flight
    for (int r = r0; r < r1; r += AHEAD) {
        float raw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (r + j < r1) raw[j] = to_f32(xp[(size_t)(r + j) * p.x_stride]);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (r + j >= r1) break;
            if (r + j == end) {
                do {
                    ++seq;
                    start = end;
                    end = seqs.start(seq + 1);
                } while (end == start && seq + 1 < p.n_seq);
                fill(0);
            }
            float s = b;
#pragma unroll
            for (int i = 0; i < W - 1; ++i) s = fmaf(w[i], win[i], s);
            s = fmaf(w[W - 1], raw[j], s);
            yp[(size_t)(r + j) * p.C] = from_f32<IO>(SILU ? s * sigmoid(s) : s);
#pragma unroll
            for (int i = 0; i + 1 < W - 1; ++i) win[i] = win[i + 1];
            win[W - 2] = raw[j];
        }
    }
}

// The same for four channels to a thread, in pairs.
template <typename IO, int W, bool SILU>
__global__ void __launch_bounds__(256, 3) conv_fwd4_kernel(ConvParams p, Sequences seqs, int run, int n_runs)
{
    const int nvec = p.C / 4;
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(unit % nvec) * 4;
    const long long job = unit / nvec;
    if (job >= n_runs) {
        if (p.final_state && job - n_runs < p.n_seq) last_rows<IO, W, 4>(p, seqs, (int)(job - n_runs), c);
        return;
    }
    const int r0 = (int)job * run, r1 = min(p.rows, r0 + run);
    const IO *xp = static_cast<const IO *>(p.x) + (size_t)r0 * p.x_stride + c;
    IO *yp = static_cast<IO *>(p.out) + (size_t)r0 * p.C + c;
    constexpr int AHEAD = sizeof(IO) == 2 ? 8 : 4;   // rows in flight
    Pack<IO, 4> raw[AHEAD], next[AHEAD];
    auto request = [&](int r, Pack<IO, 4> (&to)[AHEAD]) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (r + j < r1) to[j].load(xp + (size_t)(r + j - r0) * p.x_stride);
    };
    request(r0, raw);
    float2 w[W][2], b[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        b[e] = p.bias ? f2(p.bias[c + 2 * e], p.bias[c + 2 * e + 1]) : f2(0.f);
#pragma unroll
        for (int i = 0; i < W; ++i) w[i][e] = f2(p.weight[(size_t)(c + 2 * e) * W + i], p.weight[(size_t)(c + 2 * e + 1) * W + i]);
    }
    int seq = seqs.of_row(r0), start = seqs.start(seq), end = seqs.start(seq + 1);
    float2 win[W - 1][2];
    auto fill = [&](int pos) {   // the window before token `pos`
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            Pack<IO, 4> x;
            window_row<IO, 4>(x, p, seq, start, pos - (W - 1) + i, c);
            win[i][0] = f2(x.get(0), x.get(1));
            win[i][1] = f2(x.get(2), x.get(3));
        }
    };
    fill(r0 - start);
    auto token = [&](const Pack<IO, 4> &raw, IO *to) {
        float2 x[2] = {f2(raw.get(0), raw.get(1)), f2(raw.get(2), raw.get(3))};
        float y[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float2 s = b[e];
#pragma unroll
            for (int i = 0; i < W - 1; ++i) s = fma2(w[i][e], win[i][e], s);
            s = fma2(w[W - 1][e], x[e], s);
            if (SILU) s = mul2(s, sigmoid2(s));
            y[2 * e] = s.x;
            y[2 * e + 1] = s.y;
#pragma unroll
            for (int i = 0; i + 1 < W - 1; ++i) win[i][e] = win[i + 1][e];
            win[W - 2][e] = x[e];
        }
        Pack<IO, 4> o;
        o.set(y);
        o.store(to);
    };
#pragma unroll 1
    for (int r = r0; r < r1; r += AHEAD) {
        request(r + AHEAD, next);
        IO *to = yp + (size_t)(r - r0) * p.C;
        if (r + AHEAD <= min(r1, end)) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) token(raw[j], to + (size_t)j * p.C);
        } else {
#pragma unroll 1
            for (int j = 0; j < AHEAD; ++j) {
                if (r + j >= r1) break;
                if (r + j == end) {
                    do {
                        ++seq;
                        start = end;
                        end = seqs.start(seq + 1);
                    } while (end == start && seq + 1 < p.n_seq);
                    fill(0);
                }
                Pack<IO, 4> x;
                x.load(xp + (size_t)(r + j - r0) * p.x_stride);
                token(x, to + (size_t)j * p.C);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) raw[j] = next[j];
    }
}

// One thread: VEC channels of one sequence's next token; the window moves on by one row.
template <typename IO, int W, int VEC, bool SILU>
__global__ void __launch_bounds__(128) conv_step_kernel(ConvParams p)
{
    const int nvec = p.C / VEC;
    const long long unit = (long long)blockIdx.x * 128 + threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // what the previous kernel on the stream wrote may be read here
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (unit >= (long long)p.rows * nvec) return;
    const int c = (int)(unit % nvec) * VEC;
    const size_t n = (size_t)(unit / nvec);
    IO *state = static_cast<IO *>(p.final_state) + n * (W - 1) * p.C + c;
    Pack<IO, VEC> x[W];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) x[i].load(state + (size_t)i * p.C);
    x[W - 1].load(static_cast<const IO *>(p.x) + n * p.x_stride + c);
    float y[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        float s = p.bias ? p.bias[c + e] : 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s = fmaf(p.weight[(size_t)(c + e) * W + i], x[i].get(e), s);
        y[e] = SILU ? s * sigmoid(s) : s;
    }
    Pack<IO, VEC> o;
    o.set(y);
    o.store(static_cast<IO *>(p.out) + n * p.C + c);
#pragma unroll
    for (int i = 0; i < W - 1; ++i) x[i + 1].store(state + (size_t)i * p.C);
}

// Any number of channels, any stride: a thread to a channel.  A block: 32 channels and the rows [y rows_per, ..), an eighth of them to each of its
// warps.  The sums over rows stay in registers, then the warps' are added in shared memory and leave as one partial of [W + 1][C] per block row;
// conv_reduce_kernel adds those in order.
template <typename IO, int W, bool SILU>
__global__ void __launch_bounds__(256) conv_bwd1_kernel(ConvParams p, Sequences seqs, int rows_per)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int b0 = blockIdx.y * rows_per, b1 = min(p.rows, b0 + rows_per);
    const int sub = (rows_per + 7) / 8;
    const int r0 = min(b1, b0 + warp * sub), r1 = min(b1, r0 + sub);
    float dw[W], db = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) dw[i] = 0.f;
    if (r0 < r1 && c < p.C) {
        float w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = p.weight[(size_t)c * W + i];
        const float b = p.bias ? p.bias[c] : 0.f;
        int seq = seqs.of_row(r0), start = seqs.start(seq), end = seqs.start(seq + 1);
        float win[W - 1], acc[W];   // acc[s]: gradient of row t - s so far
        auto fill = [&](int pos) {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                Pack<IO, 1> x;
                window_row<IO, 1>(x, p, seq, start, pos - (W - 1) + i, c);
                win[i] = x.get(0);
            }
        };
        fill(r0 - start);
#pragma unroll
        for (int s = 0; s < W; ++s) acc[s] = 0.f;
        const IO *xp = static_cast<const IO *>(p.x) + c, *gp = static_cast<const IO *>(p.d_out) + c, *fp = static_cast<const IO *>(p.d_final);
        IO *dxp = static_cast<IO *>(p.dx) + c;
        const int last = r1 + W - 1;   // the rows behind the run whose windows reach into it
        constexpr int AHEAD = 4;
        for (int t0 = r0; t0 < last; t0 += AHEAD) {
            float xr[AHEAD], gr[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (t0 + j < last && t0 + j < p.rows) {
                    xr[j] = to_f32(xp[(size_t)(t0 + j) * p.x_stride]);
                    gr[j] = to_f32(gp[(size_t)(t0 + j) * p.C]);
                }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int t = t0 + j;
                if (t >= last) break;
#pragma unroll
                for (int s = W - 1; s > 0; --s) acc[s] = acc[s - 1];
                acc[0] = 0.f;
                if (t < p.rows) {
                    if (t == end) {
                        do {
                            ++seq;
                            start = end;
                            end = seqs.start(seq + 1);
                        } while (end == start && seq + 1 < p.n_seq);
                        fill(0);
                    }
                    if (fp && t >= end - (W - 1)) acc[0] = to_f32(fp[((size_t)seq * (W - 1) + (t - (end - (W - 1)))) * p.C + c]);
                    float g = gr[j];
                    if (SILU) {
                        float s = b;
#pragma unroll
                        for (int i = 0; i < W - 1; ++i) s = fmaf(w[i], win[i], s);
                        s = fmaf(w[W - 1], xr[j], s);
                        const float sig = sigmoid(s);
                        g *= sig * fmaf(s, 1.f - sig, 1.f);
                    }
                    if (t < r1) {
                        db += g;
#pragma unroll
                        for (int i = 0; i < W - 1; ++i) dw[i] = fmaf(g, win[i], dw[i]);
                        dw[W - 1] = fmaf(g, xr[j], dw[W - 1]);
                    }
#pragma unroll
                    for (int s = 0; s < W; ++s)
                        if (s <= t - start) acc[s] = fmaf(w[W - 1 - s], g, acc[s]);
#pragma unroll
                    for (int i = 0; i + 1 < W - 1; ++i) win[i] = win[i + 1];
                    win[W - 2] = xr[j];
                }
                const int done = t - (W - 1);   // (below r1: t is below r1 + W - 1)
                if (done >= r0) dxp[(size_t)done * p.C] = from_f32<IO>(acc[W - 1]);
            }
        }
    }
    __shared__ float sums[8][32];
#pragma unroll
    for (int i = 0; i <= W; ++i) {
        __syncthreads();
        sums[warp][lane] = i < W ? dw[i < W ? i : 0] : db;
        __syncthreads();
        if (warp == 0 && c < p.C) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += sums[k][lane];
            p.partial[((size_t)blockIdx.y * (W + 1) + i) * p.C + c] = s;
        }
    }
}

// Four channels to a thread, in pairs; otherwise as conv_bwd1_kernel.
template <typename IO, int W, bool SILU>
__global__ void __launch_bounds__(256, 2) conv_bwd4_kernel(ConvParams p, Sequences seqs, int rows_per)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = (blockIdx.x * 32 + lane) * 4;
    const int b0 = blockIdx.y * rows_per, b1 = min(p.rows, b0 + rows_per);
    const int sub = (rows_per + 7) / 8;
    const int r0 = min(b1, b0 + warp * sub), r1 = min(b1, r0 + sub);
    float2 dw[W][2], db[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        db[e] = f2(0.f);
#pragma unroll
        for (int i = 0; i < W; ++i) dw[i][e] = f2(0.f);
    }
    if (r0 < r1 && c < p.C) {
        float2 w[W][2], b[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            b[e] = p.bias ? f2(p.bias[c + 2 * e], p.bias[c + 2 * e + 1]) : f2(0.f);
#pragma unroll
            for (int i = 0; i < W; ++i) w[i][e] = f2(p.weight[(size_t)(c + 2 * e) * W + i], p.weight[(size_t)(c + 2 * e + 1) * W + i]);
        }
        int seq = seqs.of_row(r0), start = seqs.start(seq), end = seqs.start(seq + 1);
        float2 win[W - 1][2], acc[W - 1][2];   // acc[s]: gradient of row t - 1 - s so far, before row t
        auto fill = [&](int pos) {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                Pack<IO, 4> x;
                window_row<IO, 4>(x, p, seq, start, pos - (W - 1) + i, c);
                win[i][0] = f2(x.get(0), x.get(1));
                win[i][1] = f2(x.get(2), x.get(3));
            }
        };
        fill(r0 - start);
#pragma unroll
        for (int s = 0; s < W - 1; ++s) acc[s][0] = acc[s][1] = f2(0.f);
        const IO *xp = static_cast<const IO *>(p.x) + c, *gp = static_cast<const IO *>(p.d_out) + c, *fp = static_cast<const IO *>(p.d_final);
        IO *dxp = static_cast<IO *>(p.dx) + c;
        const int last = r1 + W - 1, stop = min(last, p.rows);   // the rows behind the run whose windows reach into it
        auto emit = [&](int row, const float2 (&x)[2]) {
            if (row < r0) return;
            const float y[4] = {x[0].x, x[0].y, x[1].x, x[1].y};
            Pack<IO, 4> o;
            o.set(y);
            o.store(dxp + (size_t)row * p.C);
        };
        // Row t: its gradient g of p_t, what it adds to the W - 1 rows before it (as far as `reach` of them belong to its sequence) and to itself.
        auto token = [&](int t, const Pack<IO, 4> &xr, const Pack<IO, 4> &gr, const float2 (&first)[2], int reach, bool mine) {
            const float2 x[2] = {f2(xr.get(0), xr.get(1)), f2(xr.get(2), xr.get(3))}, go[2] = {f2(gr.get(0), gr.get(1)), f2(gr.get(2), gr.get(3))};
            float2 done[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float2 g = go[e];
                if (SILU) {
                    float2 s = b[e];
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) s = fma2(w[i][e], win[i][e], s);
                    s = fma2(w[W - 1][e], x[e], s);
                    const float2 sig = sigmoid2(s);
                    g = mul2(g, mul2(sig, fma2(s, fma2(sig, f2(-1.f), f2(1.f)), f2(1.f))));
                }
                if (mine) {
                    db[e] = add2(db[e], g);
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) dw[i][e] = fma2(g, win[i][e], dw[i][e]);
                    dw[W - 1][e] = fma2(g, x[e], dw[W - 1][e]);
                }
#pragma unroll
                for (int s = 0; s < W - 1; ++s)
                    if (s < reach) acc[s][e] = fma2(w[W - 2 - s][e], g, acc[s][e]);
                done[e] = acc[W - 2][e];
#pragma unroll
                for (int s = W - 2; s > 0; --s) acc[s][e] = acc[s - 1][e];
                acc[0][e] = fma2(w[W - 1][e], g, first[e]);
#pragma unroll
                for (int i = 0; i + 1 < W - 1; ++i) win[i][e] = win[i + 1][e];
                win[W - 2][e] = x[e];
            }
            emit(t - (W - 1), done);
        };
        constexpr int AHEAD = sizeof(IO) == 2 ? 4 : 2;
        Pack<IO, 4> xr[AHEAD], gr[AHEAD], xn[AHEAD], gn[AHEAD];
        auto request = [&](int t, Pack<IO, 4> (&x)[AHEAD], Pack<IO, 4> (&g)[AHEAD]) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (t + j < stop) {
                    x[j].load(xp + (size_t)(t + j) * p.x_stride);
                    g[j].load(gp + (size_t)(t + j) * p.C);
                }
        };
        request(r0, xr, gr);
#pragma unroll 1
        for (int t0 = r0; t0 < stop; t0 += AHEAD) {
            request(t0 + AHEAD, xn, gn);
            const float2 none[2] = {f2(0.f), f2(0.f)};
            // (a sequence's first W - 1 rows reach behind its start, its last W - 1 have the final state's gradient)
            if (t0 + AHEAD <= r1 && t0 - start >= W - 1 && t0 + AHEAD <= (fp ? end - (W - 1) : end)) {
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) token(t0 + j, xr[j], gr[j], none, W, true);
            } else {
#pragma unroll 1
                for (int j = 0; j < AHEAD; ++j) {
                    const int t = t0 + j;
                    if (t >= stop) break;
                    if (t == end) {
                        do {
                            ++seq;
                            start = end;
                            end = seqs.start(seq + 1);
                        } while (end == start && seq + 1 < p.n_seq);
                        fill(0);
                    }
                    float2 first[2] = {f2(0.f), f2(0.f)};
                    if (fp && t >= end - (W - 1)) {
                        Pack<IO, 4> f;
                        f.load(fp + ((size_t)seq * (W - 1) + (t - (end - (W - 1)))) * p.C + c);
                        first[0] = f2(f.get(0), f.get(1));
                        first[1] = f2(f.get(2), f.get(3));
                    }
                    Pack<IO, 4> x, g;
                    x.load(xp + (size_t)t * p.x_stride);
                    g.load(gp + (size_t)t * p.C);
                    token(t, x, g, first, t - start, t < r1);
                }
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                xr[j] = xn[j];
                gr[j] = gn[j];
            }
        }
#pragma unroll
        for (int s = W - 2; s >= 0; --s)   // rows whose later neighbours do not exist (r1 within W - 1 of the end)
            if (stop - 1 - s < r1 && stop - 1 - s > stop - W) emit(stop - 1 - s, acc[s]);
    }
    __shared__ float2 sums[8][64];
#pragma unroll
    for (int i = 0; i <= W; ++i) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e) sums[warp][lane * 2 + e] = i < W ? dw[i < W ? i : 0][e] : db[e];
        __syncthreads();
        if (threadIdx.x < 64) {
            const int ch = blockIdx.x * 128 + 2 * threadIdx.x;
            if (ch < p.C) {
                float2 s = f2(0.f);
#pragma unroll
                for (int k = 0; k < 8; ++k) s = add2(s, sums[k][threadIdx.x]);
                *reinterpret_cast<float2 *>(p.partial + ((size_t)blockIdx.y * (W + 1) + i) * p.C + ch) = s;
            }
        }
    }
}

__global__ void __launch_bounds__(512) conv_reduce_kernel(const float *partial, int n, int W, int C, float *dweight, float *dbias)
{
    sum_partials(partial, n, (W + 1) * C, [&](int i, float s) {
        const int tap = i / C, c = i % C;
        if (tap < W) dweight[(size_t)c * W + tap] = s;
        else if (dbias) dbias[c] = s;
    });
}

// Gradient of the states: one thread per (sequence, channel); the first W - 1 tokens' windows reach into the state, and in a sequence
// shorter than that the final state's gradient does too.
template <typename IO, int W, bool SILU>
__global__ void __launch_bounds__(256) conv_dinit_kernel(ConvParams p, Sequences seqs)
{
    const long long unit = (long long)blockIdx.x * 256 + threadIdx.x;
    if (unit >= (long long)p.n_seq * p.C) return;
    const int n = (int)(unit / p.C), c = (int)(unit % p.C);
    const int start = seqs.start(n), len = seqs.start(n + 1) - start;
    float d[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        d[j] = p.d_final && j >= len ? to_f32(static_cast<const IO *>(p.d_final)[((size_t)n * (W - 1) + j - len) * p.C + c]) : 0.f;
#pragma unroll
    for (int t = 0; t < W - 1; ++t) {
        if (t >= len) break;
        float s = p.bias ? p.bias[c] : 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            Pack<IO, 1> x;
            window_row<IO, 1>(x, p, n, start, t - (W - 1) + i, c);
            s = fmaf(p.weight[(size_t)c * W + i], x.get(0), s);
        }
        float g = to_f32(static_cast<const IO *>(p.d_out)[(size_t)(start + t) * p.C + c]);
        if (SILU) {
            const float sig = sigmoid(s);
            g *= sig * fmaf(s, 1.f - sig, 1.f);
        }
#pragma unroll
        for (int j = t; j < W - 1; ++j) d[j] = fmaf(p.weight[(size_t)c * W + j - t], g, d[j]);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) static_cast<IO *>(p.dinit)[((size_t)n * (W - 1) + j) * p.C + c] = from_f32<IO>(d[j]);
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
static int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

template <typename F>
static cudaError_t with_taps(int taps, bool silu, F f)
{
    using std::integral_constant;
    switch (taps * 2 + (silu ? 1 : 0)) {
        case 4: return f(integral_constant<int, 2>(), integral_constant<bool, false>());
        case 5: return f(integral_constant<int, 2>(), integral_constant<bool, true>());
        case 6: return f(integral_constant<int, 3>(), integral_constant<bool, false>());
        case 7: return f(integral_constant<int, 3>(), integral_constant<bool, true>());
        case 8: return f(integral_constant<int, 4>(), integral_constant<bool, false>());
        default: return f(integral_constant<int, 4>(), integral_constant<bool, true>());
    }
}

template <typename IO, int VEC>
static cudaError_t conv_fwd_v(const ConvParams &all, cudaStream_t stream)
{
    ConvParams p = all;
    // A state updated in place is written once the runs, which read it, are done.
    const bool in_place = p.final_state && p.final_state == p.init_state && p.rows > 0;
    if (in_place) p.final_state = nullptr;
    const Sequences seqs = {p.cu_seqlens, p.T, p.n_seq};
    const int nvec = p.C / VEC;
    // Runs as long as give every SM its three blocks once (a second wave would be a short one), no shorter than 8 rows: the rows before a run
    // are loaded twice.  B8 T4096 C2304: runs of 40 rows 90 us, of 166 82.
    long long run = ((long long)p.rows * nvec + (long long)sm_count() * 768 - 1) / ((long long)sm_count() * 768);
    run = run < 8 ? 8 : run;
    const int n_runs = ceil_div(p.rows, run);
    const long long units = ((long long)n_runs + (p.final_state ? p.n_seq : 0)) * nvec;
    if (units == 0) return cudaSuccess;
    const cudaError_t err = with_taps(p.taps, p.silu, [&](auto W, auto SILU) {
        if constexpr (VEC == 4) conv_fwd4_kernel<IO, W(), SILU()><<<ceil_div(units, 256), 256, 0, stream>>>(p, seqs, (int)run, n_runs);
        else conv_fwd1_kernel<IO, W(), SILU()><<<ceil_div(units, 256), 256, 0, stream>>>(p, seqs, (int)run, n_runs);
        count_launch(1);
        return cudaGetLastError();
    });
    if (err != cudaSuccess || !in_place) return err;
    p.final_state = all.final_state;
    p.rows = 0;   // (the states alone)
    return conv_fwd_v<IO, VEC>(p, stream);
}

template <typename IO, int VEC>
static cudaError_t conv_step_v(const ConvParams &p, cudaStream_t stream)
{
    const long long units = (long long)p.rows * (p.C / VEC);
    if (units == 0) return cudaSuccess;
    return with_taps(p.taps, p.silu, [&](auto W, auto SILU) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)ceil_div(units, 128));
        cfg.blockDim = dim3(128);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t err = cudaLaunchKernelEx(&cfg, conv_step_kernel<IO, W(), VEC, SILU()>, p);
        count_launch(1);
        return err != cudaSuccess ? err : cudaGetLastError();
    });
}

// Rows of the grid of the backward: enough blocks for four on every SM, none with fewer than 64 rows.
static int conv_bwd_rows(int C, int vec, int rows)
{
    const int cols = ceil_div(C, 32 * vec);
    int ny = ceil_div(4LL * sm_count(), cols);
    const int most = ceil_div(rows, 64);
    return ny < 1 ? 1 : ny > most ? (most < 1 ? 1 : most) : ny;
}

template <typename IO, int VEC>
static cudaError_t conv_bwd_v(const ConvParams &p, cudaStream_t stream)
{
    const Sequences seqs = {p.cu_seqlens, p.T, p.n_seq};
    const int ny = conv_bwd_rows(p.C, VEC, p.rows), per = p.rows ? ceil_div(p.rows, ny) : 1;
    return with_taps(p.taps, p.silu, [&](auto W, auto SILU) {
        const dim3 grid((unsigned)ceil_div(p.C, 32 * VEC), (unsigned)ny);
        if constexpr (VEC == 4) conv_bwd4_kernel<IO, W(), SILU()><<<grid, 256, 0, stream>>>(p, seqs, per);
        else conv_bwd1_kernel<IO, W(), SILU()><<<grid, 256, 0, stream>>>(p, seqs, per);
        conv_reduce_kernel<<<ceil_div((long long)(W() + 1) * p.C, 32), 512, 0, stream>>>(p.partial, ny, W(), p.C, p.dweight, p.dbias);
        count_launch(2);
        if (p.dinit) {
            conv_dinit_kernel<IO, W(), SILU()><<<ceil_div((long long)p.n_seq * p.C, 256), 256, 0, stream>>>(p, seqs);
            count_launch(1);
        }
        return cudaGetLastError();
    });
}

// Channels of a thread: four where rows start on a boundary of four, else one.
static bool whole_packs(const ConvParams &p, int vec, int io_dtype)
{
    const int bytes = io_dtype == KLA_BF16 ? 2 : 4;
    const size_t to = (size_t)vec * bytes;
    return p.C % vec == 0 && (size_t)p.x_stride * bytes % to == 0;
}

size_t conv_bwd_workspace_bytes(int C, int taps, int rows)
{
    const int a = conv_bwd_rows(C, 4, rows), b = conv_bwd_rows(C, 1, rows);
    return (size_t)(a > b ? a : b) * (taps + 1) * C * sizeof(float);
}
cudaError_t launch_conv_fwd(const ConvParams &p, int io_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_BF16) return whole_packs(p, 4, io_dtype) ? conv_fwd_v<__nv_bfloat16, 4>(p, stream) : conv_fwd_v<__nv_bfloat16, 1>(p, stream);
    return whole_packs(p, 4, io_dtype) ? conv_fwd_v<float, 4>(p, stream) : conv_fwd_v<float, 1>(p, stream);
}
cudaError_t launch_conv_step(const ConvParams &p, int io_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_BF16) return whole_packs(p, 4, io_dtype) ? conv_step_v<__nv_bfloat16, 4>(p, stream) : conv_step_v<__nv_bfloat16, 1>(p, stream);
    return whole_packs(p, 4, io_dtype) ? conv_step_v<float, 4>(p, stream) : conv_step_v<float, 1>(p, stream);
}
cudaError_t launch_conv_bwd(const ConvParams &p, int io_dtype, cudaStream_t stream)
{
    if (io_dtype == KLA_BF16) return whole_packs(p, 4, io_dtype) ? conv_bwd_v<__nv_bfloat16, 4>(p, stream) : conv_bwd_v<__nv_bfloat16, 1>(p, stream);
    return whole_packs(p, 4, io_dtype) ? conv_bwd_v<float, 4>(p, stream) : conv_bwd_v<float, 1>(p, stream);
}

}  // namespace kla
