// Selective state space scan by chunks of 128 tokens on the tensor cores: bf16 q, k, v, N = d_k of 64 or 128, P = d_v in slices of 64.
//
// With l_i the sum of dt a up to and with token i of a chunk, L_ij = exp(l_i - l_j) for j <= i, S the state before the chunk:
//
//     o_i = e^{l_i} S^T q_i + sum_{j <= i} (q_i . k_j) L_ij dt_j v_j + d v_i
//     S'  = e^{l_Q} S + sum_j k_j (dt_j e^{l_Q - l_j} v_j)^T
//
// One block per (sequence, head, 64 columns of v) walks the chunks with the state in registers, so nothing but inputs and outputs
// touches memory.  Unlike the delta rule nothing has to be solved: of a chunk's four products three do not depend on the state, and the
// chain from state to state is one fp32 operation per element.  Roles, connected by mbarriers:
//
//   decay (4 warps)    the exponentials of sums of dt a, a chunk ahead
//   state (8 warps)    w_j v_j as an operand; S' in fp32; S as an operand
//   output (8 warps)   P_ij = (q_i . k_j) L_ij dt_j as an operand; o from the accumulators
//   issue (1 warp)     tcgen05: q k^T (128 x 128 x N), q [S_hi | S_lo] (128 x 128 x N), k^T [w v in three parts] (N x 192 x 128),
//                      P v (128 x 64 x 128); with PARTS of S and P
//   load (1 warp)      TMA, each tile as soon as the last product that reads it is done
//
// Precision.  q, k, v are exact operands.  What a chunk adds to the state is summed from w v in three bf16 parts (24 bits) and joins the
// state in one fp32 operation, so the state is fp32 (its parts are summed apart, smallest first: the tensor core truncates sums).
// P and the S of the read-out are one bf16 each where o is bf16 (each term is then off by at most 2^-8 of itself, as o is by its own
// rounding; measured, the 2-norm error of o goes from 1.7e-3, the rounding, to at most 1.4 times that) and pairs (16 bits) where o is fp32.
//
// Decays are products of exponentials of sums that do not exceed zero (for a < 0): inside a block of 32 tokens one exponential per
// element, between blocks the product of a factor per row, one per pair of blocks and one per column, which costs two multiplications.
//
// What bounds it: the port of the shared memory.  A working SM takes 5 200 cycles for a chunk at N = 128, of which by count the products' operands take 1 920,
// the loads' tiles 640, and the roles' own reads and writes 2 300.  (On 8 x 4096 tokens of 32 heads, 200 us, the SMs work 83 % of the time: 256 blocks
// on 148 SMs.)  P of the next chunk formed before the outputs of the last, with P and q S there twice and k once,
// 209 us for 201 on 8 x 4096 tokens of 32 heads (k comes too late); what helped last were accesses: one arrival per warp at a barrier and outputs staged without
// bank conflicts (201 -> 196).
//
// Few long sequences are cut into parts that run side by side: a first pass forms what each part adds to a state of zero and its whole
// decay, ssm_parts_kernel chains them, and the main pass starts every part from its true state.  The decay is a scalar per
// head, so that the chain needs no products (the delta rule's segments need whole transition maps).
#include <mutex>

#include "ssm_pieces.cuh"

namespace kla {
namespace ssm {

namespace {

constexpr int STATE_T = 256, OUT_T = 256, DECAY_T = 128;
constexpr int T_DECAY = STATE_T + OUT_T, T_ISSUE = T_DECAY + DECAY_T, NT = T_ISSUE + 128;   // (of the last warpgroup two warps work: issue, load)

// Barriers; those of a stage (of k and v) are followed by that of the second one.
enum Bar {
    B_K = 0,        // + stage: tiles of k landed
    B_X = 2,        // + stage: the tile of v landed
    B_Q = 4,
    B_TOT,          // sums over 32 tokens written
    B_W,            // weights written
    B_SCAL,         // scalars for the output role written
    B_CLEAN,        // rows behind the sequence's end zeroed
    B_WX0, B_WX1,   // w v of tokens 0 .. 63, 64 .. 127 written
    B_S,            // parts of the state written
    B_JOIN,         // what a chunk adds has been read
    B_P,            // P written
    B_YFREE,        // accumulators of o read
    B_CB,           // q k^T complete
    B_Y1,           // + stage: q S complete
    B_DS0 = B_Y1 + 2,   // + stage: k^T [w v] of tokens 0 .. 63 complete
    B_DS1 = B_DS0 + 2,  // + stage: of all tokens
    B_Y2 = B_DS1 + 2,   // + stage: P v complete
    B_COUNT = B_Y2 + 2
};

// Tensor memory: q k^T (128 columns), k^T [w v] (64 for each part), q S (64 for each part), P v (64).
constexpr uint32_t TM_CB = 0, TM_DS = 128, TM_Y1 = 320;
template <int PARTS>
constexpr uint32_t TM_Y2 = TM_Y1 + 64 * PARTS;

// PARTS of S and P as operands.  One: the shared memory of the second parts holds a second stage of k and v, so that the state role runs ahead
// of the outputs.
template <int PARTS>
struct Smem {
    static constexpr int STAGES = PARTS == 1 ? 2 : 1;
    alignas(1024) unsigned char k[STAGES][2][TILE];   // [64 of N][token][64]
    alignas(1024) unsigned char q[2][TILE];
    alignas(1024) unsigned char x[STAGES][TILE];      // v: [token][64 columns]
    alignas(1024) unsigned char s[PARTS][TILE];       // parts of the state: [row of N][64 columns]
    alignas(1024) unsigned char p[PARTS][2][TILE];    // parts of P: [64 of j][i][64]; outputs pass through the first on their way out
    alignas(1024) unsigned char w[3][TILE];           // parts of w v: [token][64 columns]
    Scalars sc;
    float weight[C];                                  // dt_j e^{l_Q - l_j}
    float tot[2][4];                                  // sums of log2 decays over 32 tokens, of chunks in turn
    alignas(8) uint64_t bar[B_COUNT];
    uint32_t tmem;
    volatile int abort_flag;
};
static_assert(sizeof(Smem<1>) <= 232448 && sizeof(Smem<2>) <= 232448, "shared memory of one block");

struct Params {
    SsmParams a;
    Parts parts;
};

// w v of 64 tokens in three parts, by 256 threads: a thread to a quarter of a token's columns.
__device__ __forceinline__ void weigh(const unsigned char *x, unsigned char (*w)[TILE], int tokens, const float *weight)
{
    const int row = tokens + (threadIdx.x & 63), c = (threadIdx.x >> 6) * 2;
    const float2 w2 = f2(weight[row]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t at = sw128(row, c + i);
        const uint4 raw = *reinterpret_cast<const uint4 *>(x + at);
        float2 v[4] = {mul2(unpack2(raw.x), w2), mul2(unpack2(raw.y), w2), mul2(unpack2(raw.z), w2), mul2(unpack2(raw.w), w2)};
        *reinterpret_cast<uint4 *>(w[0] + at) = make_uint4(part(v[0]), part(v[1]), part(v[2]), part(v[3]));
        *reinterpret_cast<uint4 *>(w[1] + at) = make_uint4(part(v[0]), part(v[1]), part(v[2]), part(v[3]));
        *reinterpret_cast<uint4 *>(w[2] + at) = make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3]));
    }
}
struct Work {
    int h, sl, tok0, len, chunks;
    const float *init;   // this head's columns of the state to start from, or null
    float *fin;          // where its last state goes, or null
};

// ---- decay role ------------------------------------------------------------------------------------------------------------------
// A thread to a token; a chunk ahead, but for the writing.
template <int PARTS>
__device__ void decay_role(Smem<PARTS> &sm, const Params &p, const Work &wk)
{
    const int t = threadIdx.x & 127, lane = t & 31, warp = t >> 5;
    const float a = p.a.a[wk.h];
    const float *dtp = p.a.dt + (size_t)wk.tok0 * p.a.H + wk.h;
    float dt = t < wk.len ? dtp[(size_t)t * p.a.H] : 0.f;
#pragma unroll 1
    for (int c = 0; c < wk.chunks; ++c) {
        const int next = (c + 1) * C + t;
        const float next_dt = next < wk.len ? dtp[(size_t)next * p.a.H] : 0.f;
        const BlockScan<true> b(dt, a);
        float *tot = sm.tot[c & 1];   // (of chunk c - 2: read before that chunk's P was written)
        if (lane == 0) {
            tot[warp] = b.tot;
            mbar_arrive(&sm.bar[B_TOT]);
        }
        const float cf = dt * exp2f(b.rest), whole = rintf(b.a2), f = (b.a2 - whole) + b.lo, dtf = dt * exp2f(-f);
        if (!bar_wait(&sm.bar[B_TOT], c, &sm.abort_flag)) break;
        const float t1 = tot[1], t2 = tot[2], t3 = tot[3];
        const float w = cf * exp2f(warp == 0 ? t1 + t2 + t3 : warp == 1 ? t2 + t3 : warp == 2 ? t3 : 0.f);
        if (c > 0 && !bar_wait(&sm.bar[B_WX1], c - 1, &sm.abort_flag)) break;   // the last chunk's weights have been used
        sm.weight[t] = w;
        warp_arrive(&sm.bar[B_W]);
        if (c > 0 && !bar_wait(&sm.bar[B_P], c - 1, &sm.abort_flag)) break;     // and its scalars
        sm.sc.nn[t] = -whole;
        sm.sc.f[t] = f;
        sm.sc.cf[t] = cf;
        sm.sc.dtf[t] = dtf;
        warp_arrive(&sm.bar[B_SCAL]);
        dt = next_dt;
    }
}

// ---- state role ------------------------------------------------------------------------------------------------------------------
template <int N, int PARTS>
__device__ void state_role(Smem<PARTS> &sm, const Params &p, const Work &wk)
{
    // thread t and t + 128: row t of the state, each half the columns
    constexpr int STAGES = Smem<PARTS>::STAGES;
    const int t = threadIdx.x & 127, half = threadIdx.x >> 7, warp = t >> 5;
    const bool row = N == 128 || t < N;
    const uint32_t tm = sm.tmem + TM_DS + half * HS + ((uint32_t)(warp * 32) << 16);
    float2 S[HS / 2];
    read_row(S, wk.init && row ? wk.init + (size_t)t * p.a.P + half * HS : nullptr);
    auto write_parts = [&]() {
        if (row)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t at = sw128(t, 4 * half + c);
                if constexpr (PARTS == 1) {
                    *reinterpret_cast<uint4 *>(sm.s[0] + at) = make_uint4(pack2(S[4 * c]), pack2(S[4 * c + 1]), pack2(S[4 * c + 2]), pack2(S[4 * c + 3]));
                } else {
                    float2 x[4] = {S[4 * c], S[4 * c + 1], S[4 * c + 2], S[4 * c + 3]};
                    *reinterpret_cast<uint4 *>(sm.s[0] + at) = make_uint4(part(x[0]), part(x[1]), part(x[2]), part(x[3]));
                    *reinterpret_cast<uint4 *>(sm.s[PARTS - 1] + at) = make_uint4(pack2(x[0]), pack2(x[1]), pack2(x[2]), pack2(x[3]));
                }
            }
        fence_async_smem();
        tc_fence_before();
        warp_arrive(&sm.bar[B_S]);
    };
    write_parts();
    float gamma = 0.f;
    // The state behind chunk c
    auto joined = [&](int c) {
        if (!bar_wait(&sm.bar[B_DS1 + c % STAGES], c / STAGES, &sm.abort_flag)) return false;
        tc_fence_after();
        join(S, tm, gamma);
        tc_fence_before();
        warp_arrive(&sm.bar[B_JOIN]);
        return true;
    };
    bool ok = true;
#pragma unroll 1
    for (int c = 0; c < wk.chunks; ++c) {
        const int m = min(C, wk.len - c * C), st = c % STAGES;
        ok = bar_wait(&sm.bar[B_W], c, &sm.abort_flag) && bar_wait(&sm.bar[B_X + st], c / STAGES, &sm.abort_flag);
        if (ok && m < C) {   // rows behind the sequence's end: another sequence's, perhaps not finite; nothing of them may meet a zero weight
            ok = bar_wait(&sm.bar[B_K + st], c / STAGES, &sm.abort_flag);
            if (t >= m) {
                zero_half_row(sm.x[st], t, half);
#pragma unroll
                for (int b2 = 0; b2 < N / 64; ++b2) zero_half_row(sm.k[st][b2], t, half);
            }
            fence_async_smem();
            warp_arrive(&sm.bar[B_CLEAN]);
            ok = ok && bar_wait(&sm.bar[B_CLEAN], 0, &sm.abort_flag);
        }
        if (ok && c > 0) ok = bar_wait(&sm.bar[B_DS0 + (c - 1) % STAGES], (c - 1) / STAGES, &sm.abort_flag);
        if (!ok) break;
        weigh(sm.x[st], sm.w, 0, sm.weight);
        fence_async_smem();
        warp_arrive(&sm.bar[B_WX0]);
        const float *tot = sm.tot[c & 1];
        const float next_gamma = exp2f(tot[0] + tot[1] + tot[2] + tot[3]);
        if (c > 0) {
            ok = joined(c - 1) && bar_wait(&sm.bar[B_Y1 + (c - 1) % STAGES], (c - 1) / STAGES, &sm.abort_flag);   // (the parts before the last chunk have been read)
            if (!ok) break;
            write_parts();
        }
        gamma = next_gamma;
        weigh(sm.x[st], sm.w, 64, sm.weight);
        fence_async_smem();
        warp_arrive(&sm.bar[B_WX1]);
    }
    ok = ok && joined(wk.chunks - 1);
    if (wk.fin && row && ok) write_row(S, wk.fin + (size_t)t * p.a.P + half * HS);
}

// ---- output role -----------------------------------------------------------------------------------------------------------------
template <typename OUT, int PARTS>
__device__ void output_role(Smem<PARTS> &sm, const Params &p, const Work &wk)
{
    // thread t and t + 128: token t; of P the columns (tokens j) 64 half .., of the outputs the channels 32 half ..
    constexpr int STAGES = Smem<PARTS>::STAGES;
    const int t = threadIdx.x & 127, half = (threadIdx.x - STATE_T) >> 7, lane = t & 31, warp = t >> 5;
    const uint32_t tm = sm.tmem + ((uint32_t)(warp * 32) << 16);
    const float2 skip = f2(p.a.skip ? p.a.skip[wk.h] : 0.f);
    const size_t stride = (size_t)p.a.H * p.a.P;
    OUT *out = static_cast<OUT *>(p.a.out) + (size_t)wk.tok0 * stride + (size_t)wk.h * p.a.P + wk.sl * NS + half * 32;
    // P of chunk c; e: decay from the chunk's start to this row
    auto scores = [&](int c, float &e, uint4 (&x)[4]) {
        const int st = c % STAGES;
        if (!bar_wait(&sm.bar[B_SCAL], c, &sm.abort_flag)) return false;
        const float whole = -sm.sc.nn[t], frac = sm.sc.f[t], r = exp2f(whole + frac);
        const float *tot = sm.tot[c & 1];
        const float t0 = tot[0], t1 = tot[1], t2 = tot[2];
        // decay from the chunk's start to this row, and from block J's end to it
        const float before = warp == 0 ? 0.f : warp == 1 ? t0 : warp == 2 ? t0 + t1 : t0 + t1 + t2;
        e = r * exp2f(before);
        const float f0 = half ? r : r * exp2f(warp == 2 ? t1 : warp == 3 ? t1 + t2 : 0.f);   // block 2 half
        const float f1 = half ? r : r * exp2f(warp == 3 ? t2 : 0.f);                          // block 2 half + 1
        if (!bar_wait(&sm.bar[B_CB], c, &sm.abort_flag)) return false;
        tc_fence_after();
#pragma unroll 1
        for (int jj = 0; jj < 2; ++jj) {
            const int J = 2 * half + jj;   // block of 32 columns
            const float2 f = f2(jj ? f1 : f0), ni = f2(whole), fi = f2(frac);
            const float *cfs = &sm.sc.cf[J * 32], *ns = &sm.sc.nn[J * 32], *ds = &sm.sc.dtf[J * 32];
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
                float2 y[8];
                if (J > warp) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) y[u] = f2(0.f);
                } else {
                    float v[16];
                    tmem_ld16(tm + TM_CB + J * 32 + i, v);
                    if (J < warp) {
#pragma unroll
                        for (int u = 0; u < 8; u += 2) {
                            const float4 cf = load4(cfs + i + 2 * u);
                            y[u] = mul2(f2(v[2 * u], v[2 * u + 1]), mul2(f, f2(cf.x, cf.y)));
                            y[u + 1] = mul2(f2(v[2 * u + 2], v[2 * u + 3]), mul2(f, f2(cf.z, cf.w)));
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < 8; u += 2) {
                            const float4 nj = load4(ns + i + 2 * u), dj = load4(ds + i + 2 * u);
                            const float2 l0 = add2(add2(ni, f2(nj.x, nj.y)), fi), l1 = add2(add2(ni, f2(nj.z, nj.w)), fi);
                            y[u] = mul2(mul2(f2(v[2 * u], v[2 * u + 1]), f2(dj.x, dj.y)), f2(ex2_approx(l0.x), ex2_approx(l0.y)));
                            y[u + 1] = mul2(mul2(f2(v[2 * u + 2], v[2 * u + 3]), f2(dj.z, dj.w)), f2(ex2_approx(l1.x), ex2_approx(l1.y)));
                        }
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            if (i + 2 * u > lane) y[u].x = 0.f;
                            if (i + 2 * u + 1 > lane) y[u].y = 0.f;
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t at = sw128(t, jj * 4 + (i >> 3) + u);
                    if constexpr (PARTS == 1) {
                        *reinterpret_cast<uint4 *>(sm.p[0][half] + at) = make_uint4(pack2(y[4 * u]), pack2(y[4 * u + 1]), pack2(y[4 * u + 2]), pack2(y[4 * u + 3]));
                    } else {
                        *reinterpret_cast<uint4 *>(sm.p[0][half] + at) = make_uint4(part(y[4 * u]), part(y[4 * u + 1]), part(y[4 * u + 2]), part(y[4 * u + 3]));
                        *reinterpret_cast<uint4 *>(sm.p[PARTS - 1][half] + at) = make_uint4(pack2(y[4 * u]), pack2(y[4 * u + 1]), pack2(y[4 * u + 2]), pack2(y[4 * u + 3]));
                    }
                }
            }
        }
        if (!bar_wait(&sm.bar[B_X + st], c / STAGES, &sm.abort_flag)) return false;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *piece(sm.x[st], t, 4 * half + i);
        fence_async_smem();
        tc_fence_before();
        warp_arrive(&sm.bar[B_P]);
        return true;
    };
    // o of chunk c
    auto outputs = [&](int c, float e, const uint4 (&x)[4]) {
        const int m = min(C, wk.len - c * C), st = c % STAGES;
        if (!bar_wait(&sm.bar[B_Y2 + st], c / STAGES, &sm.abort_flag)) return false;   // (and q S, issued before)
        tc_fence_after();
        unsigned char *stage = sm.p[0][half];   // (read by the product that has just completed, and written by this warp alone)
        constexpr int PC = std::is_same<OUT, float>::value ? 8 : 4;   // 16-byte pieces of a row
        const int swap = PC == 4 ? 4 * (lane & 1) : 0;   // (odd rows in the other half of their line: two rows are read at a time)
        const float2 e2 = f2(e);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float y1[16], y2[16];
            tmem_ld16(tm + TM_Y1 + half * 32 + g * 16, y1);
            if constexpr (PARTS == 2) {
                tmem_ld16(tm + TM_Y1 + 64 + half * 32 + g * 16, y2);
#pragma unroll
                for (int i = 0; i < 16; ++i) y1[i] += y2[i];
            }
            tmem_ld16(tm + TM_Y2<PARTS> + half * 32 + g * 16, y2);
            if (g == 1) {
                tc_fence_before();
                warp_arrive(&sm.bar[B_YFREE]);
            }
            float2 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint4 xw = x[2 * g + (i >> 2)];
                const uint32_t word = (i & 3) == 0 ? xw.x : (i & 3) == 1 ? xw.y : (i & 3) == 2 ? xw.z : xw.w;
                y[i] = fma2(skip, unpack2(word), fma2(e2, f2(y1[2 * i], y1[2 * i + 1]), f2(y2[2 * i], y2[2 * i + 1])));
            }
            if constexpr (PC == 8) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *piece(stage, t, 4 * g + i) = make_uint4(__float_as_uint(y[2 * i].x), __float_as_uint(y[2 * i].y), __float_as_uint(y[2 * i + 1].x), __float_as_uint(y[2 * i + 1].y));
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *piece(stage, t, swap ^ (2 * g + i)) = make_uint4(pack2(y[4 * i]), pack2(y[4 * i + 1]), pack2(y[4 * i + 2]), pack2(y[4 * i + 3]));
            }
        }
        // through shared memory, so that a store is 16 bytes of one token and a warp's stores are whole sectors
        __syncwarp();
        const int rr = warp * 32 + lane / PC, from = PC == 4 ? (lane & 3) ^ (lane & 4) : lane % PC;
        OUT *to = out + (size_t)(c * C + rr) * stride + lane % PC * (16 / sizeof(OUT));
        if (m == C) {
#pragma unroll
            for (int i = 0; i < 32; i += 32 / PC) *reinterpret_cast<uint4 *>(to + i * stride) = *piece(stage, rr + i, from);
        } else {
#pragma unroll 1
            for (int i = 0; i < 32; i += 32 / PC)
                if (rr + i < m) *reinterpret_cast<uint4 *>(to + i * stride) = *piece(stage, rr + i, from);
        }
        __syncwarp();
        return true;
    };
    float e;
    uint4 x[4];
#pragma unroll 1
    for (int c = 0; c < wk.chunks; ++c)
        if (!scores(c, e, x) || !outputs(c, e, x)) break;
}

// ---- issue and load roles -------------------------------------------------------------------------------------------------------------
// One warp issues all products.  (Three, each for its own products and standing at one barrier at a time: 201 -> 211 us on 8 x 4096 tokens of 32 heads;
// one that looks for whatever product of whatever chunk is ready: 218.)
template <int N, int PARTS>
__device__ void issue_role(Smem<PARTS> &sm, const Work &wk, int test_timeout)
{
    constexpr int NB = N / 64, STAGES = Smem<PARTS>::STAGES;
    constexpr uint32_t T16 = TILE / 16;
    const uint32_t tm = sm.tmem;
    auto desc = [](const void *x, uint32_t lbo) { return desc_lo(smem_desc_sw128(smem_u32(x), lbo, 1024)); };
    auto wait = [&](int b, int parity) { return bar_wait(&sm.bar[b], parity, &sm.abort_flag); };
    auto ready = [&](int b, int parity) { return __all_sync(0xffffffffu, mbar_test_wait(&sm.bar[b], parity & 1)); };
    const uint32_t q_km = desc(sm.q, 0), p_km = desc(sm.p, 0), s_mn = desc(sm.s, TILE), w_mn = desc(sm.w, TILE);
#pragma unroll 1
    for (int c = 0; c < wk.chunks; ++c) {
        const int st = c % STAGES;
        const uint32_t k_km = desc(sm.k[st], 0), x_mn = desc(sm.x[st], 0);
        // k^T as left operand: 128 rows of N, for N = 64 the one block of them twice (the second half of the accumulator is not read)
        const uint32_t k_mn = desc(sm.k[st], NB == 2 ? TILE : 0);
        if (!wait(B_K + st, c / STAGES) || !wait(B_Q, c)) return;
        if (wk.len - c * C < C && !wait(B_CLEAN, 0)) return;
        tc_fence_after();
#pragma unroll
        for (int b = 0; b < NB; ++b) mma4_bf16_lo<2, 2>(tm + TM_CB, q_km + b * T16, k_km + b * T16, idesc_bf16(128, 128, 0, 0), b > 0);
        mma_commit(&sm.bar[B_CB]);
        // P v, q S (before it), and 64 tokens at a time what the chunk adds to the state: each as soon as its operand is written
        int ds = 0;
        bool y1 = false, y2 = false;
        const uint32_t since = clock_lo();
        while (ds < 2 || !y2) {
            if (y1 && !y2 && ready(B_P, c) && ready(B_X + st, c / STAGES)) {
                tc_fence_after();
#pragma unroll
                for (int b = 0; b < 2 * PARTS; ++b) mma4_bf16_lo<2, 128>(tm + TM_Y2<PARTS>, p_km + b * T16, x_mn + (b & 1) * 512, idesc_bf16(128, 64, 0, 1), b > 0);
                if (test_timeout) return;   // test hook: the output role's wait for this product runs out
                mma_commit(&sm.bar[B_Y2 + st]);
                y2 = true;
            }
            if (!y1 && ready(B_S, c) && (c == 0 || ready(B_YFREE, c - 1))) {
                tc_fence_after();
#pragma unroll
                for (int b = 0; b < NB; ++b) mma4_bf16_lo<2, 128>(tm + TM_Y1, q_km + b * T16, s_mn + b * 512, idesc_bf16(128, 64 * PARTS, 0, 1), b > 0);
                mma_commit(&sm.bar[B_Y1 + st]);
                y1 = true;
            }
            if (ds < 2 && ready(B_WX0 + ds, c) && (ds == 1 || c == 0 || ready(B_JOIN, c - 1))) {
                tc_fence_after();
                mma4_bf16_lo<128, 128>(tm + TM_DS, k_mn + ds * 512, w_mn + ds * 512, idesc_bf16(128, 192, 1, 1), ds);
                mma_commit(&sm.bar[(ds ? B_DS1 : B_DS0) + st]);
                ++ds;
            }
            if (__any_sync(0xffffffffu, sm.abort_flag || clock_lo() - since >= WAIT_LIMIT)) {
                sm.abort_flag = 1;
                return;
            }
        }
    }
}
template <int N, int PARTS>
__device__ void load_role(Smem<PARTS> &sm, const CUtensorMap *tq, const CUtensorMap *tk, const CUtensorMap *tv, const Params &p, const Work &wk)
{
    constexpr int NB = N / 64, STAGES = Smem<PARTS>::STAGES;
    const bool first = (threadIdx.x & 31) == 0;
    const int xk = wk.h / (p.a.H / p.a.G) * N, xv = wk.h * p.a.P + wk.sl * NS;
    auto load = [&](unsigned char *to, const CUtensorMap *map, int x, int blocks, int c, int bar) {
        if (first) {
            mbar_expect_tx(&sm.bar[bar], blocks * TILE);
            for (int b = 0; b < blocks; ++b) tma_load_2d(to + b * TILE, map, x + b * 64, wk.tok0 + c * C, &sm.bar[bar]);
        }
        __syncwarp();
    };
    auto load_kx = [&](int c) {   // chunk c's stage: its last chunk's products must be done
        const int st = c % STAGES;
        if (c >= STAGES && !bar_wait(&sm.bar[B_DS1 + st], c / STAGES - 1, &sm.abort_flag)) return false;
        load(sm.k[st][0], tk, xk, NB, c, B_K + st);
        if (c >= STAGES && !bar_wait(&sm.bar[B_Y2 + st], c / STAGES - 1, &sm.abort_flag)) return false;
        load(sm.x[st], tv, xv, 1, c, B_X + st);
        return true;
    };
    if (STAGES == 2) load_kx(0);
#pragma unroll 1
    for (int c = 0; c < wk.chunks; ++c) {
        if (first && c + STAGES < wk.chunks) {   // tiles of a later chunk on their way to L2 meanwhile
            const int y = wk.tok0 + (c + STAGES) * C;
            for (int b = 0; b < NB; ++b) {
                prefetch_2d(tk, xk + b * 64, y);
                prefetch_2d(tq, xk + b * 64, y);
            }
            prefetch_2d(tv, xv, y);
        }
        for (int i = (c + 2) * C + (threadIdx.x & 31); i < (c + 3) * C && i < wk.len; i += 32) prefetch_line(p.a.dt + (size_t)(wk.tok0 + i) * p.a.H + wk.h);
        if (c > 0 && !bar_wait(&sm.bar[B_Y1 + (c - 1) % STAGES], (c - 1) / STAGES, &sm.abort_flag)) return;   // (and q k^T, issued before)
        load(sm.q[0], tq, xk, NB, c, B_Q);
        const int ahead = c + STAGES - 1;
        if (ahead < wk.chunks && !load_kx(ahead)) return;
    }
}

template <int N, typename OUT>
__global__ void __launch_bounds__(NT, 1)
ssm_chunk_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                     const __grid_constant__ Params p)
{
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    constexpr int PARTS = std::is_same<OUT, float>::value ? 2 : 1;
    Smem<PARTS> &sm = *reinterpret_cast<Smem<PARTS> *>(smem_dyn);
    if (smem_u32(smem_dyn) & 1023) {
        if (threadIdx.x == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_ALIGN);
        return;
    }
    const int tid = threadIdx.x, slices = p.a.P / NS;
    Work wk;
    wk.sl = blockIdx.x % slices;
    wk.h = blockIdx.x / slices % p.a.H;
    const int index = blockIdx.x / slices / p.a.H;
    const Piece pc(p.a.cu_seqlens, p.a.T, p.parts, index);
    const size_t head = ((size_t)wk.h * N) * p.a.P + wk.sl * NS, state = (size_t)p.a.H * N * p.a.P;
    wk.tok0 = pc.tok0;
    wk.len = pc.len;
    wk.chunks = (pc.len + C - 1) / C;
    wk.init = p.parts.n > 1 ? p.parts.state + index * state + head : p.a.init_state ? p.a.init_state + pc.n * state + head : nullptr;
    wk.fin = p.a.final_state && pc.last ? p.a.final_state + pc.n * state + head : nullptr;
    if (pc.len <= 0) {   // an empty sequence hands its state on (its first part does)
        const size_t at = (size_t)(tid >> 1) * p.a.P + (tid & 1) * HS;
        if (wk.fin && tid < 2 * N) {
            float2 S[HS / 2];
            read_row(S, p.a.init_state ? p.a.init_state + pc.n * state + head + at : nullptr);
            write_row(S, wk.fin + at);
        }
        return;
    }
    if (tid == 0) {
        for (int b = 0; b < B_COUNT; ++b) mbar_init(&sm.bar[b], b == B_TOT || b == B_W || b == B_SCAL ? 4 : b >= B_CLEAN && b < B_CB ? 8 : 1);
        sm.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tq);
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
    }
    if (tid >= T_ISSUE && tid < T_ISSUE + 32) tmem_alloc(&sm.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // 768 threads x 80 registers at launch = 128 x 480 >= 128 x (2 x 88 + 2 x 104 + 56 + 40)
    if (tid < STATE_T) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
        state_role<N, PARTS>(sm, p, wk);
    } else if (tid < T_DECAY) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        output_role<OUT, PARTS>(sm, p, wk);
    } else if (tid < T_ISSUE) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        decay_role<PARTS>(sm, p, wk);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (tid < T_ISSUE + 32) issue_role<N, PARTS>(sm, wk, p.a.test_timeout);
        else if (tid < T_ISSUE + 64) load_role<N, PARTS>(sm, &tq, &tk, &tv, p, wk);
    }
    tc_fence_before();
    __syncthreads();
    if (sm.abort_flag) {   // copies and products issued just before a wait gave up finish first
        for (int i = 0; i < 32; ++i) __nanosleep(1000);
        if (tid == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_TIMEOUT);
    }
    if (tid >= T_ISSUE && tid < T_ISSUE + 32) {
        tc_fence_after();
        tmem_dealloc(sm.tmem, 512);
    }
}

// ---- host side --------------------------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(ptr);
    });
    return fn;
}

template <int N, typename OUT>
cudaError_t launch_t(const Params &p, cudaStream_t stream)
{
    CUtensorMap tq, tk, tv;
    const uint64_t rows = (uint64_t)p.a.rows, kw = (uint64_t)p.a.G * N, vw = (uint64_t)p.a.H * p.a.P;
    if (!make_map(&tq, p.a.q, rows, kw, p.a.q_stride) || !make_map(&tk, p.a.k, rows, kw, p.a.k_stride) || !make_map(&tv, p.a.v, rows, vw, p.a.v_stride))
        return cudaErrorInvalidValue;
    auto kern = ssm_chunk_kernel<N, OUT>;
    constexpr int smem = (int)sizeof(Smem<std::is_same<OUT, float>::value ? 2 : 1>);
    const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (err != cudaSuccess) return err;
    kern<<<(unsigned)(p.a.n_seq * p.parts.n) * p.a.H * (p.a.P / NS), NT, smem, stream>>>(tq, tk, tv, p);
    count_launch(1);
    return cudaGetLastError();
}

}  // namespace

bool make_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint64_t stride)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {stride * 2};
    cuuint32_t box[2] = {64, C};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace ssm

bool ssm_chunk_supported(int io_dtype, int N, int P, int rows) { return io_dtype == KLA_BF16 && (N == 64 || N == 128) && P % ssm::NS == 0 && rows > 0; }

size_t ssm_chunk_workspace_bytes(const SsmParams &a) { return ssm::Parts(a, sm_count(), nullptr).bytes(a); }

cudaError_t launch_ssm_chunk(const SsmParams &a, int out_dtype, cudaStream_t stream)
{
    ssm::Params p = {a, ssm::Parts(a, sm_count(), a.workspace)};
    if (p.parts.n > 1) {
        const cudaError_t err = ssm::launch_part_starts(a, p.parts, false, stream);
        if (err != cudaSuccess) return err;
    }
    if (a.N == 64) return out_dtype == KLA_F32 ? ssm::launch_t<64, float>(p, stream) : ssm::launch_t<64, __nv_bfloat16>(p, stream);
    return out_dtype == KLA_F32 ? ssm::launch_t<128, float>(p, stream) : ssm::launch_t<128, __nv_bfloat16>(p, stream);
}

}  // namespace kla
