// Reverse mode of the selective state space scan on the tensor cores (bf16; formulas at the top of ssm_scan.cu): chunks of 128 tokens.
//
// Two passes over the states (ssm_state.cu) leave, in fp32, the state S before every chunk and the gradient G of the state behind it; they are
// independent of each other.  Then every (chunk, group of heads that share q and k) is by itself: a block takes one, and its heads one after another, each
// in slices of 64 columns of v.  Per slice, with rows j and columns i of 128 x 128 products, do the gradient of o, parts as in ssm_chunk.cu:
//
//     DX^T = v do^T                           L_ij = exp(l_i - l_j);  (k q^T once per block)
//     M_ji = L_ij dt_j (q_i . k_j)            dv  = M do + w_j (k G) + d do
//     sum over heads of L_ij dt_j (do_i . v_j) in registers: one product each with q and k at the end gives their parts of dk and dq
//     dq += (e^{l_i} do) S^T,  dk += (w_j v) G^T     w_j = dt_j e^{l_Q - l_j}; accumulated over the heads in tensor memory
//     x_i = e^{l_i} (q S)_i . do_i,  z_j = w_j (k G)_j . v_j
//
// Precision.  dq, dk, dv are bf16: of their derived operands M, the sum over heads, the scaled do and v are one bf16 each, and S and G two, so that
// every term carries one rounding like the result's own (with one part of S and G the 2-norm error of dq is 2.7e-3, the rounding alone 1.7e-3).
// The gradients of dt and a are fp32: their terms come from exact products (DX, k q^T) and from S and G in three bf16 parts (24 bits), summed in fp32.
//
// F_t is a sum of the terms that span token t and of no others (row sums less column sums come to the same, but a large step's terms would have to cancel in
// every token before it).  With t in block B of 32 tokens: rows i >= t against columns j of the blocks before B, columns j < t of B against rows of
// the blocks behind it, and in the diagonal tile sums over i >= t of every j < t, which are sums over columns of sums along rows.
//
// 256 threads work, a thread to half a row; one warp issues the products and loads the tiles.  The chain of one slice is what takes the time, not the
// products (about a third of it) nor memory.  8 x 4096 tokens of 32 heads, N = 128: 755 us, of which the state passes 215; 16 packed sequences of 16
// heads, N = 64: 467 us.  512 workers with a quarter of a row spill (975-995 us for 796 then), a warpgroup of its own for the scalars waits for the
// workers as they for it (831), k G beside the 128 x 128 work where N = 64 leaves tensor memory for it takes the same time.
#include "ssm_pieces.cuh"

namespace kla {
namespace ssm {

namespace {

constexpr int NT = 256 + 128;   // (of the last warpgroup one warp works)

enum Bar {
    B_QK = 0,       // q and k landed
    B_TILES,        // v and do landed
    B_CB, B_QS, B_DQ, B_DX, B_C2, B_DK, B_FIN,   // products complete: k q^T; q S; its share of dq; DX^T; M do and k G; dk's share; the last ones
    B_TOT,          // sums over 32 tokens written (a warp)
    B_CLEAN0, B_CLEAN,   // rows behind the sequence's end zeroed: of q and k, of v and do (all workers, like those below; an arrival per warp instead,
                         // as in the forward, 495 us for 486 on 16 packed sequences)
    B_S, B_SCALED, B_X, B_G, B_M,   // written: parts of S; scaled tiles; x read; parts of G; M
    B_E,            // a head's sums written
    B_FREE,         // a slice's tiles and accumulators read
    B_MS,           // the sum over heads written
    B_COUNT
};

// Tensor memory: k q^T, dq, dk (128 columns each); q S (64), then DX^T (128), then M do (64) and k G (64).
constexpr uint32_t TM_CB = 0, TM_DQ = 128, TM_DK = 256, TM_DX = 384, TM_DV = 384, TM_SG = 448;

struct Smem {
    alignas(1024) unsigned char k[2][TILE], q[2][TILE];   // [64 of N][token][64]
    alignas(1024) unsigned char v[TILE], go[TILE];        // [token][64 columns]
    alignas(1024) unsigned char sp[3][TILE];              // parts of S, then of G: [row of N][64 columns]
    alignas(1024) unsigned char m[2][TILE];               // M^T, at the end the sum over heads: [64 of i][j][64]
    alignas(1024) unsigned char gs[TILE], vs[TILE];       // e^{l_i} do, w_j v
    float a2[2][C], lo[2][C], r[2][C], dt[2][C];  // of heads in turn
    // of heads in turn:
    float rows[2][4][C];      // sums of R_ij over the 32 tokens j of a block before that of i; in i's own block of R_i'j, i' >= i > j
    float acc[2][2][5][C];    // of a token, by half of the columns: x, z, what ddt has directly, do . v, its R_ij with tokens i of later blocks
    float tot[2][4];
    float sg[2][8];
    alignas(8) uint64_t bar[B_COUNT];
    uint32_t tmem;
    volatile int abort_flag;
};
static_assert(sizeof(Smem) <= 232448, "shared memory of one block");

struct Params {
    SsmParams a;
    const float *states, *dstates;    // [slot][H][P / 64][STATE_ELEMS]
    float *part_a, *part_d;           // [slot][4][H]
    float *part_q, *part_k;           // [splits][rows][G][N], or null: dq, dk are written
    int splits;                       // blocks that share the heads of a group
};

// Lanes l and l + 16 get the sum over the warp of w x[l], w the lane's entry of `weights`, through 2 KB of the warp's own: a column of 32 rows to 128 bytes, its
// 16-byte pieces permuted so that neither the writing of a row nor the reading of a column meets a bank twice.  (By shuffles, 31 with two selections each
// for 32 columns: 788 us for 735 on 8 x 4096 tokens.)
__device__ __forceinline__ float column_sums(const float (&x)[16], float *own, const float *weights)
{
    const int lane = threadIdx.x & 31, col = lane & 15;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 16; ++c) own[c * 32 + (lane ^ (4 * (c & 7)))] = x[c];
    __syncwarp();
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float4 y = load4(own + col * 32 + 4 * (((lane >> 4) * 4 + r) ^ (col & 7))), w = load4(weights + (lane >> 4) * 16 + 4 * r);
        s += fmaf(y.x, w.x, y.y * w.y) + fmaf(y.z, w.z, y.w * w.w);
    }
    return s + __shfl_xor_sync(0xffffffffu, s, 16);
}

__device__ __forceinline__ float dot_bf16(float2 a, uint32_t b, float s)
{
    const float2 y = unpack2(b);
    return fmaf(a.x, y.x, fmaf(a.y, y.y, s));
}

template <int N>
__device__ __forceinline__ void split_state(Smem &sm, const float2 (&S)[HS / 2])
{
    const int t = threadIdx.x & 127, half = threadIdx.x >> 7;
    if (N == 64 && t >= N) return;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t at = sw128(t, 4 * half + c);
        float2 x[4] = {S[4 * c], S[4 * c + 1], S[4 * c + 2], S[4 * c + 3]};
        *reinterpret_cast<uint4 *>(sm.sp[0] + at) = make_uint4(part(x[0]), part(x[1]), part(x[2]), part(x[3]));
        *reinterpret_cast<uint4 *>(sm.sp[1] + at) = make_uint4(part(x[0]), part(x[1]), part(x[2]), part(x[3]));
        *reinterpret_cast<uint4 *>(sm.sp[2] + at) = make_uint4(pack2(x[0]), pack2(x[1]), pack2(x[2]), pack2(x[3]));
    }
}
__device__ __forceinline__ void load_state(float2 (&S)[HS / 2], const float *from)
{
#pragma unroll
    for (int i = 0; i < HS / 4; ++i) {
        const float4 t = load4(from + i * 1024);
        S[2 * i] = f2(t.x, t.y);
        S[2 * i + 1] = f2(t.z, t.w);
    }
}

struct Work {
    int slot, tok0, m, g, h0, items;   // first head, slices of all its heads
};

// 16 columns of two accumulators
__device__ __forceinline__ void tmem_ld16x2(uint32_t ta, uint32_t tb, float (&a)[16], float (&b)[16])
{
    uint32_t x[16], y[16];
#define R16(r) "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), \
               "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : R16(x), R16(y) : "r"(ta), "r"(tb) : "memory");
#undef R16
#pragma unroll
    for (int i = 0; i < 16; ++i) a[i] = __uint_as_float(x[i]), b[i] = __uint_as_float(y[i]);
}

// A head's scalars of one token.
struct Head {
    float dt, a, a2, lo;
    float w, wn;      // dt_j e^{l_Q - l_j}, and without dt_j
    float e;          // e^{l_i}
    float f0, f1;     // decay from this token to the start of block 2 half, 2 half + 1 of the columns (where that lies behind this token's block)
    float whole;      // e^{l_Q}
};

template <int N>
__device__ void workers(Smem &sm, const Params &p, const Work &wk)
{
    const int t = threadIdx.x & 127, half = threadIdx.x >> 7, lane = t & 31, warp = t >> 5, slices = p.a.P / NS, m = wk.m;
    const uint32_t tm = sm.tmem + ((uint32_t)(warp * 32) << 16);
    const bool in = t < m, row = N == 128 || t < N;
    auto wait = [&](int b, int parity) { return bar_wait(&sm.bar[b], parity, &sm.abort_flag); };
    if (m < C) {   // rows behind the sequence's end are nobody's, or another sequence's
        if (!wait(B_QK, 0)) return;
        if (!in)
#pragma unroll
            for (int b = 0; b < N / 64; ++b) {
                zero_half_row(sm.k[b], t, half);
                zero_half_row(sm.q[b], t, half);
            }
        fence_async_smem();
        mbar_arrive(&sm.bar[B_CLEAN0]);
    }
    float2 ms[32];   // sum over heads of L_ij dt_j (do_i . v_j): row j = t, columns i = 64 half ..
#pragma unroll
    for (int i = 0; i < 32; ++i) ms[i] = f2(0.f);
    const size_t row_out = (size_t)(wk.tok0 + t);
    auto state_at = [&](const float *base, int item) {
        return base + (((size_t)wk.slot * p.a.H + wk.h0) * slices + item) * STATE_ELEMS + threadIdx.x * 4;
    };
    float2 S[HS / 2], G[HS / 2];
    load_state(S, state_at(p.states, 0));
    const int heads = wk.items / slices;
    float next_dt = in ? p.a.dt[row_out * p.a.H + wk.h0] : 0.f, next_a = p.a.a[wk.h0];
    auto decays = [&](int i, Head &hd) {   // of the i-th head
        hd.a = next_a;
        hd.dt = next_dt;
        const BlockScan<true> b(hd.dt, hd.a);
        float *tot = sm.tot[i & 1];
        if (lane == 0) {
            if (half == 0) tot[warp] = b.tot;
            mbar_arrive(&sm.bar[B_TOT]);
        }
        hd.a2 = b.a2;
        hd.lo = b.lo;
        const float r = exp2f(b.a2);
        if (half == 0) sm.a2[i & 1][t] = b.a2, sm.lo[i & 1][t] = b.lo;
        else sm.r[i & 1][t] = r, sm.dt[i & 1][t] = hd.dt;
        if (!wait(B_TOT, i)) return false;
        const float t0 = tot[0], t1 = tot[1], t2 = tot[2], t3 = tot[3];
        hd.e = r * exp2f(warp == 0 ? 0.f : warp == 1 ? t0 : warp == 2 ? t0 + t1 : t0 + t1 + t2);
        hd.wn = exp2f(b.rest + (warp == 0 ? t1 + t2 + t3 : warp == 1 ? t2 + t3 : warp == 2 ? t3 : 0.f));
        hd.w = hd.dt * hd.wn;
        hd.f0 = exp2f(b.rest + (half == 0 ? 0.f : warp == 0 ? t1 : 0.f));
        hd.f1 = exp2f(b.rest + (half == 0 ? 0.f : warp == 0 ? t1 + t2 : warp == 1 ? t2 : 0.f));
        hd.whole = exp2f(t0 + t1 + t2 + t3);
        return true;
    };
    // Gradients of dt and a of the i-th head, a thread of the first half to a token; of the other blocks' tokens it needs the sums.
    auto finish = [&](int i, float a, float dt, float whole) {
        if (!wait(B_E, i)) return false;
        if (half) return true;
        const int h = wk.h0 + i;
        const auto &acc = sm.acc[i & 1];
        float all = 0.f, later = 0.f, earlier = 0.f, own = 0.f, zt = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) all += sm.sg[i & 1][k];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int at = b * 32 + lane;
            float o = 0.f, y = 0.f;
            if (b >= warp) {
                o = acc[0][0][at] + acc[1][0][at];
#pragma unroll
                for (int J = 0; J < b; ++J)
                    if (J < warp) o += sm.rows[i & 1][J][at];
            }
            if (b <= warp) y = acc[0][1][at] + acc[1][1][at];
            if (b > warp) later += o;
            if (b == warp) own = o, zt = y + (acc[0][4][at] + acc[1][4][at]);
            if (b < warp) earlier += y;
        }
        float suffix = own, prefix = zt, d = acc[0][3][t] + acc[1][3][t];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float u = __shfl_down_sync(0xffffffffu, suffix, o), y = __shfl_up_sync(0xffffffffu, prefix, o);
            if (lane + o < 32) suffix += u;
            if (lane >= o) prefix += y;
            later += __shfl_xor_sync(0xffffffffu, later, o);
            earlier += __shfl_xor_sync(0xffffffffu, earlier, o);
        }
        const float before = __shfl_up_sync(0xffffffffu, prefix, 1);
        const float F = sm.rows[i & 1][warp][t] + suffix + later + (lane ? before : 0.f) + earlier + whole * all;
        if (in) p.a.ddt[row_out * p.a.H + h] = fmaf(a, F, acc[0][2][t] + acc[1][2][t]);
        float da = in ? dt * F : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            da += __shfl_xor_sync(0xffffffffu, da, o);
            d += __shfl_xor_sync(0xffffffffu, d, o);
        }
        if (lane == 0) {
            p.part_a[((size_t)wk.slot * 4 + warp) * p.a.H + h] = da;
            p.part_d[((size_t)wk.slot * 4 + warp) * p.a.H + h] = d;
        }
        return true;
    };
    Head hd, next;
    float near = 0.f, far = 0.f, z = 0.f, x = 0.f, dd = 0.f, sg = 0.f;   // sums over a head's slices (near, far: of R without dt, in the token's block and behind)
    float old_a = 0.f, old_dt = 0.f, old_whole = 0.f;    // of the head before
    bool ok = decays(0, hd) && wait(B_CB, 0);
#pragma unroll 1
    for (int it = 0; ok && it < wk.items; ++it) {
        const int i = it / slices, h = wk.h0 + i, sl = it % slices;
        if (sl == 0 && i + 1 < heads) {   // (needed while this head's last product runs)
            next_dt = in ? p.a.dt[row_out * p.a.H + h + 1] : 0.f;
            next_a = p.a.a[h + 1];
        }
        // -- parts of S
        if (it > 0 && !(ok = wait(B_DK, it - 1))) break;
        split_state<N>(sm, S);
        fence_async_smem();
        mbar_arrive(&sm.bar[B_S]);
        // -- scaled tiles, while q S is formed
        if (!(ok = wait(B_TILES, it))) break;
        if (m < C) {
            if (!in) {
                zero_half_row(sm.v, t, half);
                zero_half_row(sm.go, t, half);
            }
            fence_async_smem();
            mbar_arrive(&sm.bar[B_CLEAN]);
        }
#pragma unroll 2
        for (int c = 0; c < 4; ++c) {
            const uint32_t at = sw128(t, 4 * half + c);
            const uint4 gv = *reinterpret_cast<const uint4 *>(sm.go + at), vv = *reinterpret_cast<const uint4 *>(sm.v + at);
            const float2 e2 = f2(hd.e), w2 = f2(hd.w);
            *reinterpret_cast<uint4 *>(sm.gs + at) = make_uint4(pack2(mul2(unpack2(gv.x), e2)), pack2(mul2(unpack2(gv.y), e2)), pack2(mul2(unpack2(gv.z), e2)), pack2(mul2(unpack2(gv.w), e2)));
            *reinterpret_cast<uint4 *>(sm.vs + at) = make_uint4(pack2(mul2(unpack2(vv.x), w2)), pack2(mul2(unpack2(vv.y), w2)), pack2(mul2(unpack2(vv.z), w2)), pack2(mul2(unpack2(vv.w), w2)));
        }
        fence_async_smem();
        mbar_arrive(&sm.bar[B_SCALED]);
        load_state(G, state_at(p.dstates, it));
        // -- x
        if (!(ok = wait(B_QS, it))) break;
        tc_fence_after();
        {
            float u[16], y[16], s = 0.f;
            tmem_ld16x2(tm + TM_SG + half * 32, tm + TM_SG + half * 32 + 16, u, y);
            tc_fence_before();
            mbar_arrive(&sm.bar[B_X]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 gv = *piece(sm.go, t, 4 * half + c);
                const float *q = c < 2 ? u + 8 * c : y + 8 * (c - 2);
                s = dot_bf16(f2(q[0], q[1]), gv.x, dot_bf16(f2(q[2], q[3]), gv.y, dot_bf16(f2(q[4], q[5]), gv.z, dot_bf16(f2(q[6], q[7]), gv.w, s))));
            }
            x = fmaf(hd.e, s, x);
        }
        // -- parts of G
        if (row)
#pragma unroll
            for (int c = 0; c < HS / 2; ++c) sg = fmaf(S[c].x, G[c].x, fmaf(S[c].y, G[c].y, sg));
        if (!(ok = wait(B_DQ, it))) break;
        split_state<N>(sm, G);
        fence_async_smem();
        mbar_arrive(&sm.bar[B_G]);
        // -- M, the sum over heads, and the sums of R
        if (!(ok = wait(B_DX, it))) break;
        tc_fence_after();
        const float *rr_ = sm.r[i & 1], *aa = sm.a2[i & 1], *ll = sm.lo[i & 1];
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
            const int I = 2 * half + ii;   // block of 32 columns i
            float behind = 0.f;            // in the diagonal tile: the row's sum from a column on
#pragma unroll
            for (int u = 16; u >= 0; u -= 16) {
                float2 mm[8];
                float rs[16], row = 0.f;
                if (I < warp) {
#pragma unroll
                    for (int y = 0; y < 8; ++y) mm[y] = f2(0.f);
                } else {
                    float cb[16], dx[16];
                    tmem_ld16x2(tm + TM_CB + I * 32 + u, tm + TM_DX + I * 32 + u, cb, dx);
                    const float2 f = f2(ii ? hd.f1 : hd.f0), dt2 = f2(hd.dt);
                    float2 sum = f2(0.f);
#pragma unroll
                    for (int y = 0; y < 16; y += 4) {
                        float2 L[2];
                        if (I > warp) {
                            const float4 ri = load4(rr_ + I * 32 + u + y);
                            L[0] = mul2(f2(ri.x, ri.y), f);
                            L[1] = mul2(f2(ri.z, ri.w), f);
                        } else {
                            const float4 ai = load4(aa + I * 32 + u + y), li = load4(ll + I * 32 + u + y);
                            auto decay = [&](int i, float hi, float lo) { return u + y + i >= lane ? ex2_approx((hi - hd.a2) + (lo - hd.lo)) : 0.f; };
                            L[0] = f2(decay(0, ai.x, li.x), decay(1, ai.y, li.y));
                            L[1] = f2(decay(2, ai.z, li.z), decay(3, ai.w, li.w));
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int c = y + 2 * k;
                            const float2 d = f2(dx[c], dx[c + 1]), lc = mul2(L[k], f2(cb[c], cb[c + 1]));
                            mm[c / 2] = mul2(lc, dt2);
                            ms[ii * 16 + (u + c) / 2] = fma2(mul2(L[k], d), dt2, ms[ii * 16 + (u + c) / 2]);
                            const float2 rr = mul2(lc, d);
                            sum = add2(sum, rr);
                            rs[c] = rr.x;
                            rs[c + 1] = rr.y;
                        }
                    }
                    row = sum.x + sum.y;
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    *piece(sm.m[half], t, ii * 4 + (u >> 3) + y) = make_uint4(pack2(mm[4 * y]), pack2(mm[4 * y + 1]), pack2(mm[4 * y + 2]), pack2(mm[4 * y + 3]));
                if (ii == 1 && u == 0) {
                    fence_async_smem();
                    tc_fence_before();
                    mbar_arrive(&sm.bar[B_M]);
                }
                if (I >= warp) {   // (the scaled do has been read by its product)
                    if (I == warp) {
#pragma unroll
                        for (int y = 15; y >= 0; --y) {
                            behind += rs[y];
                            rs[y] = u + y > lane ? behind : 0.f;
                        }
                        if (u == 0) near += behind;   // (R_tt among it)
                    } else {
                        far += row;
                    }
                    const float s = column_sums(rs, reinterpret_cast<float *>(sm.gs) + (warp * 2 + half) * 512, &sm.dt[i & 1][warp * 32]);
                    if (lane < 16) {
                        float &to = sm.rows[i & 1][warp][I * 32 + u + lane];
                        to = sl ? to + s : s;
                    }
                }
            }
        }
        if (it + 1 < wk.items) load_state(S, state_at(p.states, it + 1));   // (from L2)
        // -- the next head's decays and the last one's gradients, while M do and k G are formed
        const bool last = sl == slices - 1;
        if (last && i + 1 < heads && !(ok = decays(i + 1, next))) break;
        if (last && i > 0 && !(ok = finish(i - 1, old_a, old_dt, old_whole))) break;
        // -- dv and z
        if (!(ok = wait(B_C2, it))) break;
        tc_fence_after();
        {
            const float2 skip = f2(p.a.skip ? p.a.skip[h] : 0.f), w2 = f2(hd.w);
            float s = 0.f;
#pragma unroll
            for (int u = 0; u < 32; u += 16) {
                float kg[16], dv[16];
                tmem_ld16x2(tm + TM_SG + half * 32 + u, tm + TM_DV + half * 32 + u, kg, dv);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint4 vv = *piece(sm.v, t, 4 * half + (u >> 3) + y), gv = *piece(sm.go, t, 4 * half + (u >> 3) + y);
                    const uint32_t vw[4] = {vv.x, vv.y, vv.z, vv.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w};
                    uint32_t o[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float2 kk = f2(kg[8 * y + 2 * q], kg[8 * y + 2 * q + 1]);
                        s = dot_bf16(kk, vw[q], s);
                        dd = dot_bf16(unpack2(gw[q]), vw[q], dd);
                        o[q] = pack2(fma2(skip, unpack2(gw[q]), fma2(w2, kk, f2(dv[8 * y + 2 * q], dv[8 * y + 2 * q + 1]))));
                    }
                    *piece(sm.m[half], t, ((u >> 3) + y) ^ (4 * (t & 1))) = make_uint4(o[0], o[1], o[2], o[3]);   // (read by the products that have completed; odd rows with their halves
                    // swapped, so that the eight lanes that read two rows meet no bank twice)
                }
            }
            z += s;   // (without w_j)
        }
        tc_fence_before();
        mbar_arrive(&sm.bar[B_FREE]);
        __syncwarp();
        {
            __nv_bfloat16 *dv = static_cast<__nv_bfloat16 *>(p.a.dv) + ((size_t)(wk.tok0 + warp * 32 + (lane >> 2)) * p.a.H + h) * p.a.P + sl * NS + half * 32 + (lane & 3) * 8;
            const int rr = warp * 32 + (lane >> 2);
#pragma unroll
            for (int c = 0; c < 32; c += 8)
                if (rr + c < m) *reinterpret_cast<uint4 *>(dv + (size_t)c * p.a.H * p.a.P) = *piece(sm.m[half], rr + c, (lane & 3) ^ (lane & 4));
        }
        __syncwarp();
        if (last) {
            sm.acc[i & 1][half][0][t] = x;
            sm.acc[i & 1][half][1][t] = hd.w * z;
            sm.acc[i & 1][half][2][t] = fmaf(hd.wn, z, near + far);
            sm.acc[i & 1][half][4][t] = hd.dt * far;
            sm.acc[i & 1][half][3][t] = dd;
            for (int o = 16; o > 0; o >>= 1) sg += __shfl_xor_sync(0xffffffffu, sg, o);
            if (lane == 0) sm.sg[i & 1][threadIdx.x >> 5] = sg;
            mbar_arrive(&sm.bar[B_E]);
            old_a = hd.a;
            old_dt = hd.dt;
            old_whole = hd.whole;
            hd = next;
            near = far = z = x = dd = sg = 0.f;
        }
    }
    ok = ok && finish(heads - 1, old_a, old_dt, old_whole);
    if (!__all_sync(0xffffffffu, ok && !sm.abort_flag)) return;   // (a warp leaves as one: the wait below is a vote)
    // -- the heads' sum as an operand, row j
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *piece(sm.m[half], t, i) = make_uint4(pack2(ms[4 * i]), pack2(ms[4 * i + 1]), pack2(ms[4 * i + 2]), pack2(ms[4 * i + 3]));
    fence_async_smem();
    tc_fence_before();
    mbar_arrive(&sm.bar[B_MS]);
    if (!wait(B_FIN, 0)) return;
    tc_fence_after();
    constexpr int W = N / 2;   // columns of a thread
    const size_t at = (row_out * p.a.G + wk.g) * N + half * W;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *part = which ? p.part_k : p.part_q;
        __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(which ? p.a.dk : p.a.dq) + at;
        if (part) part += (size_t)(blockIdx.x % p.splits) * p.a.rows * p.a.G * N + at;
#pragma unroll
        for (int c = 0; c < W; c += 16) {
            float v[16];
            tmem_ld16(tm + (which ? TM_DK : TM_DQ) + half * W + c, v);
            if (!in) continue;
            if (part) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) store4(part + c + i, make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
            } else {
#pragma unroll
                for (int i = 0; i < 16; i += 8)
                    *reinterpret_cast<uint4 *>(out + c + i) = make_uint4(pack2(f2(v[i], v[i + 1])), pack2(f2(v[i + 2], v[i + 3])), pack2(f2(v[i + 4], v[i + 5])), pack2(f2(v[i + 6], v[i + 7])));
            }
        }
    }
    tc_fence_before();
}

// One warp: products and tiles.
template <int N>
__device__ void issue(Smem &sm, const CUtensorMap *tq, const CUtensorMap *tk, const CUtensorMap *tv, const CUtensorMap *tg, const Params &p, const Work &wk)
{
    constexpr int NB = N / 64;
    constexpr uint32_t T16 = TILE / 16;
    const bool first = (threadIdx.x & 31) == 0;
    const int slices = p.a.P / NS, xk = wk.g * N;
    const uint32_t tm = sm.tmem;
    auto wait = [&](int b, int parity) {
        const bool ok = bar_wait(&sm.bar[b], parity, &sm.abort_flag);
        tc_fence_after();
        return ok;
    };
    auto desc = [](const void *x, uint32_t lbo) { return desc_lo(smem_desc_sw128(smem_u32(x), lbo, 1024)); };
    if (first) {
        mbar_expect_tx(&sm.bar[B_QK], 2 * NB * TILE);
        for (int b = 0; b < NB; ++b) {
            tma_load_2d(sm.k[b], tk, xk + b * 64, wk.tok0, &sm.bar[B_QK]);
            tma_load_2d(sm.q[b], tq, xk + b * 64, wk.tok0, &sm.bar[B_QK]);
        }
    }
    __syncwarp();
    auto load = [&](int it) {
        if (first) {
            const int x = (wk.h0 + it / slices) * p.a.P + it % slices * NS;
            mbar_expect_tx(&sm.bar[B_TILES], 2 * TILE);
            tma_load_2d(sm.v, tv, x, wk.tok0, &sm.bar[B_TILES]);
            tma_load_2d(sm.go, tg, x, wk.tok0, &sm.bar[B_TILES]);
            if (it + 1 < wk.items) {
                const int y = (wk.h0 + (it + 1) / slices) * p.a.P + (it + 1) % slices * NS;
                prefetch_2d(tv, y, wk.tok0);
                prefetch_2d(tg, y, wk.tok0);
            }
        }
        __syncwarp();
    };
    // States on their way to L2, two slices ahead.
    auto fetch = [&](int it) {
        if (first && it < wk.items) {
            const size_t at = (((size_t)wk.slot * p.a.H + wk.h0) * slices + it) * STATE_ELEMS;
            prefetch_l2(p.states + at, STATE_ELEMS * 4);
            prefetch_l2(p.dstates + at, STATE_ELEMS * 4);
        }
        __syncwarp();
    };
    load(0);
    fetch(0);
    fetch(1);
    if (!wait(B_QK, 0) || (wk.m < C && !wait(B_CLEAN0, 0))) return;
    const uint32_t k_km = desc(sm.k, 0), q_km = desc(sm.q, 0), v_km = desc(sm.v, 0), go_km = desc(sm.go, 0), gs_km = desc(sm.gs, 0), vs_km = desc(sm.vs, 0);
    const uint32_t sp_km = desc(sm.sp, 0), m_km = desc(sm.m, 0), m_mn = desc(sm.m, TILE), k_mn = desc(sm.k, TILE), q_mn = desc(sm.q, TILE);
#pragma unroll
    for (int b = 0; b < NB; ++b) mma4_bf16_lo<2, 2>(tm + TM_CB, k_km + b * T16, q_km + b * T16, idesc_bf16(128, 128, 0, 0), b > 0);
    mma_commit(&sm.bar[B_CB]);
#pragma unroll 1
    for (int it = 0; it < wk.items; ++it) {
        if (it > 0) {   // (the tiles and accumulators of the last slice have been read)
            if (!wait(B_FREE, it - 1)) return;
            load(it);
        }
        fetch(it + 2);
        if (!wait(B_S, it)) return;
#pragma unroll 1
        for (int part = 2; part >= 0; --part)   // smallest first
#pragma unroll
            for (int b = 0; b < NB; ++b) mma4_bf16_lo<2, 128>(tm + TM_SG, q_km + b * T16, sp_km + part * T16 + b * 512, idesc_bf16(128, 64, 0, 1), part < 2 || b > 0);
        mma_commit(&sm.bar[B_QS]);
        if (!wait(B_SCALED, it)) return;
        mma4_bf16_lo<2, 2>(tm + TM_DQ, gs_km, sp_km + T16, idesc_bf16(128, N, 0, 0), it > 0);
        mma4_bf16_lo<2, 2>(tm + TM_DQ, gs_km, sp_km, idesc_bf16(128, N, 0, 0), 1);
        mma_commit(&sm.bar[B_DQ]);
        if (!wait(B_TILES, it) || (wk.m < C && !wait(B_CLEAN, it)) || !wait(B_X, it)) return;
        mma4_bf16_lo<2, 2>(tm + TM_DX, v_km, go_km, idesc_bf16(128, 128, 0, 0), 0);
        mma_commit(&sm.bar[B_DX]);
        if (!wait(B_G, it) || !wait(B_M, it)) return;
#pragma unroll 1
        for (int part = 2; part >= 0; --part)
#pragma unroll
            for (int b = 0; b < NB; ++b) mma4_bf16_lo<2, 128>(tm + TM_SG, k_km + b * T16, sp_km + part * T16 + b * 512, idesc_bf16(128, 64, 0, 1), part < 2 || b > 0);
#pragma unroll
        for (int b = 0; b < 2; ++b) mma4_bf16_lo<2, 128>(tm + TM_DV, m_km + b * T16, go_km + b * 512, idesc_bf16(128, 64, 0, 1), b);
        if (p.a.test_timeout) return;   // test hook: the workers' wait for these products runs out
        mma_commit(&sm.bar[B_C2]);
        mma4_bf16_lo<2, 2>(tm + TM_DK, vs_km, sp_km + T16, idesc_bf16(128, N, 0, 0), it > 0);
        mma4_bf16_lo<2, 2>(tm + TM_DK, vs_km, sp_km, idesc_bf16(128, N, 0, 0), 1);
        mma_commit(&sm.bar[B_DK]);
    }
    if (!wait(B_MS, 0)) return;
#pragma unroll
    for (int b = 0; b < 2; ++b) mma4_bf16_lo<2, 128>(tm + TM_DK, m_km + b * T16, q_mn + b * 512, idesc_bf16(128, N, 0, 1), 1);
#pragma unroll
    for (int b = 0; b < 2; ++b) mma4_bf16_lo<128, 128>(tm + TM_DQ, m_mn + b * 512, k_mn + b * 512, idesc_bf16(128, N, 1, 1), 1);
    mma_commit(&sm.bar[B_FIN]);
}

template <int N>
__global__ void __launch_bounds__(NT, 1)
ssm_grads_tc_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                    const __grid_constant__ CUtensorMap tg, const __grid_constant__ Params p)
{
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_dyn);
    if (smem_u32(smem_dyn) & 1023) {
        if (threadIdx.x == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_ALIGN);
        return;
    }
    const int tid = threadIdx.x, per = p.a.H / p.a.G, each = (per + p.splits - 1) / p.splits, split = blockIdx.x % p.splits;
    Work wk;
    wk.g = blockIdx.x / p.splits % p.a.G;
    wk.slot = blockIdx.x / p.splits / p.a.G;
    wk.h0 = wk.g * per + split * each;
    wk.items = min(each, per - split * each) * (p.a.P / NS);
    const Slots slots(p.a.cu_seqlens, p.a.T);
    int n = 0, hi = p.a.n_seq;   // the sequence whose first slot is the last one at or before this
    while (hi - n > 1) {
        const int mid = (n + hi) >> 1;
        if (slots.first(mid) <= (size_t)wk.slot) n = mid;
        else hi = mid;
    }
    const int start = p.a.cu_seqlens ? p.a.cu_seqlens[n] : n * p.a.T, end = p.a.cu_seqlens ? p.a.cu_seqlens[n + 1] : start + p.a.T;
    wk.tok0 = start + (wk.slot - (int)slots.first(n)) * C;
    wk.m = min(C, end - wk.tok0);
    if (wk.m <= 0) {   // a slot that no chunk has
        for (int i = tid; i < 4 * (wk.items / (p.a.P / NS)); i += NT) {
            const size_t at = ((size_t)wk.slot * 4 + (i & 3)) * p.a.H + wk.h0 + (i >> 2);
            p.part_a[at] = p.part_d[at] = 0.f;
        }
        return;
    }
    if (tid == 0) {
        for (int b = 0; b < B_COUNT; ++b)
            mbar_init(&sm.bar[b], b == B_TOT ? 8 : b > B_TOT ? 256 : 1);
        sm.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tq);
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
        tma_prefetch_desc(&tg);
    }
    if (tid >= 256 && tid < 288) tmem_alloc(&sm.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // 384 threads x 168 registers at launch = 128 x (2 x 232 + 40)
    if (tid < 256) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        workers<N>(sm, p, wk);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (tid < 288) issue<N>(sm, &tq, &tk, &tv, &tg, p, wk);
    }
    tc_fence_before();
    __syncthreads();
    if (sm.abort_flag) {   // copies and products issued just before a wait gave up finish first
        for (int i = 0; i < 32; ++i) __nanosleep(1000);
        if (tid == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_TIMEOUT);
    }
    if (tid >= 256 && tid < 288) {
        tc_fence_after();
        tmem_dealloc(sm.tmem, 512);
    }
}

// dq, dk from the partial sums of the blocks that shared a group's heads, in their order
__global__ void __launch_bounds__(256) ssm_join_splits_kernel(const float *part_q, const float *part_k, int splits, size_t n, __nv_bfloat16 *dq, __nv_bfloat16 *dk)
{
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const float *part = blockIdx.y ? part_k : part_q;
    float4 s = load4(part + i);
    for (int k = 1; k < splits; ++k) {
        const float4 t = load4(part + (size_t)k * n + i);
        s = make_float4(s.x + t.x, s.y + t.y, s.z + t.z, s.w + t.w);
    }
    store4((blockIdx.y ? dk : dq) + i, s);
}

// Blocks that share a group's heads: as many as it takes to give every SM one.
int splits_of(const SsmParams &a)
{
    const long long blocks = ((long long)a.rows / C + a.n_seq) * a.G;
    const int per = a.H / a.G, want = (int)(sm_count() / blocks);
    if (want <= 1 || per == 1) return 1;
    const int each = (per + want - 1) / want;
    return (per + each - 1) / each;
}
struct Layout {   // of the workspace, in bytes
    size_t states, dstates, part_a, part_d, part_q, part_k, parts, all;
    int splits;
    explicit Layout(const SsmParams &a)
    {
        const size_t slots = (size_t)a.rows / C + a.n_seq, unit = slots * a.H * (a.P / NS) * STATE_ELEMS * sizeof(float);
        auto up = [](size_t x) { return (x + 255) / 256 * 256; };
        splits = splits_of(a);
        const size_t sums = up(slots * 4 * a.H * sizeof(float)), qk = splits > 1 ? up((size_t)splits * a.rows * a.G * a.N * sizeof(float)) : 0;
        states = 0;
        dstates = unit;
        part_a = dstates + unit;
        part_d = part_a + sums;
        part_q = part_d + sums;
        part_k = part_q + qk;
        parts = part_k + qk;
        all = parts + Parts(a, sm_count(), nullptr).bytes(a);
    }
};

template <int N>
cudaError_t launch_t(const Params &p, cudaStream_t stream)
{
    CUtensorMap tq, tk, tv, tg;
    const uint64_t rows = (uint64_t)p.a.rows, kw = (uint64_t)p.a.G * N, vw = (uint64_t)p.a.H * p.a.P;
    if (!make_map(&tq, p.a.q, rows, kw, p.a.q_stride) || !make_map(&tk, p.a.k, rows, kw, p.a.k_stride) || !make_map(&tv, p.a.v, rows, vw, p.a.v_stride) ||
        !make_map(&tg, p.a.d_out, rows, vw, vw))
        return cudaErrorInvalidValue;
    auto kern = ssm_grads_tc_kernel<N>;
    const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (err != cudaSuccess) return err;
    kern<<<(unsigned)((p.a.rows / C + p.a.n_seq) * p.a.G * p.splits), NT, sizeof(Smem), stream>>>(tq, tk, tv, tg, p);
    count_launch(1);
    return cudaGetLastError();
}

}  // namespace
}  // namespace ssm

size_t ssm_bwd_chunk_workspace_bytes(const SsmParams &a) { return ssm::Layout(a).all; }

cudaError_t launch_ssm_bwd_chunk(const SsmParams &a, cudaStream_t stream)
{
    using namespace ssm;
    const Layout l(a);
    char *ws = static_cast<char *>(a.workspace);
    auto at = [&](size_t x) { return reinterpret_cast<float *>(ws + x); };
    const Parts parts(a, sm_count(), ws + l.parts);
    for (int reverse = 0; reverse < 2; ++reverse) {
        cudaError_t err = cudaSuccess;
        if (parts.n > 1) err = launch_part_starts(a, parts, reverse, stream);
        if (err == cudaSuccess) err = launch_chunk_states(a, parts, reverse, at(reverse ? l.dstates : l.states), stream);
        if (err != cudaSuccess) return err;
    }
    const bool split = l.splits > 1;
    const Params p = {a, at(l.states), at(l.dstates), at(l.part_a), at(l.part_d), split ? at(l.part_q) : nullptr, split ? at(l.part_k) : nullptr, l.splits};
    cudaError_t err = a.N == 64 ? launch_t<64>(p, stream) : launch_t<128>(p, stream);
    if (err != cudaSuccess) return err;
    if (split) {
        const size_t n = (size_t)a.rows * a.G * a.N;
        ssm_join_splits_kernel<<<dim3((unsigned)((n / 4 + 255) / 256), 2), 256, 0, stream>>>(p.part_q, p.part_k, l.splits, n, static_cast<__nv_bfloat16 *>(a.dq), static_cast<__nv_bfloat16 *>(a.dk));
        count_launch(1);
    }
    return launch_ssm_sums(p.part_a, p.part_d, (int)((a.rows / C + a.n_seq) * 4), a.H, a.da, a.dd, stream);
}

}  // namespace kla
