// State passes of the selective state space scan on the tensor cores, without outputs: what the reverse mode needs of the states, and what the parts of a
// long sequence start from.  Chunks of 128 tokens as in ssm_chunk.cu:
//
//     forward   S' = e^{l_Q} S + sum_j k_j (dt_j e^{l_Q - l_j} v_j)^T        from the first chunk to the last
//     reverse   G' = e^{l_Q} G + sum_i q_i (e^{l_i} do_i)^T                  from the last to the first: G behind a chunk -> G before it
//
// the same kernel with other tiles, weights and order.  One product per chunk, k^T [w v in three bf16 parts]; the state stays in registers, in
// fp32.  A chunk is one chain (decays, weights, product, state), so two blocks share an SM and fill each other's gaps: 112 KB of tiles each,
// 256 columns of tensor memory.  v comes a chunk ahead and the next decays are formed while the product runs; k, needed last, is there once.  A pass over
// 8 x 4096 tokens of 32 heads (N = 128) that writes every chunk's state, 268 MB: about 105 us.
#include "ssm_pieces.cuh"

namespace kla {
namespace ssm {

namespace {

constexpr int NT = 256 + 32;   // 256 work, one warp issues and loads

enum Bar { B_K = 0, B_X /* of even and odd chunks */, B_TOT = B_X + 2, B_WX, B_DS, B_COUNT };

struct Smem {
    alignas(1024) unsigned char k[2][TILE];   // k (reverse: q): [64 of N][token][64]
    alignas(1024) unsigned char x[2][TILE];   // v (reverse: do) of chunks in turn: [token][64 columns]
    alignas(1024) unsigned char w[3][TILE];   // parts of the weighted v
    float tot[2][4];
    alignas(8) uint64_t bar[B_COUNT];
    uint32_t tmem;
    volatile int abort_flag;
};
static_assert(sizeof(Smem) <= 115712, "two blocks to an SM");

struct Params {
    SsmParams a;
    Parts parts;
    float *states;   // null: only the last state, and the decay, of each part
};

// w v of all tokens, a thread to half the columns of a token
__device__ __forceinline__ void weigh(const unsigned char *x, unsigned char (*w)[TILE], float weight)
{
    const int row = threadIdx.x & 127, half = threadIdx.x >> 7;
    const float2 w2 = f2(weight);
#pragma unroll 2
    for (int i = 0; i < 4; ++i) {
        const uint32_t at = sw128(row, 4 * half + i);
        const uint4 raw = *reinterpret_cast<const uint4 *>(x + at);
        float2 v[4] = {mul2(unpack2(raw.x), w2), mul2(unpack2(raw.y), w2), mul2(unpack2(raw.z), w2), mul2(unpack2(raw.w), w2)};
        *reinterpret_cast<uint4 *>(w[0] + at) = make_uint4(part(v[0]), part(v[1]), part(v[2]), part(v[3]));
        *reinterpret_cast<uint4 *>(w[1] + at) = make_uint4(part(v[0]), part(v[1]), part(v[2]), part(v[3]));
        *reinterpret_cast<uint4 *>(w[2] + at) = make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3]));
    }
}

template <int N, bool REV>
__device__ void work(Smem &sm, const Params &p, const Piece &pc, int h, int sl, int index, const float *init, float *fin)
{
    // thread t and t + 128: token t, row t of the state, each half the columns
    const int t = threadIdx.x & 127, half = threadIdx.x >> 7, lane = t & 31, warp = t >> 5;
    const bool row = N == 128 || t < N;
    const int chunks = (pc.len + C - 1) / C;
    const uint32_t tm = sm.tmem + half * HS + ((uint32_t)(warp * 32) << 16);
    float2 S[HS / 2];
    read_row(S, init && row ? init + (size_t)t * p.a.P + half * HS : nullptr);
    const float a = p.a.a[h];
    const float *dtp = p.a.dt + (size_t)pc.tok0 * p.a.H + h;
    auto token = [&](int cx) { return (REV ? chunks - 1 - cx : cx) * C + t; };   // of the cx-th chunk in order
    float dt = token(0) < pc.len ? dtp[(size_t)token(0) * p.a.H] : 0.f, total = 0.f;
    const Slots slots(p.a.cu_seqlens, p.a.T);
    float *out = p.states ? p.states + (((slots.first(pc.n) + pc.g * (p.parts.seg_len / C)) * p.a.H + h) * (p.a.P / NS) + sl) * STATE_ELEMS + threadIdx.x * 4 : nullptr;
    const size_t out_step = (size_t)p.a.H * (p.a.P / NS) * STATE_ELEMS;
    // This token's weight in the cx-th chunk, and the chunk's decay
    auto decays = [&](int cx, float &w, float &gamma) {
        const BlockScan<false> b(dt, a);
        float *tot = sm.tot[cx & 1];   // (of two chunks before: read before the last one's product)
        if (lane == 0) {
            if (half == 0) tot[warp] = b.tot;
            mbar_arrive(&sm.bar[B_TOT]);
        }
        w = token(cx) < pc.len ? (REV ? exp2f(b.a2) : dt * exp2f(b.rest)) : 0.f;
        if (cx + 1 < chunks) dt = token(cx + 1) < pc.len ? dtp[(size_t)token(cx + 1) * p.a.H] : 0.f;
        if (!bar_wait(&sm.bar[B_TOT], cx, &sm.abort_flag)) return false;
        const float t0 = tot[0], t1 = tot[1], t2 = tot[2], t3 = tot[3];
        w *= exp2f(REV ? (warp == 0 ? 0.f : warp == 1 ? t0 : warp == 2 ? t0 + t1 : t0 + t1 + t2)
                       : (warp == 0 ? t1 + t2 + t3 : warp == 1 ? t2 + t3 : warp == 2 ? t3 : 0.f));
        gamma = exp2f(t0 + t1 + t2 + t3);
        total += t0 + t1 + t2 + t3;
        return true;
    };
    float w = 0.f, gamma = 0.f, next_gamma = 0.f;
    bool ok = decays(0, w, gamma);
#pragma unroll 1
    for (int cx = 0; ok && cx < chunks; ++cx) {
        const int c = REV ? chunks - 1 - cx : cx, m = min(C, pc.len - c * C);
        if (!(ok = bar_wait(&sm.bar[B_X + (cx & 1)], cx >> 1, &sm.abort_flag))) break;
        if (m < C) {   // rows behind the sequence's end: another sequence's, perhaps not finite; nothing of them may meet a zero weight
            if (!(ok = bar_wait(&sm.bar[B_K], cx, &sm.abort_flag))) break;
            if (t >= m) {
                zero_half_row(sm.x[cx & 1], t, half);
#pragma unroll
                for (int b2 = 0; b2 < N / 64; ++b2) zero_half_row(sm.k[b2], t, half);
            }
        }
        weigh(sm.x[cx & 1], sm.w, w);
        fence_async_smem();
        tc_fence_before();
        warp_arrive(&sm.bar[B_WX]);
        // While the product runs: the state before this chunk (in order) in a layout of whole cache lines (piece, thread, four columns), and the next
        // chunk's decays
        if (out) {
#pragma unroll
            for (int i = 0; i < HS / 4; ++i) store4(out + c * out_step + i * 1024, make_float4(S[2 * i].x, S[2 * i].y, S[2 * i + 1].x, S[2 * i + 1].y));
        }
        if (cx + 1 < chunks && !(ok = decays(cx + 1, w, next_gamma))) break;
        if (!(ok = bar_wait(&sm.bar[B_DS], cx, &sm.abort_flag))) break;
        tc_fence_after();
        join(S, tm, gamma);
        gamma = next_gamma;
    }
    tc_fence_before();
    if (!ok || sm.abort_flag) return;
    if (fin && row) write_row(S, fin + (size_t)t * p.a.P + half * HS);
    if (!p.states && threadIdx.x == 0 && sl == 0) p.parts.decay[(size_t)index * p.a.H + h] = exp2f(total);
}

template <int N, bool REV>
__global__ void __launch_bounds__(NT, 2)
ssm_state_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const __grid_constant__ Params p)
{
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_dyn);
    if (smem_u32(smem_dyn) & 1023) {
        if (threadIdx.x == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_ALIGN);
        return;
    }
    constexpr int NB = N / 64;
    const int tid = threadIdx.x, slices = p.a.P / NS, sl = blockIdx.x % slices, h = blockIdx.x / slices % p.a.H, index = blockIdx.x / slices / p.a.H;
    const Piece pc(p.a.cu_seqlens, p.a.T, p.parts, index);
    const size_t head = ((size_t)h * N) * p.a.P + sl * NS, state = (size_t)p.a.H * N * p.a.P;
    const bool cut = p.parts.n > 1;
    const float *whole = REV ? p.a.d_final : p.a.init_state;
    const float *init = !p.states ? nullptr : cut ? p.parts.state + index * state + head : whole ? whole + pc.n * state + head : nullptr;
    // what leaves the block: a part's own contribution, or (reverse) the gradient of the initial state
    float *fin = !p.states ? p.parts.state + index * state + head : REV && p.a.dinit && pc.g == 0 ? p.a.dinit + pc.n * state + head : nullptr;
    if (pc.len <= 0) {   // an empty part: nothing is added, nothing decays
        const size_t at = (size_t)(tid >> 1) * p.a.P + (tid & 1) * HS;
        if (fin && tid < 2 * N) {
            float2 S[HS / 2];
            read_row(S, init ? init + at : nullptr);
            write_row(S, fin + at);
        }
        if (!p.states && tid == 0 && sl == 0) p.parts.decay[(size_t)index * p.a.H + h] = 1.f;
        return;
    }
    if (tid == 0) {
        for (int b = 0; b < B_COUNT; ++b) mbar_init(&sm.bar[b], b == B_TOT || b == B_WX ? 8 : 1);
        sm.abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
    }
    if (tid >= 256) tmem_alloc(&sm.tmem, 256);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (tid < 256) {
        work<N, REV>(sm, p, pc, h, sl, index, init, fin);
    } else {
        const int chunks = (pc.len + C - 1) / C, xk = h / (p.a.H / p.a.G) * N, xv = h * p.a.P + sl * NS;
        const uint32_t k_mn = desc_lo(smem_desc_sw128(smem_u32(sm.k), NB == 2 ? TILE : 0, 1024)), w_mn = desc_lo(smem_desc_sw128(smem_u32(sm.w), TILE, 1024));
#pragma unroll 1
        for (int cx = 0; cx < chunks; ++cx) {
            auto y = [&](int i) { return pc.tok0 + (REV ? chunks - 1 - i : i) * C; };
            if (tid == 256) {   // k is there for one chunk, v a chunk ahead; more on their way to L2 meanwhile
                auto values = [&](int i) {
                    mbar_expect_tx(&sm.bar[B_X + (i & 1)], TILE);
                    tma_load_2d(sm.x[i & 1], &tv, xv, y(i), &sm.bar[B_X + (i & 1)]);
                };
                if (cx == 0) values(0);
                mbar_expect_tx(&sm.bar[B_K], NB * TILE);
                for (int b = 0; b < NB; ++b) tma_load_2d(sm.k[b], &tk, xk + b * 64, y(cx), &sm.bar[B_K]);
                if (cx + 1 < chunks) {
                    values(cx + 1);
                    for (int b = 0; b < NB; ++b) prefetch_2d(&tk, xk + b * 64, y(cx + 1));
                }
                if (cx + 2 < chunks) prefetch_2d(&tv, xv, y(cx + 2));
            }
            __syncwarp();
            if (cx + 2 < chunks)
                for (int i = tid & 31; i < C; i += 32) {
                    const int tok = y(cx + 2) + i;
                    if (tok < pc.tok0 + pc.len) prefetch_line(p.a.dt + (size_t)tok * p.a.H + h);
                }
            if (!bar_wait(&sm.bar[B_K], cx, &sm.abort_flag) || !bar_wait(&sm.bar[B_WX], cx, &sm.abort_flag)) break;
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < 2; ++b) mma4_bf16_lo<128, 128>(sm.tmem, k_mn + b * 512, w_mn + b * 512, idesc_bf16(128, 192, 1, 1), b);
            mma_commit(&sm.bar[B_DS]);
            if (!bar_wait(&sm.bar[B_DS], cx, &sm.abort_flag)) break;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (sm.abort_flag) {   // copies and products issued just before a wait gave up finish first
        for (int i = 0; i < 32; ++i) __nanosleep(1000);
        if (tid == 0 && p.a.status_word) atomicExch(p.a.status_word, (int)KLA_ERR_TIMEOUT);
    }
    if (tid >= 256) {
        tc_fence_after();
        tmem_dealloc(sm.tmem, 256);
    }
}

// What the parts add -> what they start from, in place: four elements of a state to a thread.
__global__ void __launch_bounds__(256) ssm_parts_kernel(Parts parts, const float *first, int H, int elems, bool reverse)
{
    const int e = (blockIdx.x * 256 + threadIdx.x) * 4, h = blockIdx.y, n = blockIdx.z;
    if (e >= elems) return;
    float4 s = first ? load4(first + ((size_t)n * H + h) * elems + e) : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < parts.n; ++i) {
        const size_t at = ((size_t)n * parts.n + (reverse ? parts.n - 1 - i : i)) * H + h;
        const float4 add = load4(parts.state + at * elems + e);
        const float d = parts.decay[at];
        store4(parts.state + at * elems + e, s);
        s = make_float4(fmaf(d, s.x, add.x), fmaf(d, s.y, add.y), fmaf(d, s.z, add.z), fmaf(d, s.w, add.w));
    }
}

template <int N, bool REV>
cudaError_t launch_t(const Params &p, cudaStream_t stream)
{
    CUtensorMap tk, tv;
    const uint64_t rows = (uint64_t)p.a.rows, kw = (uint64_t)p.a.G * N, vw = (uint64_t)p.a.H * p.a.P;
    if (!make_map(&tk, REV ? p.a.q : p.a.k, rows, kw, REV ? p.a.q_stride : p.a.k_stride) ||
        !make_map(&tv, REV ? p.a.d_out : p.a.v, rows, vw, REV ? (int64_t)vw : p.a.v_stride))
        return cudaErrorInvalidValue;
    auto kern = ssm_state_kernel<N, REV>;
    const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (err != cudaSuccess) return err;
    kern<<<(unsigned)(p.a.n_seq * p.parts.n) * p.a.H * (p.a.P / NS), NT, sizeof(Smem), stream>>>(tk, tv, p);
    count_launch(1);
    return cudaGetLastError();
}
cudaError_t launch(const Params &p, bool reverse, cudaStream_t stream)
{
    if (p.a.N == 64) return reverse ? launch_t<64, true>(p, stream) : launch_t<64, false>(p, stream);
    return reverse ? launch_t<128, true>(p, stream) : launch_t<128, false>(p, stream);
}

}  // namespace

cudaError_t launch_part_starts(const SsmParams &a, const Parts &parts, bool reverse, cudaStream_t stream)
{
    const cudaError_t err = launch({a, parts, nullptr}, reverse, stream);
    if (err != cudaSuccess) return err;
    const int elems = a.N * a.P;
    ssm_parts_kernel<<<dim3((unsigned)((elems + 1023) / 1024), (unsigned)a.H, (unsigned)a.n_seq), 256, 0, stream>>>(parts, reverse ? a.d_final : a.init_state, a.H, elems, reverse);
    count_launch(1);
    return cudaGetLastError();
}
cudaError_t launch_chunk_states(const SsmParams &a, const Parts &parts, bool reverse, float *states, cudaStream_t stream)
{
    return launch({a, parts, states}, reverse, stream);
}

}  // namespace ssm
}  // namespace kla
