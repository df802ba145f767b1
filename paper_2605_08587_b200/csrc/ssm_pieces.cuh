// Pieces of the tensor-core kernels of the selective state space scan (ssm_chunk.cu, ssm_bwd.cu): chunks of 128 tokens.
#pragma once
#include <cuda.h>

#include "layer_ops.h"
#include "scan_pieces.cuh"
#include "umma.cuh"

namespace kla {
namespace ssm {

using namespace umma;

constexpr int C = 128;        // chunk length: the rows of one tcgen05 product
constexpr int NS = 64;        // columns of the state (channels of v) per block: one 128-byte row of a tile
constexpr uint32_t WAIT_LIMIT = 2000000000u;   // SM clocks (~1 s) before a wait gives up
constexpr float LOG2E = 1.4426950408889634f;
constexpr uint32_t TILE = C * 128;             // bytes of a tile: 128 rows of 64 bf16, 128-byte swizzle

__device__ __forceinline__ uint32_t clock_lo()
{
    uint32_t t;
    asm volatile("mov.u32 %0, %%clock;" : "=r"(t));
    return t;
}
// Every lane polls; the warp leaves together.  Gives up after WAIT_LIMIT, or once another role of the block has.
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    bool ok = mbar_try_wait(bar, parity & 1);
    if (!ok) {
        const uint32_t t0 = clock_lo();
#pragma unroll 1
        do {
            ok = mbar_try_wait(bar, parity & 1);
        } while (!ok && !*abort_flag && clock_lo() - t0 < WAIT_LIMIT);
        if (!ok) *abort_flag = 1;
    }
    return __all_sync(0xffffffffu, ok);
}

// One arrival for the whole warp (a barrier takes those of 32 lanes one after another), of what all its lanes have done before.
__device__ __forceinline__ void warp_arrive(uint64_t *bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// Asks for a box of a tensor map to be brought into L2.
__device__ __forceinline__ void prefetch_2d(const void *tmap, int x, int y)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(tmap), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void *x, int bytes)   // (multiples of 16)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(x), "r"(bytes) : "memory");
}
__device__ __forceinline__ void prefetch_line(const void *x) { asm volatile("prefetch.global.L2 [%0];" ::"l"(x)); }

// Few long sequences are cut into parts of whole chunks.
struct Parts {
    int n, seg_len;      // parts of a sequence, tokens of each (the last may be shorter, later ones empty)
    float *state;        // [n_seq n][H][N][P]: what a part adds to a state of zero, then the state it starts from
    float *decay;        // [n_seq n][H]: the whole part's decay
    // Cut where the blocks of whole sequences would leave more than half the SMs without work and it pays: a chunk takes about 2.6 us in the
    // output kernel and 1.5 in the pass over the states before it, which also costs two launches, 8 us.  (65 536 tokens, H8 d 128: whole
    // 1 295 us, in nine parts 305; 777 tokens of 32 heads: whole 25 us, in four parts 29.)
    Parts(const SsmParams &a, int sms, void *workspace) : n(1), seg_len(0), state(nullptr), decay(nullptr)
    {
        int longest = a.T;
        if (a.host_seqlens) {
            longest = 0;
            for (int i = 0; i < a.n_seq; ++i) longest = longest > a.host_seqlens[i + 1] - a.host_seqlens[i] ? longest : a.host_seqlens[i + 1] - a.host_seqlens[i];
        }
        const long long units = (long long)a.n_seq * a.H * (a.P / NS);
        const int chunks = (longest + C - 1) / C;
        if (!a.whole && 2 * units <= sms) {
            const int want = (int)(sms / units), each = (chunks + want - 1) / want;
            if (each > 0 && 2.6f * chunks > 1.2f * (8.f + 4.1f * each)) n = (chunks + each - 1) / each;
        }
        seg_len = n > 1 ? (chunks + n - 1) / n * C : (chunks > 0 ? chunks : 1) * C;
        if (n > 1 && workspace) {
            state = static_cast<float *>(workspace);
            decay = state + (size_t)a.n_seq * n * a.H * a.N * a.P;
        }
    }
    size_t bytes(const SsmParams &a) const { return n > 1 ? ((size_t)a.n_seq * n * a.H * ((size_t)a.N * a.P + 1) * sizeof(float) + 255) / 256 * 256 : 0; }
};
struct Piece {
    int n, g, tok0, len;
    bool last;   // holds the sequence's end (the first part, of an empty one)
    __device__ __forceinline__ Piece(const int32_t *cu, int T, const Parts &parts, int index)
    {
        n = index / parts.n;
        g = index % parts.n;
        const int start = cu ? cu[n] : n * T, end = cu ? cu[n + 1] : start + T;
        tok0 = start + min(end - start, g * parts.seg_len);
        len = min(parts.seg_len, end - tok0);
        last = len > 0 ? tok0 + len == end : g == 0;
    }
};

// Row r of a tile as stored (16-byte pieces permuted)
__device__ __forceinline__ uint4 *piece(unsigned char *tile, int r, int c) { return reinterpret_cast<uint4 *>(tile + sw128(r, c)); }

__device__ __forceinline__ float2 unpack2(uint32_t x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(float2 x)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t *>(&p);
}
// The bf16 part of x, which keeps the rest.
__device__ __forceinline__ uint32_t part(float2 &x)
{
    const uint32_t h = pack2(x);
    x = fma2(unpack2(h), f2(-1.f), x);   // exact
    return h;
}

constexpr int HS = NS / 2;   // columns of the state of a thread: it holds half a row
// S <- gamma S + (what a chunk adds: three parts, 64 columns of tensor memory apart)
__device__ __forceinline__ void join(float2 (&S)[HS / 2], uint32_t tm, float gamma)
{
    const float2 g = f2(gamma);
#pragma unroll
    for (int c = 0; c < HS; c += 16) {
        float h[16], m[16], l[16];
        tmem_ld16(tm + c, h);
        tmem_ld16(tm + 64 + c, m);
        tmem_ld16(tm + 128 + c, l);
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float2 sum = add2(add2(f2(l[e], l[e + 1]), f2(m[e], m[e + 1])), f2(h[e], h[e + 1]));
            S[(c + e) / 2] = fma2(g, S[(c + e) / 2], sum);
        }
    }
}
__device__ __forceinline__ void read_row(float2 (&S)[HS / 2], const float *from)
{
#pragma unroll
    for (int c = 0; c < HS / 2; c += 2) {
        const float4 t = from ? load4(from + 2 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        S[c] = f2(t.x, t.y);
        S[c + 1] = f2(t.z, t.w);
    }
}
__device__ __forceinline__ void write_row(const float2 (&S)[HS / 2], float *to)
{
#pragma unroll
    for (int c = 0; c < HS / 2; c += 2) store4(to + 2 * c, make_float4(S[c].x, S[c].y, S[c + 1].x, S[c + 1].y));
}
__device__ __forceinline__ void zero_half_row(unsigned char *tile, int row, int half)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) *piece(tile, row, 4 * half + c) = make_uint4(0u, 0u, 0u, 0u);
}

// Chunk c of sequence n has slot first(n) + c: slots of different sequences do not meet, and there are at most rows / C + n_seq of them.
struct Slots {
    const int32_t *cu;
    int T;
    __device__ __forceinline__ Slots(const int32_t *cu_, int T_) : cu(cu_), T(T_) {}
    __device__ __forceinline__ size_t first(int n) const { return (size_t)((cu ? cu[n] : n * T) / C) + n; }
};
// Elements of a stored state of one head and 64 columns: piece i of thread t of 256 (row t & 127, columns 32 (t >> 7) + 4 i ..) at (256 i + t) 4.
constexpr int STATE_ELEMS = 128 * NS;

// Scalars of a chunk, a thread to a token.  Sums of log2 decays run inside blocks of 32 tokens (a warp): decays between tokens of a block are
// exponentials of differences of short sums; those from a token to its block's end come from a sum of their own, so that they are accurate
// however far the block's start lies back.  Sums whose differences count carry their rounding errors in a second float: behind tokens that decay strongly
// they are large, and the decay between two ordinary ones there would have only the digits that one float leaves (sums of 3 000: 2^-13).
//   a2 + lo inclusive sum inside the block
//   cf = dt 2^(sum of what follows in the block)
//   nn = -n, f: a2 + lo = n + f with n whole;  dtf = dt 2^-f.  L_ij dt_j = 2^(n_i - n_j + f_i) dtf_j, where n_i - n_j is exact
// A token's log2 decay below NO_DECAY counts as that (its power of two is zero in fp32 all the same), however large its step: sums stay below 2^15, where
// two floats hold them to 2^-33.
constexpr float NO_DECAY = -1024.f;
struct alignas(16) Scalars {
    float nn[C], f[C], cf[C], dtf[C];
};
template <bool DIFFERENCES>   // whether differences of a2 are taken (else lo is zero)
struct BlockScan {
    float a2, lo, rest, tot;   // inclusive sum, what follows to the block's end, the whole block
    __device__ __forceinline__ BlockScan(float dt, float a)
    {
        const int lane = threadIdx.x & 31;
        const float l = dt * a * LOG2E, x = l < NO_DECAY ? NO_DECAY : l;   // (NaN stays)
        float up = x, err = 0.f, down = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float t = __shfl_up_sync(0xffffffffu, up, o), u = __shfl_down_sync(0xffffffffu, down, o);
            if constexpr (DIFFERENCES) {
                const float te = __shfl_up_sync(0xffffffffu, err, o);
                const float sum = up + t, b = sum - up, e = (up - (sum - b)) + (t - b);   // sum + e = up + t
                if (lane >= o) err += te + e;
                if (lane >= o) up = sum;
            } else {
                if (lane >= o) up += t;
            }
            if (lane + o < 32) down += u;
        }
        a2 = up;
        lo = err;
        const float behind = __shfl_down_sync(0xffffffffu, down, 1);
        rest = lane < 31 ? behind : 0.f;
        tot = __shfl_sync(0xffffffffu, down, 0);
    }
};

// State passes (ssm_state.cu).  The states that the parts of a sequence start from: forward the state before the part, in reverse the gradient
// of the state behind it.
cudaError_t launch_part_starts(const SsmParams &a, const Parts &parts, bool reverse, cudaStream_t stream);
// The state before every chunk (reverse: the gradient of the state behind it) to states[slot of the chunk], see Slots; the gradient of the initial
// state to a.dinit.
cudaError_t launch_chunk_states(const SsmParams &a, const Parts &parts, bool reverse, float *states, cudaStream_t stream);

// Tensor map of a bf16 [rows][cols] array, rows `stride` elements apart, boxes of 128 rows x 64 elements, 128-byte swizzle.
bool make_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint64_t stride);

}  // namespace ssm
}  // namespace kla
