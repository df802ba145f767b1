// Pieces of the tensor-core kernels of the selective state space scan (ssm_chunk.cu, ssm_bwd.cu): chunks of 128 tokens.
#pragma once
#include <cuda.h>

#include "layer_ops.h"
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

// Asks for a box of a tensor map to be brought into L2.
__device__ __forceinline__ void prefetch_2d(const void *tmap, int x, int y)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(tmap), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ void prefetch_line(const void *x) { asm volatile("prefetch.global.L2 [%0];" ::"l"(x)); }

// Part g of `parts` equal ones of sequence n, in whole chunks (the last may be shorter, later ones empty).
struct Piece {
    int n, tok0, len;
    bool last;   // holds the sequence's end (its final state is the sequence's)
    __device__ __forceinline__ Piece(const int32_t *cu, int T, int parts, int seg_len, int index)
    {
        n = index / parts;
        const int g = index % parts, start = cu ? cu[n] : n * T, end = cu ? cu[n + 1] : start + T;
        tok0 = start + g * seg_len;
        len = min(seg_len, end - tok0);
        last = len > 0 ? tok0 + len == end : g == 0 && start == end;
    }
};

// Scalars of a chunk, a thread to a token.  Sums of log2 decays run inside blocks of 32 tokens (a warp): decays between tokens of a block are
// exponentials of differences of short sums; those from a token to its block's end come from a sum of their own, so that they are accurate
// however far the block's start lies back.
//   a2 inclusive sum inside the block
//   r = 2^a2 (from the block's start);  cf = dt 2^(sum of what follows in the block)
struct alignas(16) Scalars {
    float a2[C], r[C], cf[C], dt[C];
};
struct BlockScan {
    float a2, rest, tot;   // inclusive sum, what follows to the block's end, the whole block
    __device__ __forceinline__ BlockScan(float dt, float a)
    {
        const int lane = threadIdx.x & 31;
        const float x = dt * a * LOG2E;
        float up = x, down = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float t = __shfl_up_sync(0xffffffffu, up, o), u = __shfl_down_sync(0xffffffffu, down, o);
            if (lane >= o) up += t;
            if (lane + o < 32) down += u;
        }
        a2 = up;
        const float behind = __shfl_down_sync(0xffffffffu, down, 1);
        rest = lane < 31 ? behind : 0.f;
        tot = __shfl_sync(0xffffffffu, down, 0);
    }
};

// Tensor map of a bf16 [rows][cols] array, rows `stride` elements apart, boxes of 128 rows x 64 elements, 128-byte swizzle.
bool make_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint64_t stride);

}  // namespace ssm
}  // namespace kla
