// Pieces shared by the operators around a mixer (conv.cu, norm.cu, ssm_scan.cu).
#pragma once
#include "common.cuh"

namespace kla {

// N consecutive elements as loaded, converted on use.  N = 1 serves arrays whose rows do not start on 16-byte boundaries.
template <typename IO, int N>
struct Pack;
template <int N>
struct Pack<float, N> {
    float r[N];
    __device__ __forceinline__ void load(const float *p)
    {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float4 x = *reinterpret_cast<const float4 *>(p + 4 * i);
                r[4 * i] = x.x; r[4 * i + 1] = x.y; r[4 * i + 2] = x.z; r[4 * i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = p[i];
        }
    }
    __device__ __forceinline__ void store(float *p) const
    {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) *reinterpret_cast<float4 *>(p + 4 * i) = make_float4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = r[i];
        }
    }
    __device__ __forceinline__ float get(int i) const { return r[i]; }
    __device__ __forceinline__ void set(const float (&x)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = x[i];
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = 0.f;
    }
};
template <>
struct Pack<__nv_bfloat16, 1> {
    __nv_bfloat16 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *p; }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *p = r; }
    __device__ __forceinline__ float get(int) const { return __bfloat162float(r); }
    __device__ __forceinline__ void set(const float (&x)[1]) { r = __float2bfloat16_rn(x[0]); }
    __device__ __forceinline__ void zero() { r = __float2bfloat16_rn(0.f); }
};
template <int N>
struct Pack<__nv_bfloat16, N> {
    static_assert(N == 4 || N == 8, "whole words");
    uint32_t r[N / 2];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        if constexpr (N == 8) {
            const uint4 x = *reinterpret_cast<const uint4 *>(p);
            r[0] = x.x; r[1] = x.y; r[2] = x.z; r[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(p);
            r[0] = x.x; r[1] = x.y;
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const
    {
        if constexpr (N == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(r[0], r[1], r[2], r[3]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(r[0], r[1]);
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16); }
    __device__ __forceinline__ void set(const float (&x)[N])
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            r[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) r[i] = 0u;
    }
};

// First row of sequence n, and the sequence that row r belongs to (the last one that starts at or before it: never an empty one).
struct Sequences {
    const int32_t *cu;   // null: n_seq sequences of T rows
    int32_t T, n_seq;
    __device__ __forceinline__ int start(int n) const { return cu ? cu[n] : n * T; }
    __device__ __forceinline__ int of_row(int r) const
    {
        if (!cu) return T ? r / T : 0;
        int lo = 0, hi = n_seq;   // cu[lo] <= r < cu[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cu[mid] <= r) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x)   // off by at most one in the last place; 0 beyond 2^126
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / (1 + exp(-x)).  exp overflows to infinity for x < -88 and the quotient is then 0, as it should be.
__device__ __forceinline__ float sigmoid(float x) { return rcp_fast(1.f + exp2_fast(x * -1.4426950408889634f)); }

// Sums of n partials [n][M] in a fixed order: a block takes 32 columns, each of its 16 warps every 16th partial; store(i, sum).
template <typename F>
__device__ __forceinline__ void sum_partials(const float *partial, int n, int M, F store)
{
    __shared__ float part[16][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (i < M) {
        int k = warp;
        for (; k + 112 < n; k += 128) {   // eight in flight
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = partial[(size_t)(k + 16 * u) * M + i];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += x[u];
        }
        for (; k < n; k += 16) s += partial[(size_t)k * M + i];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < M) {
        for (int k = 1; k < 16; ++k) s += part[k][lane];
        store(i, s);
    }
}

}  // namespace kla
