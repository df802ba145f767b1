// Launchers of the operators around a mixer; each returns cudaGetLastError().
#pragma once
#include <initializer_list>
#include <type_traits>

#include "common.cuh"

namespace kla {

// Short causal convolution (conv.cu).
struct ConvParams {
    const void *x;                // [rows, C], rows x_stride elements apart
    const float *weight, *bias;   // [C, taps], [C] or null
    const void *init_state;       // [n_seq, taps - 1, C] or null
    void *out;                    // [rows, C]
    void *final_state;            // [n_seq, taps - 1, C]: forward, or null; the state of a step, updated in place
    const int32_t *cu_seqlens;    // null: fixed length T
    int64_t x_stride;
    int32_t rows, C, taps, T, n_seq;
    bool silu;
    // backward
    const void *d_out;            // [rows, C]
    const void *d_final;          // as final_state, or null
    void *dx;                     // [rows, C]
    float *dweight, *dbias;       // [C, taps], [C] or null
    void *dinit;                  // as init_state, or null
    float *partial;               // workspace
};
size_t conv_bwd_workspace_bytes(int C, int taps, int rows);
cudaError_t launch_conv_fwd(const ConvParams &p, int io_dtype, cudaStream_t stream);
cudaError_t launch_conv_step(const ConvParams &p, int io_dtype, cudaStream_t stream);
cudaError_t launch_conv_bwd(const ConvParams &p, int io_dtype, cudaStream_t stream);

// Norms (norm.cu).
struct NormParams {
    const void *x;                // [rows, width], rows x_stride elements apart
    const void *gate;             // [rows, width], rows gate_stride apart, or null
    const void *residual;         // [rows, width] of its own dtype, or null
    const float *scale;           // [width] or null (1): on x before it joins the residual
    const float *weight;          // [width]
    void *out;                    // [rows, width]
    void *residual_out;           // as residual
    int64_t x_stride, gate_stride;
    int32_t rows, width, group;
    float eps;
    bool gate_first;
    // backward
    const void *d_out;            // [rows, width]
    const void *d_residual_out;   // as residual, or null
    void *dx, *dgate;             // [rows, width]
    void *dresidual;              // as residual
    float *dweight, *dscale;      // [width]; dscale null without scale
    float *partial;               // workspace
};
size_t norm_bwd_workspace_bytes(int rows, int width, int group);
cudaError_t launch_norm_fwd(const NormParams &p, int io_dtype, int res_dtype, cudaStream_t stream);
cudaError_t launch_norm_bwd(const NormParams &p, int io_dtype, int res_dtype, cudaStream_t stream);

// Selective state space scan.  ssm_scan.cu: any sizes, fp32 arithmetic on CUDA cores.
struct SsmParams {
    const void *q, *k;            // [rows, G, N], rows q_stride / k_stride elements apart
    const void *v;                // [rows, H, P], rows v_stride apart
    const float *dt;              // [rows, H]
    const float *a, *skip;        // [H]; skip may be null
    const float *init_state;      // [n_seq, H, N, P] or null
    void *out;                    // [rows, H, P]
    float *final_state;           // [n_seq, H, N, P] or null; the state of a step, updated in place
    const int32_t *cu_seqlens;    // null: fixed length T
    const int32_t *host_seqlens;  // host copy
    int64_t q_stride, k_stride, v_stride;
    int32_t rows, T, n_seq, H, G, N, P;
    int32_t *status_word;         // or null
    int32_t test_timeout;
    int32_t whole;                // sequences are never cut into parts
    void *workspace;
    // backward
    const void *d_out;            // [rows, H, P]
    const float *d_final;         // [n_seq, H, N, P] or null
    void *dq, *dk, *dv;           // [rows, G, N], [rows, G, N], [rows, H, P] of the inputs' dtype
    float *ddt;                   // [rows, H]
    float *da, *dd;               // [H]; dd null without skip
    float *dinit;                 // [n_seq, H, N, P] or null
};
cudaError_t launch_ssm_scan(const SsmParams &p, int io_dtype, int out_dtype, cudaStream_t stream);
cudaError_t launch_ssm_step(const SsmParams &p, int io_dtype, int out_dtype, cudaStream_t stream);
// The same by chunks on the tensor cores (ssm_chunk.cu): bf16, N 64 or 128, P a multiple of 64.
bool ssm_chunk_supported(int io_dtype, int N, int P, int rows);
size_t ssm_chunk_workspace_bytes(const SsmParams &p);
cudaError_t launch_ssm_chunk(const SsmParams &p, int out_dtype, cudaStream_t stream);
size_t ssm_bwd_workspace_bytes(int rows, int n_seq, int H, int G, int N, int P);
cudaError_t launch_ssm_bwd(const SsmParams &p, int io_dtype, cudaStream_t stream);
// da, dd [H] from partial sums [n][H], in their order (ssm_scan.cu).
cudaError_t launch_ssm_sums(const float *part_a, const float *part_d, int n, int H, float *da, float *dd, cudaStream_t stream);
// The reverse mode on the tensor cores (ssm_bwd.cu), where ssm_chunk_supported.
size_t ssm_bwd_chunk_workspace_bytes(const SsmParams &p);
cudaError_t launch_ssm_bwd_chunk(const SsmParams &p, cudaStream_t stream);

}  // namespace kla
