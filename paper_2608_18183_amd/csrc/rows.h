// Operators on rows of logits that stand on their own (a teacher's top logits,
// the divergence from them with its gradient, penalties, biases and masks):
// what their kernels share, and the host launchers (internal interface).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "common.h"
#include "hbsjd.h"

namespace hbsjd {

// sets the calling thread's hbsjd_last_error()
hbsjd_status api_fail(hbsjd_status st, const std::string& msg);

// ------------------------------------------------------------ element types
struct Bf16 { uint16_t u; };
struct F16 { uint16_t u; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return bf16_to_f32(x.u); }
__device__ __forceinline__ float widen(F16 x) { return f16_to_f32(x.u); }
// round to nearest even, NaN stays NaN
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ Bf16 narrow<Bf16>(float x) { return Bf16{f32_to_bf16(x)}; }
template <> __device__ __forceinline__ F16 narrow<F16>(float x) { return F16{f32_to_f16_rne(x)}; }

inline size_t elem_size(int32_t elem) { return elem == HBSJD_ELEM_F32 ? 4 : 2; }

// ------------------------------------------------------------ reductions
// Block-wide reduction for blocks of NT threads in a fixed tree order; `red`
// holds NT / 64 values. The caller puts a barrier before `red` is used again.
template <int NT, typename F>
__device__ __forceinline__ float block_all(float v, float* red, F op) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
    if constexpr (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = op(r, red[w]);
    return r;
}
struct MaxOp { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct AddOp { __device__ float operator()(float a, float b) const { return a + b; } };

// Rows are dealt to at most this many workgroups, which loop over them: a grid
// of a workgroup a row would pass the 2^32 work items that a launch may have.
constexpr int64_t kRowGrid = 1 << 20;
inline dim3 row_grid(int64_t rows) { return dim3((unsigned)(rows < kRowGrid ? rows : kRowGrid)); }

// ------------------------------------------------------------ launchers
struct TopArgs {
    int64_t rows;
    int V, K;
    const void* logits;
    int32_t elem;
    int64_t ld;
    float inv_tau;
    float* values;    // [rows][K]
    int32_t* index;   // [rows][K]
    float* rest;      // [rows]
};
void top_logits(const TopArgs& a, hipStream_t s);

struct DistillArgs {
    int64_t rows;
    int V, K;
    const void* logits;
    int32_t elem;
    int64_t ld;
    const float* values;    // [rows][K]
    const int32_t* index;   // [rows][K]
    const float* rest;      // [rows] or null
    float inv_tau, alpha, beta;
    const float* weight;    // [rows] or null
    float* loss;            // [rows] or null
    void* grad;             // [rows], stride ld_grad, or null
    int64_t ld_grad;
};
void distill_top(const DistillArgs& a, hipStream_t s);

struct AdjustArgs {
    int64_t rows;
    int V;
    const void* logits;
    int32_t elem;
    int64_t ld;
    void* out;
    int32_t out_elem;
    int64_t ld_out;
    const int32_t* tokens;       // [rows] lists of up to n_tokens, or null
    int n_tokens;
    int64_t ld_tokens;
    const int32_t* token_count;  // [rows] or null
    const float *repetition, *presence, *frequency;   // [rows] or null
    const int32_t* bias_index;   // [rows] lists of n_bias, or null
    const float* bias_value;
    int n_bias;
    int64_t ld_bias;
    const uint32_t* mask;        // [n_masks][(V + 31) / 32] or null
    int n_masks;
    const int32_t* mask_row;     // [rows] or null
};
void adjust_rows(const AdjustArgs& a, hipStream_t s);

}  // namespace hbsjd
