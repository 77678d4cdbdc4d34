// Operators on rows of logits that stand on their own (a teacher's top logits,
// the divergence from them with its gradient, penalties, biases and masks):
// what their kernels share, and the host launchers (internal interface).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <type_traits>

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

// ------------------------------------------------------------ 16-byte vectors
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);   // entries per vector

// vector j of a row: an unsigned byte offset from a base that is the same for the
// whole wavefront takes one register, a 64-bit address two
template <typename V> __device__ __forceinline__ V& vec_at(V* base, int j) {
    return *(V*)((const char*)base + (uint32_t)j * 16u);
}

// a vector of -infinity
template <typename T> __device__ __forceinline__ u32x4 masked_vec();
template <> __device__ __forceinline__ u32x4 masked_vec<float>() { return 0xFF800000u; }
template <> __device__ __forceinline__ u32x4 masked_vec<Bf16>() { return 0xFF80FF80u; }
template <> __device__ __forceinline__ u32x4 masked_vec<F16>() { return 0xFC00FC00u; }

// entry i of a vector; i is known at compile time wherever this is called
template <typename T> __device__ __forceinline__ float vec_get(const u32x4& v, int i);
template <> __device__ __forceinline__ float vec_get<float>(const u32x4& v, int i) {
    return __uint_as_float(v[i]);
}
template <> __device__ __forceinline__ float vec_get<Bf16>(const u32x4& v, int i) {
    return __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
}
template <> __device__ __forceinline__ float vec_get<F16>(const u32x4& v, int i) {
    const uint32_t pair = v[i / 2];   // (a bit cast of the element itself reads the vector's first)
    return (float)__builtin_bit_cast(f16x2, pair)[i & 1];
}
// -infinity into entry i where `on`
template <typename T> __device__ __forceinline__ void vec_mask(u32x4& v, int i, bool on) {
    if constexpr (sizeof(T) == 4) {
        v[i] = on ? 0xFF800000u : v[i];
    } else {
        const uint32_t low = masked_vec<T>()[0] & 0xFFFFu;
        v[i / 2] = !on ? v[i / 2] : i & 1 ? (v[i / 2] & 0xFFFFu) | low << 16 : (v[i / 2] & 0xFFFF0000u) | low;
    }
}
// entries rounded to nearest even (the hardware's pair conversions)
template <typename T> __device__ __forceinline__ u32x4 vec_pack(const float (&x)[kVec<T>]) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __float_as_uint(x[i]);
        } else {
            const f32x2 p = {x[2 * i], x[2 * i + 1]};
            if constexpr (std::is_same_v<T, Bf16>)
                v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
            else
                v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2));
        }
    }
    return v;
}

// A row as 16-byte aligned vectors: up to kVec - 1 entries ahead of the first
// one (a row may start at any entry) and as many behind the last, which single
// threads hold ("edge" entries, numbered from 0: those ahead, then those
// behind). Nothing outside the row is accessed, and rows of odd sizes and
// strides move as whole vectors all the same.
struct Span {
    int head, vecs, tail;
    template <typename T> __device__ __forceinline__ static Span of(const T* p, int V) {
        Span s;
        s.head = min(V, (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)));
        s.vecs = (V - s.head) / kVec<T>;
        s.tail = V - s.head - s.vecs * kVec<T>;
        return s;
    }
    __device__ __forceinline__ int edges() const { return head + tail; }
    // the entry of edge e
    __device__ __forceinline__ int edge(int e, int V) const { return e < head ? e : V - tail + (e - head); }
    // Entries in the order of the vectors, the edges behind them.
    __device__ __forceinline__ int place(int v, int V) const {
        return v < head ? V - head - tail + v : v < V - tail ? v - head : v;
    }
};

// ------------------------------------------------------------ reductions
// A wavefront's reduction, the same in every lane: DPP moves within the rows of
// 16 lanes, then two row broadcasts (order fixed; a tenth of the latency of LDS
// exchanges).
template <int Ctrl, int RowMask> __device__ __forceinline__ float dpp_or(float v, float other) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(v), Ctrl,
                                                      RowMask, 0xF, false));
}
template <int Ctrl, int RowMask> __device__ __forceinline__ double dpp_or(double v, double other) {
    const uint2 x = __builtin_bit_cast(uint2, v), o = __builtin_bit_cast(uint2, other);
    return __builtin_bit_cast(
        double, make_uint2(__builtin_amdgcn_update_dpp(o.x, x.x, Ctrl, RowMask, 0xF, false),
                           __builtin_amdgcn_update_dpp(o.y, x.y, Ctrl, RowMask, 0xF, false)));
}
__device__ __forceinline__ float last_lane(float v) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ double last_lane(double v) {
    const uint2 x = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readlane(x.x, 63),
                                                 __builtin_amdgcn_readlane(x.y, 63)));
}
// a value that all lanes have, as one the compiler knows to be the same in all:
// what follows from it is scalar, branches on it among them
__device__ __forceinline__ float uniform(float v) {
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ double uniform(double v) {
    const uint2 x = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readfirstlane(x.x),
                                                 __builtin_amdgcn_readfirstlane(x.y)));
}
struct MaxOp {
    static constexpr float none = -INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct AddOp {
    static constexpr float none = 0.f;
    template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
template <typename V, typename F> __device__ __forceinline__ V wave_all(V v, F op) {
    v = op(v, dpp_or<0x111, 0xF>(v, (V)F::none));   // row_shr 1, 2, 4, 8: lane 15 of a row has its row
    v = op(v, dpp_or<0x112, 0xF>(v, (V)F::none));
    v = op(v, dpp_or<0x114, 0xF>(v, (V)F::none));
    v = op(v, dpp_or<0x118, 0xF>(v, (V)F::none));
    v = op(v, dpp_or<0x142, 0xA>(v, (V)F::none));   // row_bcast 15 and 31: lane 63 has all
    v = op(v, dpp_or<0x143, 0xC>(v, (V)F::none));
    return last_lane(v);
}
// N block-wide reductions with one barrier, for blocks of NT threads. The caller
// puts a barrier before the same `red` is used again.
template <int NT, int N, typename V, typename F>
__device__ __forceinline__ void block_all(V (&v)[N], V (*red)[NT / 64], F op) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_all(v[i], op);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i][threadIdx.x >> 6] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            V r[NT / 64];
#pragma unroll
            for (int w = 0; w < NT / 64; ++w) r[w] = red[i][w];
#pragma unroll
            for (int n = NT / 128; n > 0; n /= 2)
#pragma unroll
                for (int w = 0; w < n; ++w) r[w] = op(r[w], r[w + n]);
            v[i] = uniform(r[0]);
        }
    }
}
template <int NT, typename F> __device__ __forceinline__ float block_all(float v, float* red, F op) {
    float a[1] = {v};
    block_all<NT, 1>(a, (float (*)[NT / 64])red, op);
    return a[0];
}

// Launches over slabs of rows: one launch of all rows could pass the 2^32 work
// items that a launch may have. (Workgroups that loop over rows hold whatever
// the compiler moves out of the loop: 96 registers and spills in place of 81 in
// the divergence of fp32 rows of 16384.) f(first row, grid) with `parts`
// workgroups a row.
template <typename F> inline void by_slabs(int64_t rows, F f, int parts = 1) {
    const int64_t slab = (1 << 21) / parts;
    for (int64_t r0 = 0; r0 < rows; r0 += slab)
        f(r0, dim3((unsigned)((rows - r0 < slab ? rows - r0 : slab) * parts)));
}

// LDS to ask for so that the workgroups of a CU, each of which reads `bytes` and
// writes as much, read no more than the CU's share of the L2 (128 KB) between
// them. With more of them, rows being read and rows being written displace one
// another: divergence of 6144 fp32 rows of 16384, three and two workgroups a CU:
// 164 and 153 us; 18432 bf16 rows, six and four: 237 and 219 (two: 278); 6400
// adjusted fp32 rows, four and two: 168 and 159. (Workgroups of 1024 threads are
// one a CU by their registers, whatever they ask for.)
inline size_t resident_lds(size_t lds, size_t bytes) {
    const size_t groups = std::max<size_t>(2, (128 << 10) / bytes);
    return std::max(lds, std::min<size_t>((160 << 10) / (groups + 1), 62 << 10));
}

// ------------------------------------------------------------ launchers
struct TopArgs {
    int64_t rows;
    int V, K;
    const void* logits;
    int32_t elem;
    int64_t ld;
    double inv_tau;
    float* values;    // [rows][K]
    int32_t* index;   // [rows][K]
    float* rest;      // [rows]
};
// bytes of workspace that a call needs
size_t top_logits_workspace(int64_t rows, int V, int K, int32_t elem);
void top_logits(const TopArgs& a, void* workspace, hipStream_t s);

struct DistillArgs {
    int64_t rows;
    int V, K;
    const void* logits;
    int32_t elem;
    int64_t ld;
    const float* values;    // [rows][K]
    const int32_t* index;   // [rows][K]
    const float* rest;      // [rows] or null
    float inv_tau;
    double inv_tau_d;
    float2 log2_tau;        // log2 e / temperature in two parts
    float alpha, beta;
    const float* weight;    // [rows] or null
    float* loss;            // [rows] or null
    void* grad;             // [rows], stride ld_grad, or null
    int64_t ld_grad;
};
// bytes of workspace that a call needs
size_t distill_top_workspace(int64_t rows, int V, int K, int32_t elem);
void distill_top(const DistillArgs& a, void* workspace, hipStream_t s);

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
