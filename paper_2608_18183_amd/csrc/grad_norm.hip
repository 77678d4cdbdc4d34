// The norm of all entries of a list of tensors, and the tensors scaled by it.
//
// The tensors are cut into units of 2048 16-byte vectors, and a fixed number of
// workgroups takes an equal run of units each: many small tensors and a few huge ones
// are the same work. What describes the tensors travels in the kernel's arguments
// (kTable tensors a launch), so that a call keeps nothing and can be captured. Each
// workgroup leaves one number; every workgroup of the scaling adds them up for itself
// in the same order, which saves a launch.
#include "grad_norm.h"

#include <algorithm>

namespace hbsjd {
namespace {

constexpr int NT = 512, NV = 4;
constexpr int kUnit = NT * NV;   // vectors of a unit
constexpr int kTable = 120;      // tensors of a launch: 3.5 of the 4 KB that arguments may take
constexpr int kGroups = 1024;    // workgroups of a call: four a CU

struct Table {
    const void* in[kTable];
    void* out[kTable];
    int64_t n[kTable];
    uint32_t unit[kTable + 1];   // the tensors' first units
    uint8_t elem[kTable];
    int count;
    int groups;
    int first_group;   // of this launch among the call's
};

// A tensor as vectors: entries ahead of the first aligned one and behind the last
// whole vector are single.
struct LongSpan {
    int head, tail;
    int64_t vecs;
};
__host__ __device__ __forceinline__ LongSpan long_span(const void* p, int64_t n, int size) {
    LongSpan s;
    const int64_t head = (int)((16 - ((uintptr_t)p & 15)) & 15) / size;
    s.head = (int)(n < head ? n : head);
    const int e = 16 / size;
    s.vecs = (n - s.head) / e;
    s.tail = (int)(n - s.head - s.vecs * e);
    return s;
}

// what a workgroup's entries come to: a sum of squares, or the bits of the largest
// magnitude (as integers, so that a NaN is the largest)
struct Squares {
    double v;
    __device__ __forceinline__ void add(float x) { v = fma((double)x, (double)x, v); }
    __device__ __forceinline__ void join(const Squares& o) { v += o.v; }
    __device__ __forceinline__ double norm() const { return sqrt(v); }
};
struct Largest {
    uint32_t v;
    __device__ __forceinline__ void add(float x) { v = max(v, __float_as_uint(x) & 0x7FFFFFFFu); }
    __device__ __forceinline__ void join(const Largest& o) { v = max(v, o.v); }
    __device__ __forceinline__ double norm() const { return (double)__uint_as_float(v); }
};

template <typename A> __device__ __forceinline__ A lane_xor(const A& a, int o);
template <> __device__ __forceinline__ Squares lane_xor(const Squares& a, int o) {
    Squares r;
    r.v = __shfl_xor(a.v, o, 64);
    return r;
}
template <> __device__ __forceinline__ Largest lane_xor(const Largest& a, int o) {
    Largest r;
    r.v = __shfl_xor(a.v, o, 64);
    return r;
}
// of the workgroup, the same in every thread
template <typename A> __device__ __forceinline__ A all(A a, A* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a.join(lane_xor(a, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    __syncthreads();
    A r = red[0];
    for (int w = 1; w < NT / 64; ++w) r.join(red[w]);
    return r;
}

template <typename T, typename A>
__device__ __forceinline__ void take_unit(const Table& t, int i, uint32_t u, A& a) {
    const T* p = (const T*)t.in[i];
    const LongSpan sp = long_span(p, t.n[i], sizeof(T));
    const int64_t v0 = (int64_t)u * kUnit;
    const int vecs = (int)min(sp.vecs - v0, (int64_t)kUnit);
    const u32x4* z = (const u32x4*)(p + sp.head) + v0;
    u32x4 x[NV];
    if (vecs > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k) x[k] = vec_at(z, min((int)threadIdx.x + NT * k, vecs - 1));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if ((int)threadIdx.x + NT * k >= vecs) break;
#pragma unroll
        for (int q = 0; q < kVec<T>; ++q) a.add(vec_get<T>(x[k], q));
    }
    if (u == 0 && (int)threadIdx.x < sp.head + sp.tail) {
        const int e = threadIdx.x;
        a.add(widen(p[e < sp.head ? (int64_t)e : t.n[i] - sp.tail + (e - sp.head)]));
    }
}

// the tensor that holds unit u: the last that starts at or before it (empty ones
// start where the next one does)
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t u) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.unit[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t first_unit(const Table& t, int group) {
    return (uint32_t)((uint64_t)t.unit[t.count] * (uint32_t)group / (uint32_t)t.groups);
}

template <typename A> __global__ __launch_bounds__(NT) void k_norm_part(Table t, A* part) {
    __shared__ A red[NT / 64];
    const uint32_t end = first_unit(t, blockIdx.x + 1);
    uint32_t u = first_unit(t, blockIdx.x);
    A a{};
    for (int i = tensor_of(t, u); u < end; ++u) {
        while (u >= t.unit[i + 1]) ++i;
        const uint32_t k = u - t.unit[i];
        if (t.elem[i] == HBSJD_ELEM_F32) take_unit<float>(t, i, k, a);
        else if (t.elem[i] == HBSJD_ELEM_BF16) take_unit<Bf16>(t, i, k, a);
        else take_unit<F16>(t, i, k, a);
    }
    a = all(a, red);
    if (threadIdx.x == 0) part[t.first_group + blockIdx.x] = a;
}

template <typename A> __device__ __forceinline__ double norm_of(const A* part, int groups, A* red) {
    A a{};
    for (int i = threadIdx.x; i < groups; i += NT) a.join(part[i]);
    return all(a, red).norm();
}

template <typename A> __global__ __launch_bounds__(NT) void k_norm_join(const A* part, int groups, float* norm) {
    __shared__ A red[NT / 64];
    const double n = norm_of(part, groups, red);
    if (threadIdx.x == 0) *norm = (float)n;
}

template <typename T> __device__ __forceinline__ void scale_unit(const Table& t, int i, uint32_t u, float f) {
    const T* p = (const T*)t.in[i];
    T* g = (T*)t.out[i];
    const LongSpan sp = long_span(p, t.n[i], sizeof(T));
    const int64_t v0 = (int64_t)u * kUnit;
    const int vecs = (int)min(sp.vecs - v0, (int64_t)kUnit);
    const u32x4* z = (const u32x4*)(p + sp.head) + v0;
    T* gv = g + sp.head + v0 * kVec<T>;
    u32x4 x[NV];
    if (vecs > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k) x[k] = vec_at(z, min((int)threadIdx.x + NT * k, vecs - 1));
    const bool same = (((uintptr_t)g ^ (uintptr_t)p) & 15) == 0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int j = threadIdx.x + NT * k;
        if (j >= vecs) break;
        float y[kVec<T>];
#pragma unroll
        for (int q = 0; q < kVec<T>; ++q) y[q] = vec_get<T>(x[k], q) * f;
        if (same) {
            vec_at((u32x4*)gv, j) = f == 1.f ? x[k] : vec_pack<T>(y);   // a copy keeps NaNs' bits too
        } else {
#pragma unroll
            for (int q = 0; q < kVec<T>; ++q) gv[j * kVec<T> + q] = narrow<T>(y[q]);
        }
    }
    if (u == 0 && (int)threadIdx.x < sp.head + sp.tail) {
        const int e = threadIdx.x;
        const int64_t at = e < sp.head ? (int64_t)e : t.n[i] - sp.tail + (e - sp.head);
        g[at] = narrow<T>(widen(p[at]) * f);
    }
}

// A workgroup's units, the last one first: the norm's pass has left those in the
// last-level cache.
template <typename A>
__global__ __launch_bounds__(NT) void k_scale(Table t, const A* part, int groups, float limit, bool in_place,
                                              float* norm) {
    __shared__ A red[NT / 64];
    const double n = norm_of(part, groups, red);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const bool scaled = n > (double)limit && n < INFINITY;
    if (in_place && !scaled) return;
    const float f = uniform(scaled ? (float)((double)limit / n) : 1.f);
    const uint32_t begin = first_unit(t, blockIdx.x);
    uint32_t u = first_unit(t, blockIdx.x + 1);
    if (u == begin) return;
    int i = tensor_of(t, u - 1);
    while (u-- > begin) {
        while (u < t.unit[i]) --i;
        const uint32_t k = u - t.unit[i];
        if (t.elem[i] == HBSJD_ELEM_F32) scale_unit<float>(t, i, k, f);
        else if (t.elem[i] == HBSJD_ELEM_BF16) scale_unit<Bf16>(t, i, k, f);
        else scale_unit<F16>(t, i, k, f);
    }
}

uint32_t units_of(const void* p, int64_t n, int32_t elem) {
    const LongSpan s = long_span(p, n, (int)elem_size(elem));
    if (n == 0) return 0;
    return (uint32_t)std::max<int64_t>(1, (s.vecs + kUnit - 1) / kUnit);
}

// f(table) for the tensors in order, kTable at a time; false when one of the tables
// holds more units than a launch counts
template <typename F> bool by_tables(const GradArgs& a, uint64_t total, F f) {
    Table t;
    int groups = 0;
    for (int64_t i0 = 0; i0 < a.count; i0 += kTable) {
        t.count = (int)std::min<int64_t>(kTable, a.count - i0);
        uint64_t units = 0;
        for (int i = 0; i < t.count; ++i) {
            t.in[i] = a.data[i0 + i];
            t.out[i] = a.out ? a.out[i0 + i] : nullptr;
            t.n[i] = a.sizes[i0 + i];
            t.elem[i] = (uint8_t)a.elems[i0 + i];
            t.unit[i] = (uint32_t)units;
            units += units_of(t.in[i], t.n[i], t.elem[i]);
            if (units > UINT32_MAX) return false;
        }
        t.unit[t.count] = (uint32_t)units;
        if (units == 0) continue;
        // the call's workgroups by the tables' units
        t.groups = (int)std::min<uint64_t>(units, kGroups * units / total + 1);
        t.first_group = groups;
        groups += t.groups;
        f(t);
    }
    return true;
}

template <typename A> bool go(const GradArgs& a, void* ws, hipStream_t s) {
    A* part = (A*)ws;
    uint64_t total = 0;
    for (int64_t i = 0; i < a.count; ++i) total += units_of(a.data[i], a.sizes[i], a.elems[i]);
    int groups = 0;
    if (!by_tables(a, total, [&](const Table& t) { groups = t.first_group + t.groups; })) return false;
    by_tables(a, total, [&](const Table& t) {
        hipLaunchKernelGGL(k_norm_part<A>, dim3(t.groups), dim3(NT), 0, s, t, part);
    });
    if (!a.out || groups == 0) {
        hipLaunchKernelGGL(k_norm_join<A>, dim3(1), dim3(NT), 0, s, part, groups, a.norm);
        return true;
    }
    float* norm = a.norm;
    bool in_place = true;
    for (int64_t i = 0; i < a.count; ++i) in_place = in_place && a.out[i] == a.data[i];
    by_tables(a, total, [&](const Table& t) {
        hipLaunchKernelGGL(k_scale<A>, dim3(t.groups), dim3(NT), 0, s, t, part, groups, a.limit, in_place,
                           norm);
        norm = nullptr;
    });
    return true;
}

}  // namespace

size_t grad_norm_workspace() {
    return (kGroups + (HBSJD_GRAD_MAX_TENSORS + kTable - 1) / kTable) * sizeof(Squares);
}

bool grad_norm(const GradArgs& a, void* workspace, hipStream_t s) {
    return a.order == 2 ? go<Squares>(a, workspace, s) : go<Largest>(a, workspace, s);
}

}  // namespace hbsjd
