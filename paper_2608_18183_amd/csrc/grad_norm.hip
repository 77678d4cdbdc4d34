// The norm of all entries of a list of tensors, and the tensors scaled by it.
//
// The tensors are cut into units of 64 KB, and a fixed number of workgroups takes every
// so manieth unit each: many small tensors and a few huge ones are the same work, and
// the workgroups sweep through memory side by side. What describes the tensors travels
// in the kernels' arguments (192 tensors a launch, 136 that are copied), so that a call
// keeps nothing and can be captured. Each workgroup leaves one number; every workgroup
// of the scaling adds them up for itself in the same order, which saves a launch.
//
// Memory alone bounds both passes (squares in 64 bits or 32: 45.9 and 45.4 us for the
// 222 MB of the B model). The norm's pass reads the tensors' last kKeep bytes, which the
// second pass may find in the last-level cache (256 MB), as usual, and those before them
// as streams; in long lists the second pass is streams throughout. Clipping 111 M bf16
// entries (222 MB) into others, both passes' kernels: all loads and stores as usual 120
// us, stores alone as streams 104, the second pass's loads too 105, the norm's too 119;
// 757 M fp32 ones 1706, 1664, 1582, 1561, and 1535 with the norm's but for the last
// kKeep. (The second pass from the end on: the same.)
#include "grad_norm.h"

#include <algorithm>

namespace hbsjd {
namespace {

constexpr int NT = 512, NV = 8;
constexpr int kUnit = NT * NV;     // 16-byte vectors of a unit
constexpr int kGroups = 2048;      // workgroups of a launch at most: eight a CU
constexpr int kPartials = 8192;    // and of a call
constexpr uint64_t kKeep = ((uint64_t)192 << 20) / (kUnit * 16);   // units that stay in the last-level cache

// What a launch knows of its tensors, N of them at most: as many as 4 KB of
// arguments hold.
template <int N, bool Out> struct Table {
    static constexpr int kTensors = N;
    static constexpr bool kOut = Out;
    const void* in[N];
    void* out[Out ? N : 1];        // else the tensors themselves
    int64_t n[N];                  // entries, the type in the uppermost bits
    uint32_t unit[N + 1];          // the tensors' first units
    uint32_t stream;               // units below this one move as streams
    int count;
    int groups;
    int first_group;               // of this launch among the call's
    __host__ __device__ int64_t size(int i) const { return n[i] & (((int64_t)1 << 48) - 1); }
    __host__ __device__ int elem(int i) const { return (int)(n[i] >> 48); }
    __device__ void* to(int i) const { return Out ? out[i] : (void*)in[i]; }
};
using Inputs = Table<192, false>;
using Copies = Table<136, true>;

// Lists of up to 64 MB are scaled with usual loads and stores: whatever reads them next
// finds them in the cache (clipping 16 MB and adding the result to others: 27 us, 36 with
// streams; 64 MB 64 either way; 128 MB 165 and 145).
constexpr uint64_t kSmall = ((uint64_t)64 << 20) / (kUnit * 16);

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

// a unit's vectors: NV a thread, those behind the end repeat the last
template <bool Stream>
__device__ __forceinline__ void load_unit(const u32x4* z, int vecs, u32x4 (&x)[NV]) {
    if (vecs > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const u32x4& v = vec_at(z, min((int)threadIdx.x + NT * k, vecs - 1));
            x[k] = Stream ? __builtin_nontemporal_load(&v) : v;
        }
}

template <typename T, typename Tab, typename A>
__device__ __forceinline__ void take_unit(const Tab& t, int i, uint32_t u, A& a) {
    const T* p = (const T*)t.in[i];
    const LongSpan sp = long_span(p, t.size(i), sizeof(T));
    const int64_t v0 = (int64_t)u * kUnit;
    const int vecs = (int)min(sp.vecs - v0, (int64_t)kUnit);
    const u32x4* z = (const u32x4*)(p + sp.head) + v0;
    u32x4 x[NV];
    if (t.unit[i] + u < t.stream) {
        load_unit<true>(z, vecs, x);
        asm volatile("");   // else the compiler makes one of the two, with usual loads
    } else {
        load_unit<false>(z, vecs, x);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if ((int)threadIdx.x + NT * k >= vecs) break;
#pragma unroll
        for (int q = 0; q < kVec<T>; ++q) a.add(vec_get<T>(x[k], q));
    }
    if (u == 0 && (int)threadIdx.x < sp.head + sp.tail) {
        const int e = threadIdx.x;
        a.add(widen(p[e < sp.head ? (int64_t)e : t.size(i) - sp.tail + (e - sp.head)]));
    }
}

// the tensor that holds unit u: the last that starts at or before it (empty ones
// start where the next one does)
template <typename Tab> __device__ __forceinline__ int tensor_of(const Tab& t, uint32_t u) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.unit[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename A> __global__ __launch_bounds__(NT) void k_norm_part(Inputs t, A* part) {
    __shared__ A red[NT / 64];
    const uint32_t end = t.unit[t.count];
    uint32_t u = blockIdx.x;
    A a{};
    for (int i = tensor_of(t, u); u < end; u += t.groups) {
        while (u >= t.unit[i + 1]) ++i;
        const uint32_t k = u - t.unit[i];
        if (t.elem(i) == HBSJD_ELEM_F32) take_unit<float>(t, i, k, a);
        else if (t.elem(i) == HBSJD_ELEM_BF16) take_unit<Bf16>(t, i, k, a);
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

template <typename T, bool Stream, typename Tab>
__device__ __forceinline__ void scale_unit(const Tab& t, int i, uint32_t u, float f) {
    const T* p = (const T*)t.in[i];
    T* g = (T*)t.to(i);
    const LongSpan sp = long_span(p, t.size(i), sizeof(T));
    const int64_t v0 = (int64_t)u * kUnit;
    const int vecs = (int)min(sp.vecs - v0, (int64_t)kUnit);
    const u32x4* z = (const u32x4*)(p + sp.head) + v0;
    T* gv = g + sp.head + v0 * kVec<T>;
    u32x4 x[NV];
    load_unit<Stream>(z, vecs, x);
    const bool same = (((uintptr_t)g ^ (uintptr_t)p) & 15) == 0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int j = threadIdx.x + NT * k;
        if (j >= vecs) break;
        float y[kVec<T>];
#pragma unroll
        for (int q = 0; q < kVec<T>; ++q) y[q] = vec_get<T>(x[k], q) * f;
        if (same) {
            const u32x4 v = f == 1.f ? x[k] : vec_pack<T>(y);   // a copy keeps NaNs' bits too
            u32x4& to = vec_at((u32x4*)gv, j);
            if constexpr (Stream) __builtin_nontemporal_store(v, &to);
            else to = v;
        } else {
#pragma unroll
            for (int q = 0; q < kVec<T>; ++q) gv[j * kVec<T> + q] = narrow<T>(y[q]);
        }
    }
    if (u == 0 && (int)threadIdx.x < sp.head + sp.tail) {
        const int e = threadIdx.x;
        const int64_t at = e < sp.head ? (int64_t)e : t.size(i) - sp.tail + (e - sp.head);
        g[at] = narrow<T>(widen(p[at]) * f);
    }
}

template <typename A, typename Tab>
__global__ __launch_bounds__(NT) void k_scale(Tab t, const A* part, int groups, float limit, float* norm) {
    __shared__ A red[NT / 64];
    const double n = norm_of(part, groups, red);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const bool scaled = n > (double)limit && n < INFINITY;
    if (!Tab::kOut && !scaled) return;
    const float f = uniform(scaled ? (float)((double)limit / n) : 1.f);
    uint32_t u = blockIdx.x;
    const uint32_t end = t.unit[t.count];
    for (int i = tensor_of(t, u); u < end; u += t.groups) {
        while (u >= t.unit[i + 1]) ++i;
        const uint32_t k = u - t.unit[i];
        auto with = [&](auto type) {
            using T = decltype(type);
            if (u < t.stream) {
                scale_unit<T, true>(t, i, k, f);
                asm volatile("");   // (as above)
            } else {
                scale_unit<T, false>(t, i, k, f);
            }
        };
        if (t.elem(i) == HBSJD_ELEM_F32) with(float{});
        else if (t.elem(i) == HBSJD_ELEM_BF16) with(Bf16{});
        else with(F16{});
    }
}

uint32_t units_of(const void* p, int64_t n, int32_t elem) {
    const LongSpan s = long_span(p, n, (int)elem_size(elem));
    if (n == 0) return 0;
    return (uint32_t)std::max<int64_t>(1, (s.vecs + kUnit - 1) / kUnit);
}

// f(table) for the tensors in order, in launches of equal numbers of them
template <typename Tab, typename F> void by_tables(const GradArgs& a, F f) {
    const int64_t launches = (a.count + Tab::kTensors - 1) / Tab::kTensors;
    if (launches == 0) return;
    const int64_t each = (a.count + launches - 1) / launches;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kGroups, kPartials / launches));
    Tab t;
    t.first_group = 0;
    for (int64_t i0 = 0; i0 < a.count; i0 += each) {
        t.count = (int)std::min<int64_t>(each, a.count - i0);
        uint32_t units = 0;
        for (int i = 0; i < t.count; ++i) {
            t.in[i] = a.data[i0 + i];
            if (Tab::kOut) t.out[i] = a.out[i0 + i];
            t.n[i] = a.sizes[i0 + i] | (int64_t)a.elems[i0 + i] << 48;
            t.unit[i] = units;
            units += units_of(t.in[i], a.sizes[i0 + i], a.elems[i0 + i]);
        }
        t.unit[t.count] = units;
        if (units == 0) continue;
        t.groups = (int)std::min<int64_t>(units, most);
        f(t);
        t.first_group += t.groups;
    }
}

template <typename A, typename Tab>
void scale(const GradArgs& a, const A* part, int groups, bool stream, hipStream_t s) {
    float* norm = a.norm;
    by_tables<Tab>(a, [&](Tab& t) {
        t.stream = stream ? UINT32_MAX : 0;
        hipLaunchKernelGGL((k_scale<A, Tab>), dim3(t.groups), dim3(NT), 0, s, t, part, groups, a.limit, norm);
        norm = nullptr;   // the first launch writes it
    });
}

template <typename A> bool go(const GradArgs& a, void* ws, hipStream_t s) {
    A* part = (A*)ws;
    uint64_t units = 0;
    for (int64_t i = 0; i < a.count; ++i) units += units_of(a.data[i], a.sizes[i], a.elems[i]);
    if (units > UINT32_MAX) return false;
    int groups = 0;
    uint64_t done = 0;
    by_tables<Inputs>(a, [&](Inputs& t) {
        // the call's units from here on that are not among its last kKeep
        const uint64_t mine = t.unit[t.count];
        const uint64_t streams = units > done + kKeep ? units - done - kKeep : 0;
        t.stream = (uint32_t)std::min(mine, streams);
        done += mine;
        hipLaunchKernelGGL(k_norm_part<A>, dim3(t.groups), dim3(NT), 0, s, t, part);
        groups = t.first_group + t.groups;
    });
    if (!a.out || groups == 0) {
        hipLaunchKernelGGL(k_norm_join<A>, dim3(1), dim3(NT), 0, s, part, groups, a.norm);
        return true;
    }
    bool in_place = true;
    for (int64_t i = 0; i < a.count; ++i) in_place = in_place && a.out[i] == a.data[i];
    const bool stream = units > kSmall;
    if (in_place) scale<A, Inputs>(a, part, groups, stream, s);
    else scale<A, Copies>(a, part, groups, stream, s);
    return true;
}

}  // namespace

size_t grad_norm_workspace() {
    static_assert(sizeof(Inputs) <= 4000 && sizeof(Copies) <= 4000, "arguments of a launch");
    static_assert((HBSJD_GRAD_MAX_TENSORS + Inputs::kTensors - 1) / Inputs::kTensors <= kPartials, "");
    return kPartials * sizeof(Squares);
}

bool grad_norm(const GradArgs& a, void* workspace, hipStream_t s) {
    return a.order == 2 ? go<Squares>(a, workspace, s) : go<Largest>(a, workspace, s);
}

}  // namespace hbsjd
