// Divergence of a student's rows from a teacher's top logits, and its gradient.
//
// The teacher gives a row's K largest logits t_k at the entries v_k and, in
// full mode, the log mass `rest` that its other entries have at temperature
// tau. P = softmax over [t / tau, rest] (over t / tau alone without `rest`); q
// = softmax(z / tau) of the student, q_0 = sum of q over the unlisted entries.
// With c = log q - log P of an entry's class and R = sum q c = KL(q || P):
//   L        = alpha sum P (log P - log q) + beta R
//   dL/dz_v  = (alpha (q_v - P_v) + beta q_v (c_v - R)) / tau          listed
//            = q_v (alpha (1 - P_0 / q_0) + beta (c_0 - R)) / tau      unlisted
// (without `rest`: alpha q_v / tau unlisted). q_0 is summed over the unlisted
// entries themselves, not taken as one minus the listed mass: a student close
// to a peaked teacher has a q_0 far below the rounding of that difference. With
// m_0 the largest unlisted logit, e_v = exp((z_v - m_0) / tau) and s_0 their
// sum, the unlisted gradient is one factor for the row times e_v.
#include "rows.h"

namespace hbsjd {
namespace {

constexpr float kNan = __builtin_nanf("");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What a workgroup of NT threads works out about a row once the row's unlisted
// maximum is known; the same for every way the row itself is held.
struct Entries {
    uint32_t* listed;   // a bit per entry, in the order of the row's vectors
    int* entry;         // [K] the listed entries, -1 unused
    float* zk;          // [K] the student's logits there
    float* tk;          // [K] the teacher's / tau
    __device__ __forceinline__ static Entries in(void* lds, int V, int K) {
        Entries e;
        e.listed = (uint32_t*)lds;
        e.entry = (int*)(e.listed + (V + 31) / 32);
        e.zk = (float*)(e.entry + K);
        e.tk = e.zk + K;
        return e;
    }
};
inline size_t entries_bytes(int V, int K) { return ((size_t)(V + 31) / 32 + 3 * (size_t)K) * 4; }

// fetches the answer, marks its entries and gathers the student's logits there
// (before anything of the gradient is written: it may take the logits' place);
// returns the largest t_k / tau and z_k seen by this thread
template <int NT, typename T>
__device__ __forceinline__ void fetch(const DistillArgs& a, int64_t r, const T* z, const Span& sp,
                                      const Entries& e, int* bad, float& mt, float& mk) {
    const float* tv = a.values + r * a.K;
    const int32_t* ti = a.index + r * a.K;
    for (int k = threadIdx.x; k < a.K; k += NT) {
        int v = ti[k];
        const float x = tv[k] * a.inv_tau;
        if (v < 0 || v >= a.V) {
            if (v != -1) *bad = 1;
            v = -1;
        } else {
            const int p = sp.place(v, a.V);
            if (atomicOr(&e.listed[p >> 5], 1u << (p & 31)) >> (p & 31) & 1) *bad = 1;
            const float y = widen(z[v]);
            e.zk[k] = y;
            mk = fmaxf(mk, y);
            mt = fmaxf(mt, x);
        }
        e.entry[k] = v;
        e.tk[k] = x;
    }
}

struct RowStats {
    float m, lz, lt, rsum, loss, factor;   // factor: of e_v in the unlisted gradient
    bool ok;
};

// everything but the row's own sum: from the maxima (block-wide) and this
// thread's part of s_0
template <int NT>
__device__ __forceinline__ RowStats classes(const DistillArgs& a, const Entries& e, float rest, float m0,
                                            float mk, float mt, float s0_part, bool bad,
                                            float (*red)[NT / 64], float (*red2)[NT / 64]) {
    RowStats w;
    w.m = fmaxf(m0, mk);
    float s[3] = {s0_part, 0.f, 0.f};
    for (int k = threadIdx.x; k < a.K; k += NT) {
        if (e.entry[k] < 0) continue;
        s[1] += __expf((e.zk[k] - w.m) * a.inv_tau);
        s[2] += __expf(e.tk[k] - mt);
    }
    block_all<NT, 3>(s, red, AddOp());
    const float s0 = s[0], st = a.rest ? s[2] + __expf(rest - mt) : s[2];
    const float sz = s0 * __expf((m0 - w.m) * a.inv_tau) + s[1];
    // no distribution: nothing left, a NaN or an infinity (the sums are then 0 or NaN)
    const bool some = sz > 0.f && st > 0.f;
    w.lz = __logf(sz);
    w.lt = mt + __logf(st);
    float d[2] = {0.f, 0.f};   // sum P (log P - log q), sum q (log q - log P)
    for (int k = threadIdx.x; k < a.K; k += NT) {
        if (e.entry[k] < 0) continue;
        const float lp = e.tk[k] - w.lt, lq = (e.zk[k] - w.m) * a.inv_tau - w.lz;
        const float p = __expf(lp), q = __expf(lq), c = lq - lp;
        if (p > 0.f) d[0] -= p * c;
        if (q > 0.f) d[1] += q * c;
    }
    block_all<NT, 2>(d, red2, AddOp());
    const float lq0 = (m0 - w.m) * a.inv_tau + __logf(s0) - w.lz, q0 = __expf(lq0);
    float f = a.alpha * q0;
    if (a.rest) {
        const float lp = rest - w.lt, p = __expf(lp), c = lq0 - lp;
        if (p > 0.f) d[0] -= p * c;
        if (q0 > 0.f) d[1] += q0 * c;
        f -= a.alpha * p;
        if (a.beta > 0.f && q0 > 0.f) f += a.beta * q0 * (c - d[1]);
    }
    w.factor = s0 > 0.f ? f / s0 : 0.f;
    w.rsum = d[1];
    w.loss = a.alpha > 0.f ? a.alpha * d[0] : 0.f;
    if (a.beta > 0.f) w.loss += a.beta * d[1];
    if (bad || !some) w.loss = kNan;
    w.ok = w.loss > -INFINITY && w.loss < INFINITY;
    return w;
}

// the gradient at the listed entries
template <int NT, typename T>
__device__ __forceinline__ void listed_gradient(const DistillArgs& a, const Entries& e,
                                                const RowStats& w, float wt, T* g) {
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const int v = e.entry[k];
        if (v < 0) continue;
        const float lp = e.tk[k] - w.lt, lq = (e.zk[k] - w.m) * a.inv_tau - w.lz;
        const float p = __expf(lp), q = __expf(lq);
        float d = a.alpha * (q - p);
        if (a.beta > 0.f && q > 0.f) d += a.beta * q * (lq - lp - w.rsum);
        g[v] = narrow<T>(wt * d);
    }
}

// a gradient row of one value
template <int NT, typename T>
__device__ __forceinline__ void fill_row(T* g, int V, float x) {
    const Span sp = Span::of(g, V);
    float xs[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) xs[i] = x;
    const u32x4 raw = vec_pack<T>(xs);
    u32x4* g4 = (u32x4*)(g + sp.head);
    for (int j = threadIdx.x; j < sp.vecs; j += NT) g4[j] = raw;
    if ((int)threadIdx.x < sp.edges()) g[sp.edge(threadIdx.x, V)] = narrow<T>(x);
}

// A workgroup of NT threads per row, the row in registers, NV 16-byte vectors a
// thread: logits leave memory once. Listed entries become -infinity in the
// registers, so that the maximum, the sum and the gradient's factor are of the
// unlisted ones alone; their own gradient is stored over the row's afterwards.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(NV * 4 > 32 ? 4 : 5))) void k_distill(
    DistillArgs a, int64_t r0) {
    constexpr int E = kVec<T>;
    extern __shared__ uint32_t lds[];
    __shared__ float red[8][NT / 64];
    __shared__ int bad;
    const int t = threadIdx.x;
    const Entries e = Entries::in(lds, a.V, a.K);
    const float c2 = a.inv_tau * kLog2e;
    const int64_t r = r0 + blockIdx.x;
    const T* z = (const T*)a.logits + r * a.ld;
    T* g = a.grad ? (T*)a.grad + r * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (g) fill_row<NT>(g, a.V, 0.f);
        if (a.loss && t == 0) a.loss[r] = 0.f;
        return;
    }
    const Span sp = Span::of(z, a.V);
    u32x4 x[NV];
    float xe = -INFINITY;
    const u32x4* z4 = (const u32x4*)(z + sp.head);
    if (sp.vecs > 0)
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = vec_at(z4, min(t + NT * i, sp.vecs - 1));
    if (t < sp.edges()) xe = widen(z[sp.edge(t, a.V)]);
    const float rest = a.rest ? a.rest[r] : -INFINITY;
    for (int i = t; i < (a.V + 31) / 32; i += NT) e.listed[i] = 0;
    if (t == 0) bad = 0;
    __syncthreads();
    float mm[3] = {-INFINITY, -INFINITY, rest};   // maxima: unlisted, listed, teacher
    fetch<NT>(a, r, z, sp, e, &bad, mm[2], mm[1]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t + NT * i;
        if (j >= sp.vecs) {
            x[i] = masked_vec<T>();
            continue;
        }
        const uint32_t bits = e.listed[j * E >> 5] >> (j * E & 31);
#pragma unroll
        for (int q = 0; q < E; ++q) {
            vec_mask<T>(x[i], q, bits >> q & 1);
            mm[0] = fmaxf(mm[0], vec_get<T>(x[i], q));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (t < sp.edges()) {
        const int p = sp.vecs * E + t;
        if (e.listed[p >> 5] >> (p & 31) & 1) xe = -INFINITY;
    }
    mm[0] = fmaxf(mm[0], xe);
    block_all<NT, 3>(mm, red, MaxOp());
    const float m0 = mm[0] == -INFINITY ? fmaxf(mm[1], mm[0]) : mm[0];
    // fp32 rows: the exponentials take the logits' registers
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            const float y = __builtin_amdgcn_exp2f((vec_get<T>(x[i], q) - m0) * c2);
            s += y;
            if constexpr (E == 4) x[i][q] = __float_as_uint(y);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    const float ye = __builtin_amdgcn_exp2f((xe - m0) * c2);
    s += ye;
    const RowStats st = classes<NT>(a, e, rest, m0, mm[1], mm[2], s, bad != 0, red + 3, red + 6);
    if (a.loss && t == 0) a.loss[r] = w * st.loss;
    if (g && !st.ok) fill_row<NT>(g, a.V, kNan);
    if (g && st.ok) {
        // (16-bit rows: the exponentials are worked out again, rather than
        // kept in twice the registers)
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(x[i]));
        const float wt = w * a.inv_tau, f = wt * st.factor;
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        T* gv = g + sp.head;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = t + NT * i;
            float y[E];
#pragma unroll
            for (int q = 0; q < E; ++q) {
                if constexpr (E == 4) y[q] = f * __uint_as_float(x[i][q]);
                else y[q] = f * __builtin_amdgcn_exp2f((vec_get<T>(x[i], q) - m0) * c2);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (j >= sp.vecs) continue;
            if (same) {
                vec_at((u32x4*)gv, j) = vec_pack<T>(y);
            } else {
#pragma unroll
                for (int q = 0; q < E; ++q) gv[j * E + q] = narrow<T>(y[q]);
            }
        }
        if (t < sp.edges()) g[sp.edge(t, a.V)] = narrow<T>(f * ye);
        __syncthreads();   // the row's stores are done
        listed_gradient<NT>(a, e, st, wt, g);
    }
}

// Rows too long for the registers: three passes over them in memory.
template <typename T>
__global__ __launch_bounds__(1024) void k_distill_long(DistillArgs a, int64_t r0) {
    constexpr int NT = 1024;
    extern __shared__ uint32_t lds[];
    __shared__ float red[8][NT / 64];
    __shared__ int bad;
    const int t = threadIdx.x;
    const Entries e = Entries::in(lds, a.V, a.K);
    const int64_t r = r0 + blockIdx.x;
    const T* z = (const T*)a.logits + r * a.ld;
    T* g = a.grad ? (T*)a.grad + r * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (g) fill_row<NT>(g, a.V, 0.f);
        if (a.loss && t == 0) a.loss[r] = 0.f;
        return;
    }
    const Span sp{0, a.V, 0};
    const float rest = a.rest ? a.rest[r] : -INFINITY;
    for (int i = t; i < (a.V + 31) / 32; i += NT) e.listed[i] = 0;
    if (t == 0) bad = 0;
    __syncthreads();
    float mm[3] = {-INFINITY, -INFINITY, rest};
    fetch<NT>(a, r, z, sp, e, &bad, mm[2], mm[1]);
    __syncthreads();
    auto unlisted = [&](int v) { return !(e.listed[v >> 5] >> (v & 31) & 1); };
    for (int v = t; v < a.V; v += NT)
        if (unlisted(v)) mm[0] = fmaxf(mm[0], widen(z[v]));
    block_all<NT, 3>(mm, red, MaxOp());
    const float m0 = mm[0] == -INFINITY ? fmaxf(mm[1], mm[0]) : mm[0];
    float s = 0.f;
    for (int v = t; v < a.V; v += NT)
        if (unlisted(v)) s += __expf((widen(z[v]) - m0) * a.inv_tau);
    const RowStats st = classes<NT>(a, e, rest, m0, mm[1], mm[2], s, bad != 0, red + 3, red + 6);
    if (a.loss && t == 0) a.loss[r] = w * st.loss;
    if (g && !st.ok) fill_row<NT>(g, a.V, kNan);
    if (g && st.ok) {
        const float wt = w * a.inv_tau, f = wt * st.factor;
        for (int v = t; v < a.V; v += NT)
            if (unlisted(v)) g[v] = narrow<T>(f * __expf((widen(z[v]) - m0) * a.inv_tau));
        listed_gradient<NT>(a, e, st, wt, g);
    }
}

template <typename T> void go(const DistillArgs& a, hipStream_t s) {
    const size_t lds = entries_bytes(a.V, a.K);
    const int vecs = a.V / kVec<T>;
    auto held = [&](auto nt, auto nv) {
        by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
            hipLaunchKernelGGL((k_distill<T, decltype(nt)::value, decltype(nv)::value>), grid,
                               dim3(decltype(nt)::value), lds, s, a, r0);
        });
    };
    using std::integral_constant;
#define HOLD(nt, nv) held(integral_constant<int, nt>{}, integral_constant<int, nv>{})
    if (vecs <= 64 * 2) HOLD(64, 2);
    else if (vecs <= 64 * 8) HOLD(64, 8);
    else if (vecs <= 256 * 4) HOLD(256, 4);
    else if (vecs <= 256 * 8) HOLD(256, 8);
    else if (vecs <= 512 * 8) HOLD(512, 8);
    else if (vecs <= 1024 * 8) HOLD(1024, 8);
    else if (vecs <= 1024 * 16) HOLD(1024, 16);
    else
        by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
            hipLaunchKernelGGL(k_distill_long<T>, grid, dim3(1024), lds, s, a, r0);
        });
#undef HOLD
}

}  // namespace

void distill_top(const DistillArgs& a, hipStream_t s) {
    if (a.elem == HBSJD_ELEM_F32) go<float>(a, s);
    else if (a.elem == HBSJD_ELEM_BF16) go<Bf16>(a, s);
    else go<F16>(a, s);
}

}  // namespace hbsjd
