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

#include <algorithm>

namespace hbsjd {
namespace {

constexpr float kNan = __builtin_nanf("");
constexpr float kLn2 = 0.6931471805599453f;

// What a workgroup of NT threads works out about a row once the row's unlisted
// maximum is known; the same for every way the row itself is held.
struct Entries {
    uint32_t* listed;   // a bit per entry, in the order of the row's vectors
    int* entry;         // [K] the listed entries, -1 unused
    float* zk;          // [K] the student's logits there
    float* tk;          // [K] the teacher's
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

// Fetches the answer and marks its entries that lie among the V from `first` on.
// Their logits are gathered here (before anything of the gradient is written: it
// may take the logits' place), or read from `gathered`. mt and mk: the largest t_k
// and z_k that this thread has seen.
template <int NT, typename T>
__device__ __forceinline__ void fetch(const DistillArgs& a, int64_t r, const T* z, const Span& sp,
                                      int first, int V, const Entries& e, int* bad, float* gathered,
                                      bool gather, float& mt, float& mk) {
    const float* tv = a.values + r * a.K;
    const int32_t* ti = a.index + r * a.K;
    for (int k = threadIdx.x; k < a.K; k += NT) {
        int v = ti[k];
        const float x = tv[k];
        if (v < 0 || v >= a.V) {
            if (v != -1) *bad = 1;
            v = -1;
        } else {
            const int at = v - first;
            float y;
            if (at >= 0 && at < V) {
                const int p = sp.place(at, V);
                if (atomicOr(&e.listed[p >> 5], 1u << (p & 31)) >> (p & 31) & 1) *bad = 1;
                if (gather) {
                    y = widen(z[at]);
                    if (gathered) gathered[k] = y;
                }
            }
            if (!gather) y = gathered[k];
            if (!gather || !gathered) {
                e.zk[k] = y;
                mk = fmaxf(mk, y);
                mt = fmaxf(mt, x);
            }
        }
        e.entry[k] = v;
        e.tk[k] = x;
    }
}

// exp of a number held in 64 bits, to a rounding or two of fp32: the hardware's
// exp2 takes 32 bits, the argument's own rounding is put back to first order
__device__ __forceinline__ float exp_of(double x) {
    const double u = x * 1.4426950408889634074;
    const float h = (float)u;
    const float e = __builtin_amdgcn_exp2f(h);
    return h < -200.f ? 0.f : fmaf(e, (float)(u - (double)h) * kLn2, e);
}

struct RowStats {
    float less;     // R, and what the listed entries' c have of D too much
    float loss;
    float factor;   // of e_v in the unlisted gradient
    bool ok;
};

// Everything but the row's own sum: from the maxima (block-wide) and this
// thread's part of s_0. With a = log P and b = log q up to their normalisers'
// logs, an entry's c is b - a - D, D the difference of those logs. A loss far
// below the logs it is made of keeps its digits: a and b are differences in 64
// bits, c is formed with any D_f near D, the sums of P c and q c are held in 64
// bits, and D - D_f, which every entry shares, joins them at the end. One
// wavefront works out the logs in 64 bits; the exponentials are fp32's. The
// largest of either side has the exponent 0 exactly, whatever the temperature: the
// logits are subtracted before they are divided (a quotient's rounding in fp32 is
// larger than exp's range from 1e9 on, and one in 64 bits from 1e18 on).
// Leaves alpha (q - P) + beta q c in zk and beta q in tk for listed_gradient().
template <int NT>
__device__ __forceinline__ RowStats classes(const DistillArgs& a, const Entries& e, float rest, float m0,
                                            float mk, float mt, float s0_part, bool bad,
                                            float (*red)[NT / 64], double (*red2)[NT / 64],
                                            double* shared) {
    const float m = fmaxf(m0, mk);
    auto student = [&](float z) { return ((double)z - (double)m) * a.inv_tau_d; };
    // the teacher's terms relative to the larger of its largest logit and `rest`;
    // an infinite or NaN `rest` that is the larger leaves NaN
    const double top = (double)mt * a.inv_tau_d, from = mt == -INFINITY ? 0.0 : (double)mt;
    const bool listed_top = top >= (double)rest;
    const double shift = listed_top ? 0.0 : from * a.inv_tau_d - (double)rest;
    const double a0 = (double)rest - (listed_top ? top : (double)rest);
    auto teacher = [&](float t) { return ((double)t - from) * a.inv_tau_d + shift; };
    float s[3] = {s0_part, 0.f, 0.f};
    for (int k = threadIdx.x; k < a.K; k += NT) {
        if (e.entry[k] < 0) continue;
        s[1] += exp_of(student(e.zk[k]));
        s[2] += exp_of(teacher(e.tk[k]));
    }
    block_all<NT, 3>(s, red, AddOp());
    const double b0_ref = student(m0);
    const float s0 = s[0], s0m = s0 * exp_of(b0_ref);
    const float rest_e = a.rest ? exp_of(a0) : 0.f;
    const float sz = s0m + s[1], st = s[2] + rest_e;
    const float iz = 1.f / sz, it = 1.f / st;
    const float D_f = __logf(sz) - __logf(st);
    const float q0 = s0m * iz, p0 = rest_e * it;
    const bool reverse = a.beta > 0.f;   // else its sums may be infinite, and count for nothing
    double d[2] = {0.0, 0.0};   // sum P (log P - log q), sum q (log q - log P)
    for (int k = threadIdx.x; k < a.K; k += NT) {
        if (e.entry[k] < 0) continue;
        const double b = student(e.zk[k]), t = teacher(e.tk[k]), c = b - t - (double)D_f;
        const float p = exp_of(t) * it, q = exp_of(b) * iz;
        if (p > 0.f) d[0] -= (double)p * c;
        if (q > 0.f) d[1] += (double)q * c;
        e.zk[k] = a.alpha * (q - p) + (reverse && q > 0.f ? a.beta * q * (float)c : 0.f);
        e.tk[k] = a.beta * q;
    }
    if (threadIdx.x < 64) {
        const double D = log((double)sz / (double)st);
        const double c = a.rest ? b0_ref + log((double)s0) - a0 : 0.0;   // of the others, + D
        if (threadIdx.x == 0) {
            if (a.rest) {
                if (p0 > 0.f) d[0] -= (double)p0 * (c - (double)D_f);
                if (q0 > 0.f) d[1] += (double)q0 * (c - (double)D_f);
            }
            shared[0] = D - (double)D_f;
            shared[1] = c - D;
        }
    }
    block_all<NT, 2>(d, red2, AddOp());
    if (NT == 64) __syncthreads();
    const double late = uniform(shared[0]);
    const float R = reverse ? (float)(d[1] - late) : 0.f;
    RowStats w;
    w.loss = (float)((a.alpha > 0.f ? a.alpha * (d[0] + late) : 0.0) +
                     (reverse ? a.beta * (d[1] - late) : 0.0));
    // no distribution: nothing left, a NaN or an infinity (the sums are then 0 or NaN)
    if (bad || !(sz > 0.f && st > 0.f)) w.loss = kNan;
    w.ok = w.loss > -INFINITY && w.loss < INFINITY;
    float f = a.alpha * (q0 - p0);
    if (reverse && q0 > 0.f) f += a.beta * q0 * ((float)uniform(shared[1]) - R);
    w.factor = s0 > 0.f ? f / s0 : 0.f;
    w.less = R + (float)late;
    return w;
}

// the gradient at the listed entries among the V from `first` on; g: of the first
template <int NT, typename T>
__device__ __forceinline__ void listed_gradient(const DistillArgs& a, const Entries& e,
                                                const RowStats& w, float wt, T* g, int first, int V) {
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const int v = e.entry[k] - first;
        if (e.entry[k] < 0 || v < 0 || v >= V) continue;
        g[v] = narrow<T>(wt * (e.zk[k] - e.tk[k] * w.less));
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

// exp(d / tau): log2 e / tau in two parts, since the rounding of one alone would
// put all entries of the sum off the same way. (Both are positive: d = -infinity
// gives 0.)
__device__ __forceinline__ float power(float d, float2 c2) {
    return __builtin_amdgcn_exp2f(fmaf(d, c2.x, d * c2.y));
}

// ---- a row, or a part of one, in registers: NV 16-byte vectors a thread

template <typename T, int NT, int NV> struct Held {
    static constexpr int E = kVec<T>;
    u32x4 x[NV];
    float xe;   // this thread's edge entry
    Span sp;

    __device__ __forceinline__ void load(const T* z, int V) {
        sp = Span::of(z, V);
        xe = -INFINITY;
        const u32x4* z4 = (const u32x4*)(z + sp.head);
        if (sp.vecs > 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) x[i] = vec_at(z4, min((int)threadIdx.x + NT * i, sp.vecs - 1));
        if ((int)threadIdx.x < sp.edges()) xe = widen(z[sp.edge(threadIdx.x, V)]);
    }
    // Listed entries become -infinity, so that the maximum, the sum and the
    // gradient's factor are of the unlisted ones alone. Returns the largest.
    __device__ __forceinline__ float mask(const uint32_t* listed) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = threadIdx.x + NT * i;
            if (j >= sp.vecs) {
                x[i] = masked_vec<T>();
                continue;
            }
            const uint32_t bits = listed[j * E >> 5] >> (j * E & 31);
#pragma unroll
            for (int q = 0; q < E; ++q) {
                vec_mask<T>(x[i], q, bits >> q & 1);
                m = fmaxf(m, vec_get<T>(x[i], q));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if ((int)threadIdx.x < sp.edges()) {
            const int p = sp.vecs * E + threadIdx.x;
            if (listed[p >> 5] >> (p & 31) & 1) xe = -INFINITY;
        }
        return fmaxf(m, xe);
    }
    // x becomes exp2((x - m0) c2) in fp32 rows (16-bit ones keep the logits, and
    // work the exponentials out again when they are stored: half the registers)
    __device__ __forceinline__ float sum(float m0, float2 c2) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int q = 0; q < E; ++q) {
                const float y = power(vec_get<T>(x[i], q) - m0, c2);
                s += y;
                if constexpr (E == 4) x[i][q] = __float_as_uint(y);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        xe = power(xe - m0, c2);
        return s + xe;
    }
    // f times the exponentials, after sum()
    __device__ __forceinline__ void store(T* g, const T* z, int V, float f, float m0, float2 c2) {
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(x[i]));
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        T* gv = g + sp.head;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = threadIdx.x + NT * i;
            float y[E];
#pragma unroll
            for (int q = 0; q < E; ++q) {
                if constexpr (E == 4) y[q] = f * __uint_as_float(x[i][q]);
                else y[q] = f * __builtin_amdgcn_exp2f((vec_get<T>(x[i], q) - m0) * c2.x);
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
        if ((int)threadIdx.x < sp.edges()) g[sp.edge(threadIdx.x, V)] = narrow<T>(f * xe);
    }
};

constexpr int waves_of(int nt) { return nt == 1024 ? 4 : 5; }

// A workgroup of NT threads per row: logits leave memory once. The gradient at
// the listed entries is stored over the row's afterwards.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT)))) void k_distill(
    DistillArgs a, int64_t r0) {
    extern __shared__ uint32_t lds[];
    __shared__ float red[6][NT / 64];
    __shared__ double red2[2][NT / 64], shared[2];
    __shared__ int bad;
    const int t = threadIdx.x;
    const Entries e = Entries::in(lds, a.V, a.K);
    const float2 c2 = a.log2_tau;
    const int64_t r = r0 + blockIdx.x;
    const T* z = (const T*)a.logits + r * a.ld;
    T* g = a.grad ? (T*)a.grad + r * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (g) fill_row<NT>(g, a.V, 0.f);
        if (a.loss && t == 0) a.loss[r] = 0.f;
        return;
    }
    Held<T, NT, NV> h;
    h.load(z, a.V);
    const float rest = a.rest ? a.rest[r] : -INFINITY;
    for (int i = t; i < (a.V + 31) / 32; i += NT) e.listed[i] = 0;
    if (t == 0) bad = 0;
    __syncthreads();
    float mm[3] = {-INFINITY, -INFINITY, -INFINITY};   // maxima: unlisted, listed, teacher's listed
    fetch<NT>(a, r, z, h.sp, 0, a.V, e, &bad, nullptr, true, mm[2], mm[1]);
    __syncthreads();
    mm[0] = h.mask(e.listed);
    block_all<NT, 3>(mm, red, MaxOp());
    const float m0 = mm[0] == -INFINITY ? fmaxf(mm[1], mm[0]) : mm[0];
    const float s0 = h.sum(m0, c2);
    const RowStats st = classes<NT>(a, e, rest, m0, mm[1], mm[2], s0, uniform(bad) != 0, red + 3, red2, shared);
    if (a.loss && t == 0) a.loss[r] = w * st.loss;
    if (g && !st.ok) fill_row<NT>(g, a.V, kNan);
    if (g && st.ok) {
        const float wt = w * a.inv_tau;
        h.store(g, z, a.V, wt * st.factor, m0, c2);
        __syncthreads();   // the row's stores come first
        listed_gradient<NT>(a, e, st, wt, g, 0, a.V);
    }
}

// Rows too long for a workgroup's registers, or long and few: `parts` workgroups
// a row, in two launches. The first leaves each part's unlisted maximum and sum,
// and the listed entries' logits, in the workspace; the second joins them (every
// part's workgroup works the classes out for itself) and writes the gradient,
// reading the part again. (Rows in slabs that the last-level cache holds make the
// second reading cheaper and the whole slower, by the launches' ends: 2000 bf16
// rows of 200000 in slabs of 192 MB 566 us, of 384 MB 535, at once 515.)
struct PartsArgs {
    int parts, len;
    float* zk;       // [rows of the slab][K]
    float* stats;    // [rows of the slab][parts][3]: maximum, sum, whether refused
};

template <typename T, int NT, int NV, bool Second>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT)))) void k_distill_part(
    DistillArgs a, PartsArgs p, int64_t r0) {
    extern __shared__ uint32_t lds[];
    __shared__ float red[6][NT / 64];
    __shared__ double red2[2][NT / 64], shared[2];
    __shared__ int bad;
    const int t = threadIdx.x;
    const Entries e = Entries::in(lds, p.len, a.K);
    const float2 c2 = a.log2_tau;
    const int row = blockIdx.x / p.parts, c = blockIdx.x - row * p.parts;
    const int64_t r = r0 + row;
    const int first = c * p.len, V = min(p.len, a.V - first);
    const T* z = (const T*)a.logits + r * a.ld + first;
    T* g = a.grad ? (T*)a.grad + r * a.ld_grad + first : nullptr;
    const float w = a.weight ? a.weight[r] : 1.f;
    if (w == 0.f) {
        if (Second && g) fill_row<NT>(g, V, 0.f);
        if (Second && a.loss && c == 0 && t == 0) a.loss[r] = 0.f;
        return;
    }
    Held<T, NT, NV> h;
    // the loss alone takes one workgroup a row, which needs no logits
    if (!Second || g) h.load(z, V);
    else if (c > 0) return;
    else h.sp = Span::of(z, V);
    const float rest = a.rest ? a.rest[r] : -INFINITY;
    float* zk = p.zk + (int64_t)row * a.K;
    float* stats = p.stats + (int64_t)row * p.parts * 3;
    float part_m = -INFINITY, part_s = 0.f, part_bad = 0.f;
    if (Second && (t & 63) < p.parts) {
        part_m = stats[3 * (t & 63)];
        part_s = stats[3 * (t & 63) + 1];
        part_bad = stats[3 * (t & 63) + 2];
    }
    for (int i = t; i < (V + 31) / 32; i += NT) e.listed[i] = 0;
    if (t == 0) bad = 0;
    __syncthreads();
    float mm[3] = {-INFINITY, -INFINITY, -INFINITY};
    fetch<NT>(a, r, z, h.sp, first, V, e, &bad, zk, !Second, mm[2], mm[1]);
    __syncthreads();
    if constexpr (!Second) {
        float m0 = block_all<NT>(h.mask(e.listed), red[0], MaxOp());
        // relative to a finite number: a part without an unlisted mass sums to 0
        const float s = block_all<NT>(h.sum(m0 == -INFINITY ? 0.f : m0, c2), red[1], AddOp());
        if (t == 0) {
            stats[3 * c] = m0;
            stats[3 * c + 1] = s;
            stats[3 * c + 2] = bad;
        }
    } else {
        // every wavefront joins the parts, a lane each
        block_all<NT, 2>(*(float(*)[2])(mm + 1), red, MaxOp());
        float m0 = wave_all(part_m, MaxOp());
        const bool refused = uniform(bad) || wave_all(part_bad, MaxOp()) > 0.f;
        if (m0 == -INFINITY) m0 = mm[1];
        const float s0 =
            wave_all(part_m == -INFINITY ? part_s : part_s * power(part_m - m0, c2), AddOp());
        const RowStats st = classes<NT>(a, e, rest, m0, mm[1], mm[2], t == 0 ? s0 : 0.f, refused, red + 3,
                                        red2, shared);
        if (a.loss && c == 0 && t == 0) a.loss[r] = w * st.loss;
        if (!g) return;
        if (!st.ok) {
            fill_row<NT>(g, V, kNan);
            return;
        }
        const float wt = w * a.inv_tau;
        h.mask(e.listed);
        h.sum(m0, c2);
        h.store(g, z, V, wt * st.factor, m0, c2);
        __syncthreads();
        listed_gradient<NT>(a, e, st, wt, g, first, V);
    }
}

// How a call runs: whole rows, or in parts with workspace for `slab` rows.
struct Plan {
    int parts = 0, len = 0;
    int64_t slab = 0;
};
constexpr int kPart = 16384;   // entries of a part at most

inline size_t part_row_bytes(const Plan& p, int K) { return ((size_t)K + 3 * (size_t)p.parts) * 4; }

// Parts where a workgroup cannot hold the row, and for rows above 128 KB that are
// few: then enough of them for two workgroups a CU, of 4096 entries at least. (64
// fp16 rows of 128257: 24 us in parts, 32 held; 140 bf16 rows of 100000: 33 and 31;
// 200 fp32 rows of 60000: 40 and 27; 900 of them 159 and 116; 140 fp32 rows of
// 20000: 24 and 15.) Rows held by 1024 threads, those above 64 KB, are one
// workgroup a CU (its 16 wavefronts at 82 to 128 registers): one's loads do not
// overlap another's stores, and 900 fp32 rows of 60000 take 1.5 times the bytes' 77.
Plan plan_of(int64_t rows, int V, int K, int32_t elem) {
    Plan p;
    const int64_t size = elem_size(elem);
    const int64_t held = 1024 * 16 * (16 / size);
    if (V * size <= 128 << 10 || (V <= held && rows >= 112)) return p;
    p.parts = (V + kPart - 1) / kPart;
    while (rows * p.parts < 512 && V / (2 * p.parts) >= 4096) p.parts *= 2;   // 64 at most: a lane each
    p.len = ((V + p.parts - 1) / p.parts + 7) / 8 * 8;
    p.parts = (V + p.len - 1) / p.len;
    p.slab = std::max<int64_t>(1, (64 << 20) / (int64_t)part_row_bytes(p, K));
    p.slab = std::min(p.slab, rows);
    return p;
}

template <typename T> void go_parts(const DistillArgs& a, const Plan& plan, void* ws, hipStream_t s) {
    constexpr int NT = 512, NV = kPart / kVec<T> / NT;
    PartsArgs p{plan.parts, plan.len, (float*)ws, (float*)ws + plan.slab * a.K};
    const size_t lds = entries_bytes(p.len, a.K);
    for (int64_t r0 = 0; r0 < a.rows; r0 += plan.slab) {
        const dim3 grid((unsigned)(std::min(plan.slab, a.rows - r0) * p.parts));
        hipLaunchKernelGGL((k_distill_part<T, NT, NV, false>), grid, dim3(NT), lds, s, a, p, r0);
        hipLaunchKernelGGL((k_distill_part<T, NT, NV, true>), grid, dim3(NT), lds, s, a, p, r0);
    }
}

template <typename T> void go(const DistillArgs& a, void* ws, hipStream_t s) {
    const Plan plan = plan_of(a.rows, a.V, a.K, a.elem);
    if (plan.parts) return go_parts<T>(a, plan, ws, s);
    size_t lds = entries_bytes(a.V, a.K);
    if (a.grad) lds = resident_lds(lds, a.V * sizeof(T));
    const int vecs = a.V / kVec<T>;
    auto held = [&](auto nt, auto nv) {
        by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
            hipLaunchKernelGGL((k_distill<T, decltype(nt)::value, decltype(nv)::value>), grid,
                               dim3(decltype(nt)::value), lds, s, a, r0);
        });
    };
    using std::integral_constant;
#define HELD(nt, nv) held(integral_constant<int, nt>{}, integral_constant<int, nv>{})
    if (vecs <= 64 * 2) HELD(64, 2);
    else if (vecs <= 64 * 8) HELD(64, 8);
    else if (vecs <= 256 * 4) HELD(256, 4);
    else if (vecs <= 256 * 8) HELD(256, 8);
    else if (vecs <= 512 * 8) HELD(512, 8);
    else if (vecs <= 1024 * 8) HELD(1024, 8);
    else HELD(1024, 16);
#undef HELD
}

}  // namespace

size_t distill_top_workspace(int64_t rows, int V, int K, int32_t elem) {
    const Plan p = plan_of(rows, V, K, elem);
    return p.parts ? p.slab * part_row_bytes(p, K) : 0;
}

void distill_top(const DistillArgs& a, void* workspace, hipStream_t s) {
    if (a.elem == HBSJD_ELEM_F32) go<float>(a, workspace, s);
    else if (a.elem == HBSJD_ELEM_BF16) go<Bf16>(a, workspace, s);
    else go<F16>(a, workspace, s);
}

}  // namespace hbsjd
