// Log-probabilities of rows' tokens, the losses made of them, and their gradients
// by the logits.
//
// With p = softmax(z / tau) of a row, y its token, l = log p_y and H = -sum p log p:
//   dl/dz_v = (1[v = y] - p_v) / tau,   dH/dz_v = -p_v (log p_v + H) / tau.
// All losses here reach the logits through the two slopes g = dL/dl and h = dL/dH.
// An entry's exponential is e_v = 2^x_v, x_v = z_v c - k with c = log2 e / tau and k
// next to the largest z c: one fused operation ahead of the hardware's exp2. k is a
// rounded number, and what it is off by is put back in 64 bits. With s = sum e and
// X = sum e x / s, log p_v = x_v ln 2 - log s, H = log s - X ln 2, and the gradient is
//   e_v (A_0 + A_1 x_v),   A_0 = -(g - h X ln 2) / (tau s),   A_1 = -h ln 2 / (tau s)
// away from the token, and at it
//   (g s_o / s - h p_y (l + H)) / tau,
// s_o the sum over all entries but the token's. That sum is formed by itself: for a
// token that is nearly certain, 1 - p_y = s_o / s and l = -log(1 + s_o / e_y) would
// be differences of almost equal numbers.
//
// A row is read once and stays in its workgroup's registers until its gradient is
// stored; long rows go in parts, pairs of sequences in two readings with the pair's
// loss between them.
#include "rows.h"

#include <algorithm>

namespace hbsjd {
namespace {

// exponents (to base 2) below this give an e_v of 0 in any case
constexpr float kFar = -200.f;

// How a row's exponents are formed: as above, or (logits so large, or a temperature so
// small, that z c has no digits left behind the binary point, and rows without a largest
// logit) with the entries replaced by z - m first, and k = 0. Of two entries of such a
// row whose exponents differ by less than 200, z - m is exact in fp32; in 16 bits there
// are none but equal ones.
struct Exponents {
    float c, k;
    double off;   // what k falls short of m c by, in nats: exponents are that much too large
    bool near;

    __device__ __forceinline__ static Exponents of(float m, float2 c2) {
        Exponents x;
        // One fp32 number: a second part would be an operation more an entry. Its rounding
        // puts x of an entry y nats below the largest off by y 2^-24, as the rounding of x
        // itself may, but all entries the same way: log s by up to 2^-24 times the mean of
        // y under p, 2e-7 where that is 4.
        x.c = c2.x + c2.y;
        x.k = m * x.c;
        x.near = fabsf(x.k) < 1048576.f;
        x.off = fma((double)m, (double)x.c, -(double)x.k) * 0.6931471805599453094;
        if (!x.near) {
            x.k = 0.f;
            x.off = 0.0;
        }
        return x;
    }
    __device__ __forceinline__ float at(float z) const { return fmaf(z, c, -k); }
};

// What the entries of a row or a part come to.
struct Sums {
    double s = 0.0, t = 0.0;   // sums of e and e x, without the token's entry
};

// the largest entry of a vector, and m; a NaN counts for nothing, or for all there was
// (the sum is none then)
template <typename T> struct Largest {
    float m = -INFINITY;
    __device__ __forceinline__ void add(const u32x4& v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) m = fmaxf(m, __uint_as_float(v[q]));
    }
    __device__ __forceinline__ float get() const { return m; }
};
// as pairs. The upper entry without the lower one's digits, which would make a masked
// entry's -infinity a signalling NaN: the hardware's maximum of that and all before it is a
// NaN, and the next one leaves it out. (The integers' packed maximum and minimum, two
// operations a pair for four, take 5% more in readings of long rows.)
template <> struct Largest<Bf16> {
    float lo = -INFINITY, hi = -INFINITY;
    __device__ __forceinline__ void add(const u32x4& v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lo = fmaxf(lo, __uint_as_float(v[q] << 16));
            hi = fmaxf(hi, __uint_as_float(v[q] & 0xFFFF0000u));
        }
    }
    __device__ __forceinline__ float get() const { return fmaxf(lo, hi); }
};
template <> struct Largest<F16> {
    f16x2 m = {(_Float16)-INFINITY, (_Float16)-INFINITY};
    __device__ __forceinline__ void add(const u32x4& v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t pair = v[q];
            m = __builtin_elementwise_max(m, __builtin_bit_cast(f16x2, pair));
        }
    }
    __device__ __forceinline__ float get() const { return fmaxf((float)m[0], (float)m[1]); }
};

template <typename T, int NT, int NV> struct TokenRow : RowRegs<T, NT, NV> {
    using RowRegs<T, NT, NV>::E;
    using RowRegs<T, NT, NV>::x;
    using RowRegs<T, NT, NV>::xe;
    using RowRegs<T, NT, NV>::sp;
    int jy, qy, ey;   // the token's vector and place in it, or its edge; -1: elsewhere

    // stream: the row is not looked for in the caches again
    __device__ __forceinline__ void load(const T* z, int V, bool stream) {
        if (!stream) return RowRegs<T, NT, NV>::load(z, V);
        sp = Span::of(z, V);
        xe = -INFINITY;
        const u32x4* z4 = (const u32x4*)(z + sp.head);
        if (sp.vecs > 0)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                x[i] = __builtin_nontemporal_load(&vec_at(z4, min((int)threadIdx.x + NT * i, sp.vecs - 1)));
        if ((int)threadIdx.x < sp.edges()) xe = widen(z[sp.edge(threadIdx.x, V)]);
        asm volatile("");   // else the compiler makes one of the two, with usual loads
    }
    // y: the token's entry relative to this row or part
    __device__ __forceinline__ void find(int y, int V) {
        jy = ey = -1;
        qy = 0;
        if (y < 0 || y >= V) return;
        const int p = sp.place(y, V);
        if (p >= sp.vecs * E) {
            ey = p - sp.vecs * E;
        } else {
            jy = p / E;
            qy = p % E;
        }
    }
    // z - m in place of z
    __device__ __forceinline__ void recenter(float m) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float y[E];
#pragma unroll
            for (int q = 0; q < E; ++q) y[q] = vec_get<T>(x[i], q) - m;
            x[i] = vec_pack<T>(y);
            asm volatile("" : "+v"(x[i]));   // (as below)
            __builtin_amdgcn_sched_barrier(0);
        }
        xe -= m;
    }
    // else the compiler keeps entries that a pass has unpacked for the next one
    __device__ __forceinline__ void keep_packed() {
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(x[i]));
    }
    // The token's entry and what lies behind the row become -infinity. Returns the
    // largest of the rest.
    __device__ __forceinline__ float largest() {
        Largest<T> m;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = threadIdx.x + NT * i;
            if (j >= sp.vecs) {
                x[i] = masked_vec<T>();
            } else if (j == jy) {
#pragma unroll
                for (int q = 0; q < E; ++q) vec_mask<T>(x[i], q, q == qy);
            }
            m.add(x[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if ((int)threadIdx.x == ey) xe = -INFINITY;
        keep_packed();
        return fmaxf(m.get(), xe);
    }
    template <bool Ent>
    __device__ __forceinline__ void add(float z, const Exponents& ex, float& s, float& t) const {
        const float y = ex.at(z), e = __builtin_amdgcn_exp2f(y);
        s += e;
        if constexpr (Ent) t = fmaf(e, fmaxf(y, kFar), t);
    }
    // this thread's part of the sums
    template <bool Ent> __device__ __forceinline__ Sums sum(const Exponents& ex) {
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float sv = 0.f, tv = 0.f;   // a vector's own sums: shorter chains of roundings
#pragma unroll
            for (int q = 0; q < E; ++q) {
                add<Ent>(vec_get<T>(x[i], q), ex, sv, tv);
                // else the compiler unpacks bf16 vectors ahead, and spills
                if constexpr (Ent) asm volatile("" : "+v"(sv), "+v"(tv));
            }
            s += sv;
            t += tv;
            __builtin_amdgcn_sched_barrier(0);
        }
        add<Ent>(xe, ex, s, t);
        return Sums{(double)s, (double)t};
    }
    template <bool Ent>
    __device__ __forceinline__ static float value(float z, const Exponents& ex, float a0, float a1) {
        const float y = ex.at(z), e = __builtin_amdgcn_exp2f(y);
        return Ent ? e * fmaf(a1, fmaxf(y, kFar), a0) : e * a0;
    }
    // the gradient; gy: at the token
    template <bool Ent>
    __device__ __forceinline__ void store(T* g, const T* z, int V, bool stream, const Exponents& ex, float a0,
                                          float a1, float gy) {
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        T* gv = g + sp.head;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = threadIdx.x + NT * i;
            float y[E];
#pragma unroll
            for (int q = 0; q < E; ++q) y[q] = value<Ent>(vec_get<T>(x[i], q), ex, a0, a1);
            if (j == jy)
#pragma unroll
                for (int q = 0; q < E; ++q) y[q] = q == qy ? gy : y[q];
            __builtin_amdgcn_sched_barrier(0);
            if (j >= sp.vecs) continue;
            if (same) {
                if (stream) {
                    asm volatile("");   // (as above)
                    __builtin_nontemporal_store(vec_pack<T>(y), &vec_at((u32x4*)gv, j));
                    asm volatile("");
                } else {
                    vec_at((u32x4*)gv, j) = vec_pack<T>(y);
                }
            } else {
#pragma unroll
                for (int q = 0; q < E; ++q) gv[j * E + q] = narrow<T>(y[q]);
            }
        }
        if ((int)threadIdx.x < sp.edges()) {
            const float ye = value<Ent>(xe, ex, a0, a1);
            g[sp.edge(threadIdx.x, V)] = narrow<T>((int)threadIdx.x == ey ? gy : ye);
        }
    }
};

// ---- a row's results from its sums

constexpr double kLn2d = 0.6931471805599453094;

struct RowEnd {
    double l, entropy;
    double s, se, ey;   // sums of e: the row's, without the token, the token's
    double mean, over;  // the mean of all exponents in nats, and what the token's is above it
};

// a condition; One: every lane of the wavefront has the same
template <bool One> __device__ __forceinline__ bool holds(bool x) {
    if constexpr (One) return uniform((int)x) != 0;
    return x;
}

// m: the largest logit, zy: the token's, o: the sums with the exponents ex. One: the
// wavefront works on one row, else every lane on its own
template <bool One>
__device__ __forceinline__ RowEnd row_end(float m, float zy, Sums o, double off, double inv_tau) {
    RowEnd r;
    const double x = ((double)zy - (double)m) * inv_tau;
    const double xy = x + off;
    r.ey = exp_of(xy);
    r.se = o.s;
    r.s = o.s + r.ey;
    // a token that has most of the mass is the largest entry: x is 0
    const bool most = holds<One>(r.ey >= o.s);
    double up;
    if (most) up = log1p(o.s / r.ey);
    else up = log(r.s);
    r.l = most ? -up : xy - up;
    const double per = 1.0 / r.s;
    r.mean = (o.t * kLn2d + (r.ey > 0.0 ? r.ey * xy : 0.0)) * per;
    // xy - mean, which for a token that is nearly certain are almost equal
    r.over = r.ey > 0.0 ? (xy * o.s - o.t * kLn2d) * per : 0.0;
    r.entropy = most ? up + r.over : up - r.mean;
    // no distribution: nothing left, a NaN or an infinity (the sums are then 0 or none)
    if (!(r.s > 0.0 && r.s < INFINITY)) r.l = r.entropy = (double)kNan;
    return r;
}

struct Goal {
    double loss, g, h;
};

// The loss of row r and its slopes by l and H, w the row's weight.
__device__ __forceinline__ Goal goal_of(const TokenArgs& a, int64_t r, double l, double entropy, float w) {
    Goal o{0.0, 0.0, 0.0};
    if (!a.advantage) {
        if (a.logprob_weight) o.g = a.logprob_weight[r];
        if (a.entropy_weight) o.h = a.entropy_weight[r];
        o.loss = l;   // whose being no number the gradient shows
        return o;
    }
    const double adv = a.advantage[r];
    double rho = l == l ? 1.0 : l;
    if (a.old_logprob) rho = exp(l - (double)a.old_logprob[r]);
    const double bound = adv > 0.0 ? a.high : a.low;
    const bool beyond = adv > 0.0 ? rho > bound : rho < bound;
    if (adv != 0.0) {   // (a NaN is taken along)
        o.loss = -adv * (beyond ? bound : rho);
        o.g = beyond ? 0.0 : -adv * rho;
    } else if (rho != rho) {
        o.loss = rho;
    }
    if (a.kl > 0.f && a.ref_logprob) {
        const double d = (double)a.ref_logprob[r] - l, e = expm1(d);
        o.loss += a.kl * (e < INFINITY ? e - d : e);
        o.g -= a.kl * e;
    }
    if (a.bonus > 0.f) {
        o.loss -= a.bonus * entropy;
        o.h = -a.bonus;
    }
    o.loss *= w;
    o.g *= w;
    o.h *= w;
    return o;
}

// what the stores need
struct Slopes {
    float a0, a1, gy;
    bool ok;
};
__device__ __forceinline__ Slopes slopes_of(const RowEnd& e, const Goal& o, double inv_tau) {
    const double f = inv_tau / e.s;
    Slopes s;
    s.a0 = (float)(-f * (o.g - o.h * e.mean));
    s.a1 = (float)(-f * o.h * kLn2d);
    s.gy = (float)(f * (o.g * e.se - o.h * e.ey * e.over));
    return s;
}

// a row that takes no part
template <int NT, typename T>
__device__ __forceinline__ void no_part(const TokenArgs& a, int64_t r, T* g, int V, bool first) {
    if (g) fill_row<NT>(g, V, 0.f);
    if (first && threadIdx.x == 0) {
        if (a.loss) a.loss[r] = 0.f;
        if (a.logprob) a.logprob[r] = 0.f;
        if (a.entropy) a.entropy[r] = 0.f;
    }
}
template <int NT, typename T>
__device__ __forceinline__ void no_number(const TokenArgs& a, int64_t r, T* g, int V, bool first) {
    if (g) fill_row<NT>(g, V, kNan);
    if (first && threadIdx.x == 0) {
        if (a.loss) a.loss[r] = kNan;
        if (a.logprob) a.logprob[r] = kNan;
        if (a.entropy) a.entropy[r] = kNan;
    }
}

// One wavefront works a row out in 64 bits and leaves the slopes in `shared`
// (every wavefront doing so would take as long as the exponentials).
__device__ __forceinline__ void finish(const TokenArgs& a, int64_t r, float m, float zy, Sums o, double off,
                                       float w, bool first, Slopes* shared) {
    // one after the other: the row's registers leave little room
    const RowEnd e = row_end<true>(m, zy, o, off, a.inv_tau);
    __builtin_amdgcn_sched_barrier(0);
    const Goal goal = goal_of(a, r, e.l, e.entropy, w);
    __builtin_amdgcn_sched_barrier(0);
    Slopes s = slopes_of(e, goal, a.inv_tau);
    // a loss without an end leaves no gradient; a log-probability of -infinity does
    const float loss = (float)goal.loss;
    s.ok = a.advantage ? loss > -INFINITY && loss < INFINITY : loss == loss;
    if (threadIdx.x == 0) {
        *shared = s;
        if (first) {
            if (a.loss) a.loss[r] = loss;
            if (a.logprob) a.logprob[r] = (float)e.l;
            if (a.entropy) a.entropy[r] = (float)e.entropy;
        }
    }
}

// A workgroup of NT threads a row. (With a gradient four wavefronts a SIMD are what the
// rows in flight leave, see resident_lds().)
template <typename T, int NT, int NV, bool Ent, bool Grad>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(Grad ? 4 : waves_of(NT)))) void k_token(
    TokenArgs a, int64_t r0) {
    __shared__ float red[NT / 64];
    __shared__ double red2[2][NT / 64];
    __shared__ Slopes shared;
    const int64_t r = r0 + blockIdx.x;
    const T* z = (const T*)a.logits + r * a.ld;
    T* g = Grad ? (T*)a.grad + r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y == -1 || w == 0.f) return no_part<NT>(a, r, g, a.V, true);
    if (y < 0 || y >= a.V) return no_number<NT>(a, r, g, a.V, true);
    TokenRow<T, NT, NV> row;
    row.load(z, a.V, a.stream);
    const float zy = widen(z[y]);
    row.find(y, a.V);
    const float m = fmaxf(block_all<NT>(row.largest(), red, MaxOp()), zy);
    const Exponents ex = Exponents::of(uniform(m), a.log2_tau);
    if (!ex.near) row.recenter(m);
    const Sums o = row.template sum<Ent>(ex);
    double s[2] = {o.s, o.t};
    block_all<NT, Ent ? 2 : 1>(*(double(*)[Ent ? 2 : 1])s, red2, AddOp());
    if (threadIdx.x < 64) finish(a, r, m, zy, Sums{s[0], s[1]}, ex.off, w, true, &shared);
    if constexpr (!Grad) return;
    __syncthreads();
    const Slopes sl = shared;
    if (!sl.ok) return fill_row<NT>(g, a.V, kNan);
    const float a0 = uniform(sl.a0), a1 = uniform(sl.a1), gy = uniform(sl.gy);
    row.keep_packed();
    row.template store<Ent>(g, z, a.V, a.stream, ex, a0, a1, gy);
}

// ---- rows in parts

// what a part leaves in the workspace
struct PartStats {
    float m, s, t, zy;   // zy: the token's logit, in the part that holds it
};
struct PartsArgs {
    int parts, len;
    PartStats* stats;   // [rows][parts]
};

// the sums of a part, or of a whole row where parts = 1
template <typename T, int NT, int NV, bool Ent>
__device__ __forceinline__ void part_stats(const TokenArgs& a, const PartsArgs& p, int64_t r, int c, int y,
                                           PartStats* out, bool stream) {
    __shared__ float red[NT / 64];
    __shared__ double red2[2][NT / 64];
    const int first = c * p.len, V = min(p.len, a.V - first);
    const T* z = (const T*)a.logits + r * a.ld + first;
    TokenRow<T, NT, NV> row;
    row.load(z, V, stream);
    const bool here = y >= first && y < first + V;
    const float zy = here ? widen(z[y - first]) : 0.f;
    row.find(y - first, V);
    const float m = block_all<NT>(row.largest(), red, MaxOp());
    // relative to a finite number: a part of -infinities sums to 0
    const float from = m == -INFINITY ? 0.f : m;
    const Exponents ex = Exponents::of(from, a.log2_tau);
    if (!ex.near) row.recenter(from);
    const Sums o = row.template sum<Ent>(ex);
    double s[2] = {o.s, o.t};
    block_all<NT, Ent ? 2 : 1>(*(double(*)[Ent ? 2 : 1])s, red2, AddOp());
    if (threadIdx.x == 0) *out = PartStats{m, (float)s[0], Ent ? (float)s[1] : 0.f, zy};
}

// The sums of a part with the exponents of its row.
template <bool Ent>
__device__ __forceinline__ Sums part_sums(const PartStats& q, float m, const Exponents& ex, float2 c2,
                                          double inv_tau) {
    if (q.m == -INFINITY) return Sums{(double)q.s, 0.0};
    // what the part's exponents are off by in the row, to base 2
    const double by = (((double)q.m - (double)m) * inv_tau + ex.off - Exponents::of(q.m, c2).off) / kLn2d;
    const float e = exp_of(by * kLn2d);
    return Sums{(double)q.s * e, Ent && e > 0.f ? ((double)q.t + (double)q.s * by) * e : 0.0};
}

template <typename T, int NT, int NV, bool Ent>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT)))) void k_token_part(
    TokenArgs a, PartsArgs p, int64_t r0) {
    const int row = blockIdx.x / p.parts, c = blockIdx.x - row * p.parts;
    const int64_t r = r0 + row;
    const int y = a.tokens[r];
    if (y < 0 || y >= a.V || (a.weight && a.weight[r] == 0.f)) return;
    part_stats<T, NT, NV, Ent>(a, p, r, c, y, p.stats + (int64_t)row * p.parts + c, a.stream && !a.grad);
}

// Joins a row's parts (every part's workgroup does, a lane a part) and stores the
// gradient, reading the part again. Without a gradient: a wavefront a row.
template <typename T, int NT, int NV, bool Ent, bool Grad>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT)))) void k_token_rest(
    TokenArgs a, PartsArgs p, int64_t r0) {
    __shared__ Slopes shared;
    const int row = Grad ? blockIdx.x / p.parts : blockIdx.x, c = Grad ? blockIdx.x - row * p.parts : 0;
    const int64_t r = r0 + row;
    const int first = c * p.len, V = min(p.len, a.V - first);
    const T* z = (const T*)a.logits + r * a.ld + first;
    T* g = Grad ? (T*)a.grad + r * a.ld_grad + first : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y == -1 || w == 0.f) return no_part<NT>(a, r, g, V, c == 0);
    if (y < 0 || y >= a.V) return no_number<NT>(a, r, g, V, c == 0);
    TokenRow<T, NT, NV> part;
    if constexpr (Grad) part.load(z, V, a.stream);
    const PartStats* stats = p.stats + (int64_t)row * p.parts;
    const int lane = threadIdx.x & 63;
    const float2 c2 = a.log2_tau;
    const float zy = stats[y / p.len].zy;
    PartStats q{-INFINITY, 0.f, 0.f, 0.f};
    if (lane < p.parts) q = stats[lane];
    const float m = fmaxf(wave_all(q.m, MaxOp()), zy);
    const Exponents ex = Exponents::of(m, c2);
    if (threadIdx.x < 64) {
        Sums o = part_sums<Ent>(q, m, ex, c2, a.inv_tau);
        o.s = wave_all(o.s, AddOp());
        if constexpr (Ent) o.t = wave_all(o.t, AddOp());
        finish(a, r, m, zy, o, ex.off, w, c == 0, &shared);
    }
    if constexpr (!Grad) return;
    __syncthreads();
    const Slopes sl = shared;
    if (!sl.ok) return fill_row<NT>(g, V, kNan);
    part.find(y - first, V);
    const float a0 = uniform(sl.a0), a1 = uniform(sl.a1), gy = uniform(sl.gy);
    if (!ex.near) part.recenter(m);
    part.template store<Ent>(g, z, V, a.stream, ex, a0, a1, gy);
}

// ---- pairs of sequences

// A row's largest logit, what the stores of its log-probability's gradient need, and
// how many pairs take it as one of theirs (two do where offsets descend).
struct RowSlope {
    float m, a0, gy;
    int pairs;
};
struct PairArgs {
    PartsArgs p;
    RowSlope* slope;   // [rows]
    // [rows], a0 and gy times what the row's pair makes of them. (In the slopes' own place
    // two pairs of a row could scale it twice; apart, with the counting, the pairs' kernel
    // takes 0.4 to 0.7 us more.)
    float2* scaled;
    int64_t streams;   // rows that the second reading will not find in the caches
};

// rows ahead of the first sequence and behind the last are left out
__device__ __forceinline__ bool in_sequences(const PreferenceArgs& q, int64_t r) {
    return !q.first || (r >= q.first[0] && r < q.first[2 * q.pairs]);
}

// the first reading: a row's sums
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT)))) void k_pair_stats(
    TokenArgs a, PreferenceArgs q, PairArgs b, int64_t r0) {
    const int row = blockIdx.x / b.p.parts, c = blockIdx.x - row * b.p.parts;
    const int64_t r = r0 + row;
    const int y = a.tokens[r];
    const bool in = in_sequences(q, r);
    if (c == 0 && threadIdx.x == 0) b.slope[r] = RowSlope{0.f, 0.f, 0.f, 0};
    if (!in || y < 0 || y >= a.V) return;
    part_stats<T, NT, NV, false>(a, b.p, r, c, y, b.p.stats + r * b.p.parts + c, r < b.streams);
}

constexpr int kPairThreads = 1024;

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }
__device__ __forceinline__ double logistic(double x) { return 1.0 / (1.0 + exp(-x)); }

// l - ref of a row that has a token, from its parts; leaves the slopes of l
__device__ __forceinline__ double row_ratio(const TokenArgs& a, const PreferenceArgs& q, const PairArgs& b,
                                            int64_t r, int y) {
    RowSlope o{0.f, kNan, kNan, 0};
    double l = (double)kNan;
    if (y >= 0 && y < a.V) {
        const PartStats* stats = b.p.stats + r * b.p.parts;
        const float zy = stats[y / b.p.len].zy;
        o.m = zy;
        for (int c = 0; c < b.p.parts; ++c) o.m = fmaxf(o.m, stats[c].m);
        const Exponents ex = Exponents::of(o.m, a.log2_tau);
        Sums sum;
        for (int c = 0; c < b.p.parts; ++c)
            sum.s += part_sums<false>(stats[c], o.m, ex, a.log2_tau, a.inv_tau).s;
        const RowEnd e = row_end<false>(o.m, zy, sum, ex.off, a.inv_tau);
        l = e.l;
        const Slopes sl = slopes_of(e, Goal{0.0, 1.0, 0.0}, a.inv_tau);
        o.a0 = sl.a0;
        o.gy = sl.gy;
    }
    RowSlope& slope = b.slope[r];   // (another pair may count itself there meanwhile)
    slope.m = o.m;
    slope.a0 = o.a0;
    slope.gy = o.gy;
    return q.ref_logprob ? l - (double)q.ref_logprob[r] : l;
}

// the place of a row's l - ref where k_pair_rows() has formed it: its first part's sums
__device__ __forceinline__ double* ratio_at(const PairArgs& b, int64_t r) {
    return (double*)(b.p.stats + r * b.p.parts);
}

constexpr int kRowThreads = 256;

// The rows' log-probabilities ahead of the pairs, a lane a row, where the pairs have on
// average more than twice the rows that their workgroup has threads for. (One pair of
// 16384 rows of 300 fp32 entries 62 -> 38 us. The host does not know the offsets: a long
// pair beside many short ones is left to its workgroup.)
__global__ __launch_bounds__(kRowThreads) void k_pair_rows(TokenArgs a, PreferenceArgs q, PairArgs b) {
    const int64_t r = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    if (r >= a.rows) return;
    const int y = a.tokens[r];
    if (y != -1 && in_sequences(q, r)) *ratio_at(b, r) = row_ratio(a, q, b, r, y);
}

// A workgroup a pair: its rows' log-probabilities (or what k_pair_rows() has left of
// them), its loss, and the slope that each of its rows takes from that.
template <bool Formed>
__global__ __launch_bounds__(kPairThreads) void k_pair(TokenArgs a, PreferenceArgs q, PairArgs b,
                                                       int64_t pair0) {
    constexpr int NT = kPairThreads;
    __shared__ double red[4][NT / 64];
    const int64_t pair = pair0 + blockIdx.x;
    int64_t at[3];
    bool bad = false;
    for (int i = 0; i < 3; ++i) {
        const int64_t s = 2 * pair + i;
        at[i] = q.first ? (int64_t)q.first[s] : s * (a.rows / (2 * q.pairs));
        if (at[i] < 0 || at[i] > a.rows || (i && at[i] < at[i - 1])) bad = true;
    }
    // rows that in_sequences() leaves out have no sums
    if (q.first && (at[0] < q.first[0] || at[2] > q.first[2 * q.pairs])) bad = true;
    if (bad)
        for (int i = 0; i < 3; ++i) at[i] = min(max(at[i], (int64_t)0), a.rows);
    double s[4] = {0.0, 0.0, 0.0, 0.0};   // sums of l - ref, rows, of the two sequences
#pragma unroll Formed ? 4 : 1
    for (int64_t r = at[0] + threadIdx.x; r < at[2] && !bad; r += NT) {
        const int y = a.tokens[r];
        if (y == -1) continue;
        const double l = Formed ? *ratio_at(b, r) : row_ratio(a, q, b, r, y);
        const bool rejected = r >= at[1];
        s[0] += rejected ? 0.0 : l;
        s[1] += rejected ? l : 0.0;
        s[2] += rejected ? 0.0 : 1.0;
        s[3] += rejected ? 1.0 : 0.0;
    }
    block_all<NT, 4>(s, red, AddOp());
    __shared__ double by_l[2];   // the loss's slopes by the two sequences' log-probabilities
    __shared__ int sound;
    if (threadIdx.x < 64) {      // every wavefront doing this would take 4 us
        double n[2] = {1.0, 1.0};
        if (q.mean)
            for (int i = 0; i < 2; ++i) n[i] = fmax(s[2 + i], 1.0);
        const double chosen = bad ? (double)kNan : s[0] / n[0], rejected = bad ? (double)kNan : s[1] / n[1];
        const double u = chosen - rejected - q.margin, h = q.beta * u;
        double loss, slope;   // slope: by u
        if (q.form == HBSJD_PREFERENCE_SIGMOID) {
            loss = (1.0 - q.smoothing) * softplus(-h);
            slope = -(1.0 - q.smoothing) * logistic(-h);
            if (q.smoothing > 0.0) {
                loss += q.smoothing * softplus(h);
                slope += q.smoothing * logistic(h);
            }
            slope *= q.beta;
        } else if (q.form == HBSJD_PREFERENCE_HINGE) {
            loss = h < 1.0 ? 1.0 - h : h == h ? 0.0 : h;
            slope = h < 1.0 ? -q.beta : 0.0;
        } else {
            const double d = u - 0.5 / q.beta;
            loss = d * d;
            slope = 2.0 * d;
        }
        const float w = q.weight ? q.weight[pair] : 1.f;
        const float value = w == 0.f ? 0.f : (float)(w * loss);
        if (threadIdx.x == 0) {
            if (q.loss) q.loss[pair] = value;
            if (q.log_ratio) {
                q.log_ratio[2 * pair] = (float)chosen;
                q.log_ratio[2 * pair + 1] = (float)rejected;
            }
            sound = !bad && value > -INFINITY && value < INFINITY;
            by_l[0] = w == 0.f ? 0.0 : w * slope / n[0];
            by_l[1] = w == 0.f ? 0.0 : -w * slope / n[1];
        }
    }
    if (!a.grad) return;
    __syncthreads();
    // a pair in error may have one sequence that descends: the other one's rows are its
    for (int64_t r = min(at[0], at[1]) + threadIdx.x; r < max(at[1], at[2]); r += NT) {
        if (a.tokens[r] == -1) continue;
        float2 y = make_float2(kNan, kNan);
        if (sound) {
            const double f = by_l[r >= at[1] ? 1 : 0];
            y.x = f == 0.0 ? 0.f : (float)(b.slope[r].a0 * f);   // (a row in error weighted out)
            y.y = f == 0.0 ? 0.f : (float)(b.slope[r].gy * f);
        }
        b.scaled[r] = y;   // of no use where another pair stores its own
        atomicAdd(&b.slope[r].pairs, 1);
    }
}

// The second reading: the gradient. (From the last rows on, those that the first reading
// has left in the last-level cache, it is slower: 32 pairs of 256 fp32 rows of 16384 526
// us, so 515.)
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) void k_pair_grad(TokenArgs a, PairArgs b, int chunks, int len, int64_t r0) {
    const int row = blockIdx.x / chunks, c = blockIdx.x - row * chunks;
    const int64_t r = r0 + row;
    const int first = c * len, V = min(len, a.V - first);
    const T* z = (const T*)a.logits + r * a.ld + first;
    T* g = (T*)a.grad + r * a.ld_grad + first;
    const RowSlope o = b.slope[r];
    const float2 y = b.scaled[r];   // none where no pair has the row
    const float a0 = uniform(y.x), gy = uniform(y.y), m = uniform(o.m);
    const int pairs = uniform(o.pairs);
    if (pairs == 0 || (pairs == 1 && a0 == 0.f && gy == 0.f)) return fill_row<NT>(g, V, 0.f);
    if (pairs > 1 || a0 != a0 || gy != gy) return fill_row<NT>(g, V, kNan);
    TokenRow<T, NT, NV> part;
    part.load(z, V, a.stream);
    part.find(a.tokens[r] - first, V);
    const Exponents ex = Exponents::of(m, a.log2_tau);
    if (!ex.near) part.recenter(m);
    part.template store<false>(g, z, V, a.stream, ex, a0, 0.f, gy);
}

// ---- how a call runs

struct Plan {
    int parts = 0, len = 0;
    int64_t slab = 0;   // rows that the workspace holds at a time
};
constexpr int kPart = 16384;   // entries of a part at most

// parts of up to kPart entries, more of them until there are 512 workgroups, of
// 4096 entries at least and 64 at most (a lane each joins them)
void cut(Plan& p, int64_t rows, int V) {
    p.parts = (V + kPart - 1) / kPart;
    while (rows * p.parts < 512 && V / (2 * p.parts) >= 4096 && p.parts <= 32) p.parts *= 2;
    p.len = ((V + p.parts - 1) / p.parts + 7) / 8 * 8;
    p.parts = (V + p.len - 1) / p.len;
}

// Rows above 128 KB go in parts, but for those of up to 256 KB that a workgroup holds, one
// a CU: from 112 rows on (fewer leave CUs idle), with a gradient as long as the last
// round of the 256 CUs is not mostly idle, without one where there is one round only. In
// parts a gradient's rows are read twice, but reading alone has no need of registers:
// policy loss and gradient, held and in parts, 900 fp32 rows of 60000 95 and 114 us, 1000
// fp16 rows of 80000 81 and 86, 150 of 128257 26 and 29, but 300 bf16 ones of 70000 38
// and 31; log-probabilities of 130 fp32 rows of 60000 9 and 15, of 900 49 and 36.
Plan plan_of(int64_t rows, int V, int32_t elem, bool grad) {
    Plan p;
    const int64_t bytes = V * (int64_t)elem_size(elem);
    const int64_t places = (rows + 255) / 256 * 256;
    const bool filled = rows <= 256 || (grad && 4 * rows >= 3 * places);
    if (bytes <= 128 << 10 || (bytes <= 256 << 10 && rows >= 112 && filled)) return p;
    cut(p, rows, V);
    p.slab = std::min<int64_t>(rows, (1 << 20) / p.parts);
    return p;
}

// f(threads, vectors a thread) of the workgroups that hold rows of V entries. (Two
// workgroups of 512 threads and 16 vectors a CU, whose loads and stores overlap, for
// rows of 64 to 128 KB: 1000 fp32 rows of 30000 45 us, one of 1024 threads and 8 vectors
// 54; 3000 of 20000 92 and 122.)
template <typename T, typename F> void by_size(int V, F f) {
    using std::integral_constant;
    const int vecs = V / kVec<T>;
#define HELD(nt, nv) f(integral_constant<int, nt>{}, integral_constant<int, nv>{})
    if (vecs <= 64 * 2) HELD(64, 2);
    else if (vecs <= 64 * 8) HELD(64, 8);
    else if (vecs <= 256 * 4) HELD(256, 4);
    else if (vecs <= 256 * 8) HELD(256, 8);
    else if (vecs <= 512 * 8) HELD(512, 8);
    else if (vecs <= 512 * 16) HELD(512, 16);
    else if (vecs <= 1024 * 12) HELD(1024, 12);
    else HELD(1024, 16);
#undef HELD
}

template <typename T, bool Ent> void go(const TokenArgs& a, void* ws, hipStream_t s) {
    const Plan plan = plan_of(a.rows, a.V, a.elem, a.grad != nullptr);
    if (plan.parts) {
        constexpr int NT = 512, NV = kPart / kVec<T> / NT;
        const PartsArgs p{plan.parts, plan.len, (PartStats*)ws};
        for (int64_t r0 = 0; r0 < a.rows; r0 += plan.slab) {
            const dim3 rows((unsigned)std::min(plan.slab, a.rows - r0)), grid(rows.x * p.parts);
            hipLaunchKernelGGL((k_token_part<T, NT, NV, Ent>), grid, dim3(NT), 0, s, a, p, r0);
            if (a.grad) hipLaunchKernelGGL((k_token_rest<T, NT, NV, Ent, true>), grid, dim3(NT), 0, s, a, p, r0);
            else hipLaunchKernelGGL((k_token_rest<T, 64, 1, Ent, false>), rows, dim3(64), 0, s, a, p, r0);
        }
        return;
    }
    const size_t lds = resident_lds(0, a.V * sizeof(T));
    by_size<T>(a.V, [&](auto nt, auto nv) {
        by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            if (a.grad) hipLaunchKernelGGL((k_token<T, NT, NV, Ent, true>), grid, dim3(NT), lds, s, a, r0);
            else hipLaunchKernelGGL((k_token<T, NT, NV, Ent, false>), grid, dim3(NT), 0, s, a, r0);
        });
    });
}

// Calls on more than 64 MB read rows for the last time, and write gradients, as streams.
// Passes among others, with usual loads and stores, with streamed stores, with both: log-
// probabilities of 6144 fp32 rows of 16384 72, 72, 65 us; policy loss and gradient there
// 147, 141, 142; gradients of 18432 bf16 rows 195, 191, 177; 8192 bf16 rows in pairs 132,
// 121, 120; 4 pairs of 101 bf16 rows of 128257 104, 97, 89. (Of less, what reads the
// gradient next finds it in the cache.) The first reading of pairs is streams but for its
// last 192 MB, which the second one may find in the last-level cache of 256 (the 8192
// rows 119 us without, 116).
constexpr int64_t kSmall = 64 << 20, kCached = 192 << 20;
template <typename T> TokenArgs streamed(const TokenArgs& a) {
    TokenArgs b = a;
    b.stream = a.rows * a.V * (int64_t)sizeof(T) > kSmall;
    return b;
}

template <typename T> void go_token(const TokenArgs& args, void* ws, hipStream_t s) {
    const TokenArgs a = streamed<T>(args);
    const bool entropy = a.entropy || a.entropy_weight || (a.advantage && a.bonus > 0.f);
    if (entropy) go<T, true>(a, ws, s);
    else go<T, false>(a, ws, s);
}

Plan pair_plan(int64_t rows, int V) {
    Plan p;
    cut(p, rows, V);
    return p;
}

// entries of a row that a workgroup of the second reading takes: 16 KB
template <typename T> constexpr int kChunk2 = 256 * 4 * kVec<T>;

template <typename T>
void go_pairs(const TokenArgs& args, const PreferenceArgs& q, void* ws, hipStream_t s) {
    const TokenArgs a = streamed<T>(args);
    const Plan plan = pair_plan(a.rows, a.V);
    PairArgs b;
    b.slope = (RowSlope*)ws;
    b.streams = a.rows - kCached / (int64_t)(a.V * sizeof(T));
    b.p = PartsArgs{plan.parts, plan.len, (PartStats*)(b.slope + a.rows)};
    b.scaled = (float2*)(b.p.stats + a.rows * plan.parts);
    const size_t lds = resident_lds(0, plan.len * sizeof(T));
    by_size<T>(plan.len, [&](auto nt, auto nv) {
        constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
        if constexpr (NT <= 512 && NV <= 8)   // a part's entries are no more
            by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
                hipLaunchKernelGGL((k_pair_stats<T, NT, NV>), grid, dim3(NT), lds, s, a, q, b, r0);
            }, plan.parts);
    });
    const bool formed = a.rows > 2 * kPairThreads * q.pairs;
    if (formed)
        hipLaunchKernelGGL(k_pair_rows, dim3((unsigned)((a.rows + kRowThreads - 1) / kRowThreads)),
                           dim3(kRowThreads), 0, s, a, q, b);
    by_slabs(q.pairs, [&](int64_t p0, dim3 grid) {
        if (formed) hipLaunchKernelGGL(k_pair<true>, grid, dim3(kPairThreads), 0, s, a, q, b, p0);
        else hipLaunchKernelGGL(k_pair<false>, grid, dim3(kPairThreads), 0, s, a, q, b, p0);
    });
    if (!a.grad) return;
    const int chunks = (a.V + kChunk2<T> - 1) / kChunk2<T>;
    const int len = ((a.V + chunks - 1) / chunks + 7) / 8 * 8;
    by_size<T>(len, [&](auto nt, auto nv) {
        constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
        if constexpr (NT * NV <= 1024) {   // up to kChunk2
            by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
                hipLaunchKernelGGL((k_pair_grad<T, NT, NV>), grid, dim3(NT), 0, s, a, b, chunks, len, r0);
            }, chunks);
        }
    });
}

}  // namespace

size_t token_workspace(int64_t rows, int V, int32_t elem) {
    const Plan p = plan_of(rows, V, elem, false);   // where a gradient goes in parts, so does none
    return (size_t)p.slab * p.parts * sizeof(PartStats);
}

void token_rows(const TokenArgs& a, void* workspace, hipStream_t s) {
    if (a.elem == HBSJD_ELEM_F32) go_token<float>(a, workspace, s);
    else if (a.elem == HBSJD_ELEM_BF16) go_token<Bf16>(a, workspace, s);
    else go_token<F16>(a, workspace, s);
}

size_t preference_workspace(int64_t rows, int V, int32_t) {
    const Plan p = pair_plan(rows, V);
    return (size_t)rows * (sizeof(RowSlope) + p.parts * sizeof(PartStats) + sizeof(float2));
}

void preference_rows(const TokenArgs& a, const PreferenceArgs& p, void* workspace, hipStream_t s) {
    if (a.elem == HBSJD_ELEM_F32) go_pairs<float>(a, p, workspace, s);
    else if (a.elem == HBSJD_ELEM_BF16) go_pairs<Bf16>(a, p, workspace, s);
    else go_pairs<F16>(a, p, workspace, s);
}

}  // namespace hbsjd
