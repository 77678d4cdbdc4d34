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
// to a peaked teacher has a q_0 far below the rounding of that difference.
#include "rows.h"

namespace hbsjd {
namespace {

constexpr float kNan = __builtin_nanf("");

template <typename T>
__global__ __launch_bounds__(256) void k_distill(DistillArgs a) {
    constexpr int NT = 256;
    __shared__ float red[6][NT / 64];
    __shared__ uint32_t listed[HBSJD_ROWS_MAX_VOCAB / 32];
    __shared__ float zk[HBSJD_TOP_MAX];   // the student's logits at the listed entries
    __shared__ int bad;
    const int t = threadIdx.x;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* z = (const T*)a.logits + r * a.ld;
        T* g = a.grad ? (T*)a.grad + r * a.ld_grad : nullptr;
        const float w = a.weight ? a.weight[r] : 1.f;
        if (w == 0.f) {
            if (g)
                for (int v = t; v < a.V; v += NT) g[v] = narrow<T>(0.f);
            if (a.loss && t == 0) a.loss[r] = 0.f;
            continue;
        }
        __syncthreads();
        for (int i = t; i < (a.V + 31) / 32; i += NT) listed[i] = 0;
        if (t == 0) bad = 0;
        __syncthreads();
        const float* tv = a.values + r * a.K;
        const int32_t* ti = a.index + r * a.K;
        const float rest = a.rest ? a.rest[r] : -INFINITY;
        float mt = rest;
        for (int k = t; k < a.K; k += NT) {
            const int v = ti[k];
            if (v == -1) continue;
            if (v < 0 || v >= a.V) { bad = 1; continue; }
            if (atomicOr(&listed[v >> 5], 1u << (v & 31)) >> (v & 31) & 1) bad = 1;
            zk[k] = widen(z[v]);
            mt = fmaxf(mt, tv[k] * a.inv_tau);
        }
        __syncthreads();
        float m0 = -INFINITY, mk = -INFINITY;   // maxima of the unlisted and the listed entries
        for (int v = t; v < a.V; v += NT)
            if (!(listed[v >> 5] >> (v & 31) & 1)) m0 = fmaxf(m0, widen(z[v]));
        for (int k = t; k < a.K; k += NT) {
            const int v = ti[k];
            if (v >= 0 && v < a.V) mk = fmaxf(mk, zk[k]);
        }
        m0 = block_all<NT>(m0, red[0], MaxOp());
        mk = block_all<NT>(mk, red[1], MaxOp());
        mt = block_all<NT>(mt, red[2], MaxOp());
        const float m = fmaxf(m0, mk);
        if (m0 == -INFINITY) m0 = m;
        float s0 = 0.f, sk = 0.f, st = 0.f;
        for (int v = t; v < a.V; v += NT)
            if (!(listed[v >> 5] >> (v & 31) & 1)) s0 += __expf((widen(z[v]) - m0) * a.inv_tau);
        for (int k = t; k < a.K; k += NT) {
            const int v = ti[k];
            if (v < 0 || v >= a.V) continue;
            sk += __expf((zk[k] - m) * a.inv_tau);
            st += __expf(tv[k] * a.inv_tau - mt);
        }
        s0 = block_all<NT>(s0, red[3], AddOp());
        sk = block_all<NT>(sk, red[4], AddOp());
        st = block_all<NT>(st, red[5], AddOp());
        if (a.rest) st += __expf(rest - mt);
        const float sz = s0 * __expf((m0 - m) * a.inv_tau) + sk;
        // no distribution: nothing left, a NaN or an infinity (the sums are then 0 or NaN)
        const bool refused = bad || !(sz > 0.f && st > 0.f);
        const float lz = __logf(sz), lt = mt + __logf(st);
        float lsum = 0.f, rsum = 0.f;
        auto cls = [&](int k, float& p, float& q, float& c) {
            const float lp = tv[k] * a.inv_tau - lt, lq = (zk[k] - m) * a.inv_tau - lz;
            p = __expf(lp);
            q = __expf(lq);
            c = lq - lp;
        };
        for (int k = t; k < a.K; k += NT) {
            const int v = ti[k];
            if (v < 0 || v >= a.V) continue;
            float p, q, c;
            cls(k, p, q, c);
            if (p > 0.f) lsum -= p * c;
            if (q > 0.f) rsum += q * c;
        }
        __syncthreads();
        lsum = block_all<NT>(lsum, red[0], AddOp());
        rsum = block_all<NT>(rsum, red[1], AddOp());
        const float lq0 = (m0 - m) * a.inv_tau + __logf(s0) - lz, q0 = __expf(lq0);
        float a0 = a.alpha * q0;   // unlisted: the gradient is a0 exp((z - m0) / tau) / s0
        if (a.rest) {
            const float lp = rest - lt, p = __expf(lp), c = lq0 - lp;
            if (p > 0.f) lsum -= p * c;
            if (q0 > 0.f) rsum += q0 * c;
            a0 -= a.alpha * p;
            if (a.beta > 0.f && q0 > 0.f) a0 += a.beta * q0 * (c - rsum);
        }
        a0 = s0 > 0.f ? a0 / s0 : 0.f;
        float loss = a.alpha > 0.f ? a.alpha * lsum : 0.f;
        if (a.beta > 0.f) loss += a.beta * rsum;
        if (refused || !(loss > -INFINITY && loss < INFINITY)) {
            const float l = refused || loss != loss ? kNan : loss;
            if (a.loss && t == 0) a.loss[r] = w * l;
            if (g) {
                __syncthreads();
                for (int v = t; v < a.V; v += NT) g[v] = narrow<T>(kNan);
            }
            continue;
        }
        if (a.loss && t == 0) a.loss[r] = w * loss;
        if (!g) continue;
        const float wt = w * a.inv_tau;
        for (int v = t; v < a.V; v += NT)
            if (!(listed[v >> 5] >> (v & 31) & 1))
                g[v] = narrow<T>(wt * a0 * __expf((widen(z[v]) - m0) * a.inv_tau));
        for (int k = t; k < a.K; k += NT) {
            const int v = ti[k];
            if (v < 0) continue;
            float p, q, c;
            cls(k, p, q, c);
            float d = a.alpha * (q - p);
            if (a.beta > 0.f && q > 0.f) d += a.beta * q * (c - rsum);
            g[v] = narrow<T>(wt * d);
        }
    }
}

}  // namespace

void distill_top(const DistillArgs& a, hipStream_t s) {
    const dim3 grid = row_grid(a.rows), block(256);
    if (a.elem == HBSJD_ELEM_F32)
        hipLaunchKernelGGL(k_distill<float>, grid, block, 0, s, a);
    else if (a.elem == HBSJD_ELEM_BF16)
        hipLaunchKernelGGL(k_distill<Bf16>, grid, block, 0, s, a);
    else
        hipLaunchKernelGGL(k_distill<F16>, grid, block, 0, s, a);
}

}  // namespace hbsjd
