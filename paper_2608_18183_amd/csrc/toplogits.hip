// A row's K largest logits in descending order (the lowest index first among
// equals), their indices, and the log mass of all other entries at temperature
// tau: rest = log sum over the unlisted v of exp(z_v / tau).
//
// Logits are compared by an order-preserving 32-bit image. The K-th largest
// image is found digit by digit from the top; among the entries equal to it the
// lowest indices are taken, up to an index found the same way. The kept
// entries are collected and sorted as 64-bit numbers, image above complemented
// index, so no two are equal and the order of collection does not matter.
#include "rows.h"

namespace hbsjd {
namespace {

// larger for larger logits; -0 as +0, every NaN above +infinity
__device__ __forceinline__ uint32_t order_of(float x) {
    uint32_t u = __float_as_uint(x + 0.f);
    if (x != x) return 0xFFFFFFFFu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <typename T>
__global__ __launch_bounds__(256) void k_top(TopArgs a, int64_t r0) {
    constexpr int NT = 256;
    __shared__ uint64_t kept[HBSJD_TOP_MAX];
    __shared__ int hist[256];
    __shared__ int s_digit, s_above, s_n;
    __shared__ float red[NT / 64], red2[NT / 64];
    const int t = threadIdx.x;
    {
        const int64_t r = r0 + blockIdx.x;
        const T* z = (const T*)a.logits + r * a.ld;
        // the composite's upper 32 bits, then the 18 bits of the index
        uint64_t prefix = 0;
        int need = a.K;   // rank of the wanted entry among those that share the prefix
        for (int shift = 48; shift >= 0; shift -= 8) {
            __syncthreads();
            hist[t] = 0;
            __syncthreads();
            for (int v = t; v < a.V; v += NT) {
                const uint64_t c = (uint64_t)order_of(widen(z[v])) << 24 | (0xFFFFFFu - v);
                if (shift == 48 || c >> (shift + 8) == prefix) atomicAdd(&hist[c >> shift & 255], 1);
            }
            __syncthreads();
            if (t == 0) {
                int above = 0, d = 255;
                while (above + hist[d] < need) above += hist[d--];
                s_digit = d;
                s_above = above;
            }
            __syncthreads();
            prefix = prefix << 8 | s_digit;
            need -= s_above;
        }
        if (t == 0) s_n = 0;
        __syncthreads();
        float m = -INFINITY;
        for (int v = t; v < a.V; v += NT) {
            const float x = widen(z[v]);
            const uint64_t c = (uint64_t)order_of(x) << 24 | (0xFFFFFFu - v);
            if (c >= prefix) kept[atomicAdd(&s_n, 1)] = c;
            else m = fmaxf(m, x);
        }
        int n = 1;
        while (n < a.K) n *= 2;
        for (int i = a.K + t; i < n; i += NT) kept[i] = 0;
        m = block_all<NT>(m, red, MaxOp());
        float s = 0.f;
        for (int v = t; v < a.V; v += NT) {
            const float x = widen(z[v]);
            const uint64_t c = (uint64_t)order_of(x) << 24 | (0xFFFFFFu - v);
            if (c < prefix) s += __expf((x - m) * a.inv_tau);
        }
        s = block_all<NT>(s, red2, AddOp());
        for (int size = 2; size <= n; size *= 2)
            for (int step = size / 2; step > 0; step /= 2) {
                __syncthreads();
                for (int i = t; i < n / 2; i += NT) {
                    const int lo = (i / step) * 2 * step + i % step, hi = lo + step;
                    const uint64_t x = kept[lo], y = kept[hi];
                    if ((x < y) == !(lo & size)) {
                        kept[lo] = y;
                        kept[hi] = x;
                    }
                }
            }
        __syncthreads();
        for (int k = t; k < a.K; k += NT) {
            const int v = 0xFFFFFF - (int)(kept[k] & 0xFFFFFF);
            a.values[r * a.K + k] = widen(z[v]);
            a.index[r * a.K + k] = v;
        }
        if (t == 0) {
            const bool nan = kept[0] >> 24 == 0xFFFFFFFFu;
            a.rest[r] = nan ? __builtin_nanf("") : fabsf(m) == INFINITY ? m : m * a.inv_tau + __logf(s);
        }
    }
}

}  // namespace

void top_logits(const TopArgs& a, hipStream_t s) {
    by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
    const dim3 block(256);
    if (a.elem == HBSJD_ELEM_F32)
        hipLaunchKernelGGL(k_top<float>, grid, block, 0, s, a, r0);
    else if (a.elem == HBSJD_ELEM_BF16)
        hipLaunchKernelGGL(k_top<Bf16>, grid, block, 0, s, a, r0);
    else
        hipLaunchKernelGGL(k_top<F16>, grid, block, 0, s, a, r0);
    });
}

}  // namespace hbsjd
