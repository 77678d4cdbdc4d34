// What is done to logits before a draw, per entry v of row r:
//   1. v held by the row's sequence (count c > 0): x = x > 0 ? x / theta : x theta
//   2. x = x - frequency c, then x = x - presence for c > 0
//   3. x = x + the row's bias on v
//   4. -infinity where the row's mask does not allow v
// each operation rounded once in fp32, the result once to the output's type.
#include "rows.h"

#pragma clang fp contract(off)

namespace hbsjd {
namespace {

constexpr int kPart = 4096;   // entries per workgroup

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_adjust(AdjustArgs a, int parts, int64_t item0) {
    constexpr int NT = 256;
    __shared__ int count[kPart];
    __shared__ float bias[kPart];
    __shared__ int list[HBSJD_ADJUST_MAX_BIASES];
    const int t = threadIdx.x;
    {
        const int64_t item = item0 + blockIdx.x;
        const int64_t r = item / parts;
        const int v0 = (int)(item - r * parts) * kPart, n = min(kPart, a.V - v0);
        const T* z = (const T*)a.logits + r * a.ld + v0;
        O* o = (O*)a.out + r * a.ld_out + v0;
        __syncthreads();
        for (int i = t; i < n; i += NT) {
            count[i] = 0;
            bias[i] = 0.f;
        }
        for (int i = t; i < a.n_bias; i += NT) list[i] = a.bias_index[r * a.ld_bias + i];
        __syncthreads();
        if (a.tokens) {
            const int held = a.token_count ? min(a.token_count[r], a.n_tokens) : a.n_tokens;
            for (int i = t; i < held; i += NT) {
                const int64_t v = (int64_t)a.tokens[r * a.ld_tokens + i] - v0;
                if (v >= 0 && v < n) atomicAdd(&count[v], 1);
            }
        }
        for (int i = t; i < a.n_bias; i += NT) {
            const int64_t v = (int64_t)list[i] - v0;
            if (v < 0 || v >= n) continue;
            // an entry listed more than once: its first place adds them all, in order
            bool first = true;
            for (int j = 0; j < i; ++j) first &= list[j] != list[i];
            if (!first) continue;
            float b = a.bias_value[r * a.ld_bias + i];
            for (int j = i + 1; j < a.n_bias; ++j)
                if (list[j] == list[i]) b = b + a.bias_value[r * a.ld_bias + j];
            bias[v] = b;
        }
        __syncthreads();
        const float theta = a.repetition ? a.repetition[r] : 1.f;
        const float presence = a.presence ? a.presence[r] : 0.f;
        const float frequency = a.frequency ? a.frequency[r] : 0.f;
        const uint32_t* mask = a.mask;
        bool bad = false;
        if (mask) {
            const int64_t q = a.mask_row ? a.mask_row[r] : r;
            bad = q >= a.n_masks;
            mask = q < 0 || bad ? nullptr : mask + q * ((a.V + 31) / 32);
        }
        for (int i = t; i < n; i += NT) {
            float x = widen(z[i]);
            const int c = count[i];
            if (c > 0) {
                x = x > 0.f ? x / theta : x * theta;
                x = x - frequency * (float)c;
                x = x - presence;
            }
            x = x + bias[i];
            const int v = v0 + i;
            if (mask && !(mask[v >> 5] >> (v & 31) & 1)) x = -INFINITY;
            o[i] = narrow<O>(bad ? __builtin_nanf("") : x);
        }
    }
}

template <typename T, typename O>
void go(const AdjustArgs& a, hipStream_t s) {
    const int parts = (a.V + kPart - 1) / kPart;
    by_slabs(a.rows * parts, [&](int64_t item0, dim3 grid) {
        hipLaunchKernelGGL((k_adjust<T, O>), grid, dim3(256), 0, s, a, parts, item0);
    });
}

}  // namespace

void adjust_rows(const AdjustArgs& a, hipStream_t s) {
    const bool wide = a.out_elem == HBSJD_ELEM_F32;
    if (a.elem == HBSJD_ELEM_F32)
        go<float, float>(a, s);
    else if (a.elem == HBSJD_ELEM_BF16)
        wide ? go<Bf16, float>(a, s) : go<Bf16, Bf16>(a, s);
    else
        wide ? go<F16, float>(a, s) : go<F16, F16>(a, s);
}

}  // namespace hbsjd
