// What is done to logits before a draw, per entry v of row r:
//   1. v held by the row's sequence (count c > 0): x = x > 0 ? x / theta : x theta
//   2. x = x - frequency c, then x = x - presence for c > 0
//   3. x = x + the row's bias on v
//   4. -infinity where the row's mask does not allow v
// each operation rounded once in fp32, the result once to the output's type.
//
// A workgroup takes a part of a row. It counts the sequence's tokens that fall
// into its part in LDS, so that an entry's count costs a fraction of a vector's
// LDS access, and moves the logits through registers once, as 16-byte vectors.
// Biased entries are few: a thread works one out by itself and leaves the result
// in LDS, with a tag in place of the entry's count. (Storing such entries over
// the part's vectors instead costs more than the vectors' arithmetic: 4224 bf16
// rows with 64 biases took 12 us longer, and 6400 fp32 rows whose penalties were
// stored that way 40.)
#include "rows.h"

#include <algorithm>

static_assert((HBSJD_ADJUST_MAX_BIASES & (HBSJD_ADJUST_MAX_BIASES - 1)) == 0, "a place in the list is a tag's low bits");

#pragma clang fp contract(off)

namespace hbsjd {
namespace {

// LDS of a workgroup: counts or tags of its entries, 16 bits each (32 where a row
// may hold more tokens than 15 bits count); the mask's words; the bias list's
// entries and what becomes of them
struct AdjustLds {
    uint32_t* count;
    uint32_t* biased;   // a bit per entry
    uint32_t* mask;
    int32_t* list;
    float* result;
};
constexpr int kCountMost = 32767;
inline __host__ __device__ int count_words(int len, bool wide) { return wide ? len : (len + 1) / 2; }

struct Penalties {
    float theta, presence, frequency;
    __device__ __forceinline__ float operator()(float x, uint32_t c) const {
        float y = x > 0.f ? x / theta : x * theta;
        y = y - frequency * (float)c;
        y = y - presence;
        return c > 0 ? y : x;
    }
};

template <typename O>
__device__ __forceinline__ void store_vec(O* o, const float* y, int n, bool aligned) {
    if (aligned) {
#pragma unroll
        for (int i = 0; i < n; i += kVec<O>) {
            float part[kVec<O>];
#pragma unroll
            for (int q = 0; q < kVec<O>; ++q) part[q] = y[i + q];
            *(u32x4*)(o + i) = vec_pack<O>(part);
        }
    } else {
#pragma unroll
        for (int q = 0; q < n; ++q) o[q] = narrow<O>(y[q]);
    }
}

template <typename T, typename O, int NT, int NV, bool Biased>
__global__ __launch_bounds__(NT) void k_adjust(AdjustArgs a, int parts, int len, bool wide, int64_t r0) {
    constexpr int E = kVec<T>;
    constexpr int NB = (HBSJD_ADJUST_MAX_BIASES + NT - 1) / NT;
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ int twice;
    const int t = threadIdx.x;
    const int row = blockIdx.x / parts;
    const int64_t r = r0 + row;
    const int first = (blockIdx.x - row * parts) * len, V = min(len, a.V - first);
    const T* z = (const T*)a.logits + r * a.ld + first;
    O* o = (O*)a.out + r * a.ld_out + first;
    const bool counts = a.tokens != nullptr, listed = counts || Biased;
    const uint32_t tag = wide ? 0x80000000u : 0x8000u;

    const Span sp = Span::of(z, V);
    const u32x4* z4 = (const u32x4*)(z + sp.head);
    u32x4 x[NV];
    float xe = 0.f;
    if (sp.vecs > 0)
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = vec_at(z4, min(t + NT * i, sp.vecs - 1));
    if (t < sp.edges()) xe = widen(z[sp.edge(t, V)]);

    AdjustLds l;
    l.count = lds;
    l.biased = l.count + (listed ? (count_words(len, wide) + 3) / 4 * 4 : 0);
    l.mask = l.biased + (Biased ? (len + 31) / 32 : 0);
    l.list = (int32_t*)(l.mask + (a.mask ? len / 32 + 2 : 0));
    l.result = (float*)(l.list + a.n_bias);

    const uint32_t* mask = a.mask;
    bool bad = false;
    if (mask) {
        const int64_t q = a.mask_row ? a.mask_row[r] : r;
        bad = q >= a.n_masks;
        const int words = (a.V + 31) / 32;
        mask = q < 0 || bad ? nullptr : mask + q * words;
        if (mask)
            for (int i = t; i < len / 32 + 2; i += NT) l.mask[i] = mask[min((first >> 5) + i, words - 1)];
    }
    if (listed)
        for (int i = t; i < count_words(V, wide); i += NT) l.count[i] = 0;
    if (Biased)
        for (int i = t; i < (V + 31) / 32; i += NT) l.biased[i] = 0;
    if (t == 0) twice = 0;
    __syncthreads();
    Penalties pen{1.f, 0.f, 0.f};
    if (counts) {
        pen.theta = a.repetition ? a.repetition[r] : 1.f;
        pen.presence = a.presence ? a.presence[r] : 0.f;
        pen.frequency = a.frequency ? a.frequency[r] : 0.f;
        const unsigned held = a.token_count ? max(0, min(a.token_count[r], a.n_tokens)) : a.n_tokens;
        const int32_t* tok = a.tokens + r * a.ld_tokens;
        // two loads in flight a thread: 64 rows of 128257 with 4096 tokens take 16.4
        // us so, 17.3 with one; more slow ordinary lists down
        for (unsigned i = t; i < held; i += 2 * NT) {
            int v[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) v[n] = tok[min(i + NT * n, held - 1)];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (i + NT * n >= held || v[n] < first || v[n] - first >= V) continue;
                const int p = sp.place(v[n] - first, V);
                if (wide) atomicAdd(&l.count[p], 1u);
                else atomicAdd(&l.count[p >> 1], 1u << (p & 1) * 16);
            }
        }
    }
    // this thread's biased entries (-1: none), their logits and biases
    int bv[NB];
    float bz[NB], bb[NB];
    const float* bval = Biased ? a.bias_value + r * a.ld_bias : nullptr;
    if constexpr (Biased) {
        const int32_t* bi = a.bias_index + r * a.ld_bias;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int i = t + NT * n;
            bv[n] = -1;
            if (i >= a.n_bias) continue;
            const bool here = bi[i] >= first && bi[i] - first < V;
            l.list[i] = here ? bi[i] - first : -1;
            if (!here) continue;
            const int v = l.list[i];
            bv[n] = v;
            bz[n] = widen(z[v]);
            bb[n] = bval[i];
            if (atomicOr(&l.biased[v >> 5], 1u << (v & 31)) >> (v & 31) & 1) twice = 1;
        }
    }
    __syncthreads();
    auto count_of = [&](int p) -> uint32_t {
        return !listed ? 0 : wide ? l.count[p] : l.count[p >> 1] >> (p & 1) * 16 & 0xFFFFu;
    };
    if constexpr (Biased) {
        const bool searched = twice;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int i = t + NT * n, v = bv[n];
            if (v < 0) continue;
            if (searched) {
                // an entry listed more than once: its first mention adds them all, in order.
                // Every biased entry of the part looks for its equals then: 4224 bf16 rows
                // with one entry twice among 64, 300 and 1024 biases take 120, 184 and 768
                // us, without it 98, 102 and 122.
                bool mentioned = false;
                for (int j = 0; j < i; ++j) mentioned |= l.list[j] == v;
                if (mentioned) continue;
                for (int j = i + 1; j < a.n_bias; ++j)
                    if (l.list[j] == v) bb[n] = bb[n] + bval[j];
            }
            const int p = sp.place(v, V);
            l.result[i] = pen(bz[n], count_of(p)) + bb[n];
            if (wide) l.count[p] = tag | i;
            else ((uint16_t*)l.count)[p] = (uint16_t)(tag | i);
        }
        __syncthreads();
    }
    auto apply = [&](float x, uint32_t c) {
        if constexpr (!Biased) return pen(x, c);
        return c & tag ? l.result[c & (HBSJD_ADJUST_MAX_BIASES - 1)] : pen(x, c);
    };
    // the mask's bits from entry v of the part on
    auto allowed = [&](int v) -> uint32_t {
        const int b = (first & 31) + v;
        return __builtin_amdgcn_alignbit(l.mask[(b >> 5) + 1], l.mask[b >> 5], b & 31);
    };
    const bool aligned = ((uintptr_t)(o + sp.head) & 15) == 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = t + NT * i;
        if (j >= sp.vecs) continue;
        float y[E];
#pragma unroll
        for (int q = 0; q < E; ++q) y[q] = vec_get<T>(x[i], q);
        if (listed) {
            uint32_t c[E];
            if (wide) {
#pragma unroll
                for (int q = 0; q < E; q += 4) {
                    const u32x4 w = *(const u32x4*)(l.count + j * E + q);
#pragma unroll
                    for (int k = 0; k < 4; ++k) c[q + k] = w[k];
                }
            } else {
#pragma unroll
                for (int q = 0; q < E; q += 4) {
                    const uint2 w = *(const uint2*)(l.count + (j * E + q) / 2);
                    c[q] = w.x & 0xFFFFu;
                    c[q + 1] = w.x >> 16;
                    c[q + 2] = w.y & 0xFFFFu;
                    c[q + 3] = w.y >> 16;
                }
            }
            uint32_t any = 0;
#pragma unroll
            for (int q = 0; q < E; ++q) any |= c[q];
            if (any) {
#pragma unroll
                for (int q = 0; q < E; ++q) y[q] = apply(y[q], c[q]);
            }
        }
        if (mask) {
            const uint32_t bits = allowed(sp.head + j * E);
#pragma unroll
            for (int q = 0; q < E; ++q) y[q] = bits >> q & 1 ? y[q] : -INFINITY;
        }
        if (bad)
#pragma unroll
            for (int q = 0; q < E; ++q) y[q] = __builtin_nanf("");
        store_vec(o + sp.head + j * E, y, E, aligned);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (t < sp.edges()) {
        const int v = sp.edge(t, V);
        float y = apply(xe, count_of(sp.vecs * E + t));
        if (mask && !(allowed(v) & 1)) y = -INFINITY;
        o[v] = narrow<O>(bad ? __builtin_nanf("") : y);
    }
}

template <typename T, typename O, int NT, int NV> void run(const AdjustArgs& a, hipStream_t s) {
    // 16 entries: a part starts where a vector of the row does, for every type
    const int most = NT * NV * kVec<T>;
    int parts = (a.V + most - 1) / most;
    const int len = ((a.V + parts - 1) / parts + 15) / 16 * 16;
    parts = (a.V + len - 1) / len;
    const bool wide = a.n_tokens > kCountMost;
    size_t lds = 0;
    if (a.tokens || a.n_bias) lds += (count_words(len, wide) + 3) / 4 * 4;
    if (a.n_bias) lds += (len + 31) / 32 + 2 * a.n_bias;
    if (a.mask) lds += len / 32 + 2;
    lds = resident_lds(lds * 4, len * sizeof(T));
    by_slabs(
        a.rows,
        [&](int64_t r0, dim3 grid) {
            if (a.n_bias)
                hipLaunchKernelGGL((k_adjust<T, O, NT, NV, true>), grid, dim3(NT), lds, s, a, parts, len,
                                   wide, r0);
            else
                hipLaunchKernelGGL((k_adjust<T, O, NT, NV, false>), grid, dim3(NT), lds, s, a, parts, len,
                                   wide, r0);
        },
        parts);
}

template <typename T, typename O> void go(const AdjustArgs& a, hipStream_t s) {
    // Larger parts read a row's token list fewer times; smaller ones spread few
    // rows over more CUs. 32-bit counts of the largest would not fit.
    const int vecs = a.V / kVec<T>;
    if (vecs <= 64 * 2) run<T, O, 64, 2>(a, s);
    else if (a.rows * ((a.V + 16383) / 16384) < 512 || vecs <= 256 * 4 || a.n_tokens > kCountMost)
        run<T, O, 256, 4>(a, s);
    else run<T, O, 512, 16384 / kVec<T> / 512>(a, s);
}

}  // namespace

void adjust_rows(const AdjustArgs& a, hipStream_t s) {
    const bool wide = a.out_elem == HBSJD_ELEM_F32;
    if (a.elem == HBSJD_ELEM_F32) go<float, float>(a, s);
    else if (a.elem == HBSJD_ELEM_BF16) wide ? go<Bf16, float>(a, s) : go<Bf16, Bf16>(a, s);
    else wide ? go<F16, float>(a, s) : go<F16, F16>(a, s);
}

}  // namespace hbsjd
