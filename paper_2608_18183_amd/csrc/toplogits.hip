// A row's K largest logits in descending order (the lowest index first among
// equals), their indices, and the log mass of all other entries at temperature
// tau: rest = log sum over the unlisted v of exp(z_v / tau).
//
// The row is read once and held in registers. Its K largest entries are found
// in three steps:
//   1. A pivot p0 that at least K entries reach. The row is cut into groups
//      (a thread's entries, or an eighth of them for large K), each wavefront
//      takes the ceil(K / wavefronts)-th largest of its groups' maxima, and p0 is
//      the least of these: as many different entries as groups reach it.
//      Sampling maxima this way leaves 1.3 to 2 K candidates where a logit's size
//      has nothing to do with its index.
//   2. The entries that reach p0 are collected as 64-bit numbers, an
//      order-preserving image of the logit above the complemented index, so no
//      two are equal. The mass below p0 is summed in the same pass.
//   3. A candidate's place in the output is the number of larger ones: counted
//      over all of them when they are few, else over those of its bin, in bins
//      of equal width between the least and the largest candidate.
// Rows on which this fails (more candidates or equal ones than there is room
// for, NaN, a pivot next to fp32's ends) take digit-by-digit selection and a
// bitonic sort instead, with the same results. Equal entries are one cause, large
// logits that lie together the other: a wavefront holds runs of neighbouring
// entries, the one with the smallest takes its share from those, and more than
// there is room for reach its pivot. 2048 rows of 16384, us, fp32 and bf16:
//                                          K 64         K 256         K 2000
//   noise                                40    37      45    42      83    68
//   noise - ln(1 + index)                42   116     216   384     599   467
//   noise - 1.5 ln(1 + index)            43   383     534   404     589   460
//   descending or ascending         500-530  435-470  510-540 485  570-590 500-520
//   all masked but 1100 neighbours      483   428     518   460     119   100
//   all masked but 2000 neighbours       38   419      40   443     119   101
//   rounded to halves                   132    42     534    53     610   517
//   all equal                          1004  1076    1137  1033    1119  1102
#include "rows.h"

#include <algorithm>

namespace hbsjd {
namespace {

constexpr int kPairs = 256;      // candidates compared with all others
constexpr int kBinMost = 256;    // entries of one bin
constexpr double kLog2e = 1.4426950408889634;

// larger for larger logits; -0 as +0, every NaN above +infinity
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return x != x ? 0xFFFFFFFFu : k;
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t ranked(float x, int v) {
    return (uint64_t)order_of(x) << 32 | (uint32_t)~v;
}
__device__ __forceinline__ int index_of(uint64_t c) { return (int)~(uint32_t)c; }
__device__ __forceinline__ float logit_of(uint64_t c) { return value_of((uint32_t)(c >> 32)); }

// A candidate as one number: an order-preserving image of its logit above its
// complemented index. 16-bit logits have 16-bit images, and with the 14 or 15 bits
// of an index within what a workgroup holds (Held entries; no more bits than that:
// equal logits are binned by their index) the number takes 32 bits: half the LDS,
// and comparisons at full rate (K = 2000 of 16384 bf16 entries, where equal logits share bins:
// 54 us with 64 bits).
constexpr int kWhole = 32768;  // entries of a row that goes whole at most
constexpr int kPart = 16384;   // of a part
template <typename T, int Held> struct Candidate {
    using Key = uint64_t;
    static constexpr int kBins = 1024;
    __device__ __forceinline__ static Key of(float x, int v) { return ranked(x, v); }
    __device__ __forceinline__ static int index(Key c) { return index_of(c); }
    __device__ __forceinline__ static float logit(Key c) { return logit_of(c); }
    // the image with what is worth binning by
    __device__ __forceinline__ static uint32_t image(Key c) { return (uint32_t)(c >> 32); }
    __device__ __forceinline__ static uint32_t least(float x) { return order_of(x); }
    __device__ __forceinline__ static uint32_t most(float x) { return order_of(x); }
};
template <typename T, int Held> struct Candidate16 {
    using Key = uint32_t;
    static constexpr int kShift = Held <= 16384 ? 14 : 15, kLow = (1 << kShift) - 1;
    static_assert(Held <= 1 << kShift, "an index has to fit");
    static constexpr int kBins = 2048;
    __device__ __forceinline__ static uint32_t order(float x) {
        uint32_t u;
        if constexpr (std::is_same_v<T, Bf16>) u = __float_as_uint(x + 0.f) >> 16;
        else u = __builtin_bit_cast(uint16_t, (_Float16)(x + 0.f));
        return u & 0x8000u ? ~u & 0xFFFFu : u | 0x8000u;
    }
    __device__ __forceinline__ static Key of(float x, int v) { return order(x) << kShift | (kLow - v); }
    __device__ __forceinline__ static int index(Key c) { return kLow - (int)(c & kLow); }
    __device__ __forceinline__ static float logit(Key c) {
        const uint32_t k = c >> kShift, u = k & 0x8000u ? k & 0x7FFFu : ~k & 0xFFFFu;
        if constexpr (std::is_same_v<T, Bf16>) return __uint_as_float(u << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
    }
    __device__ __forceinline__ static uint32_t image(Key c) { return c; }
    __device__ __forceinline__ static uint32_t least(float x) { return order(x) << kShift; }
    __device__ __forceinline__ static uint32_t most(float x) { return order(x) << kShift | kLow; }
};
template <int Held> struct Candidate<Bf16, Held> : Candidate16<Bf16, Held> {};
template <int Held> struct Candidate<F16, Held> : Candidate16<F16, Held> {};

// room for candidates
constexpr int kFew = 1024, kMany = 4096;

// Where a row's results go. A row of logits is a whole one or a part; a join's
// row are the lists of a row's parts, whose place v holds entry map[v], and to
// whose rest the parts' rests are added.
struct TopRow {
    float* values;
    int32_t* index;
    float* rest;
    const int32_t* map;
    const float* rests;
    int n_rests;
    int first;   // of the row's entries in the whole row
    int parts;   // of a part: the row's; 0 otherwise
    // how place v is to be called: its entry, for equal logits to be ordered by
    __device__ __forceinline__ int entry(int v) const { return map ? map[v] : v; }
    __device__ __forceinline__ void put(int k, float x, int entry, int K) const {
        const int at = parts ? list_place(k, K, parts) : k;
        values[at] = x;
        index[at] = first + entry;
    }
    // What a part writes for a join. Four places in a row, one of the join's
    // vectors, take the entries of one list a quarter of it apart: then the
    // largest of each, by which the join finds its pivot, are the lists' first
    // quarters, and the row's largest entries are mostly among those.
    __device__ __forceinline__ static int list_place(int k, int K, int parts) {
        const int q = (K + 3) / 4;
        return (k % q * parts) * 4 + k / q;
    }
    __device__ __forceinline__ void pad(int K) const {
        const int k = K + threadIdx.x;
        if (parts && k < (K + 3) / 4 * 4) put(k, -INFINITY, 0x7FFFFFFF - first, K);
    }
    // the rest of this lane's part (of 64 at most)
    __device__ __forceinline__ float part_rest() const {
        return (int)(threadIdx.x & 63) < n_rests ? rests[threadIdx.x & 63] : -INFINITY;
    }
    // rest from the log of what the kernel itself left over; by whole wavefronts
    __device__ __forceinline__ void put_rest(double own, float part) const {
        if (n_rests && own == own) {
            const double m = fmax(own, (double)wave_all(part, MaxOp()));
            if (fabs(m) == INFINITY) own = m;
            else
                own = m + (double)__logf(__expf((float)(own - m)) +
                                         wave_all(__expf((float)((double)part - m)), AddOp()));
        }
        if (threadIdx.x == 0) *rest = (float)own;
    }
};

// log of sum exp((z - ref) / tau) and its reference, joined: the two may nearly
// cancel, so they are added in 64 bits (the log itself, of a number that is
// neither tiny nor above V, is fp32's: 64-bit ones cost 8% of a batch's time)
__device__ __forceinline__ double log_mass(float ref, double inv_tau, float sum) {
    return sum > 0.f ? (double)ref * inv_tau + (double)__logf(sum) : -INFINITY;
}

// the digits' way, from memory, for rows of any kind
template <int NT, typename T>
__device__ void top_by_digits(const T* z, int V, int K, double inv_tau, const TopRow& out,
                              uint64_t* kept, int* hist, float* red, int* word) {
    const int t = threadIdx.x;
    uint64_t prefix = 0;
    int need = K;   // rank of the wanted entry among those that share the prefix
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = t; i < 256; i += NT) hist[i] = 0;
        __syncthreads();
        for (int v = t; v < V; v += NT) {
            const uint64_t c = ranked(widen(z[v]), out.entry(v));
            if (shift == 56 || c >> (shift + 8) == prefix) atomicAdd(&hist[c >> shift & 255], 1);
        }
        __syncthreads();
        if (t == 0) {
            int above = 0, d = 255;
            while (d > 0 && above + hist[d] < need) above += hist[d--];
            word[0] = d;
            word[1] = above;
        }
        __syncthreads();
        prefix = prefix << 8 | word[0];
        need -= word[1];
    }
    if (t == 0) word[2] = 0;
    __syncthreads();
    float m = -INFINITY;
    for (int v = t; v < V; v += NT) {
        const float x = widen(z[v]);
        const uint64_t c = ranked(x, out.entry(v));
        if (c >= prefix) kept[atomicAdd(&word[2], 1)] = c;
        else m = fmaxf(m, x);
    }
    int n = 1;
    while (n < K) n *= 2;
    for (int i = K + t; i < n; i += NT) kept[i] = 0;
    m = block_all<NT>(m, red, MaxOp());
    float s = 0.f;
    for (int v = t; v < V; v += NT) {
        const float x = widen(z[v]);
        if (ranked(x, out.entry(v)) < prefix) s += __expf((x - m) * (float)inv_tau);
    }
    __syncthreads();
    s = block_all<NT>(s, red, AddOp());
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
    for (int k = t; k < K; k += NT) out.put(k, logit_of(kept[k]), index_of(kept[k]), K);
    if (t < 64) {
        const bool nan = kept[0] >> 32 == 0xFFFFFFFFu;
        out.put_rest(nan ? __builtin_nanf("") : fabsf(m) == INFINITY ? m : log_mass(m, inv_tau, s),
                     out.part_rest());
    }
}

// exclusive prefix sum over a wavefront's lanes, and the wavefront's total
__device__ __forceinline__ int wave_prefix(int v, int& total) {
    int s = v;
    auto step = [&](int moved) { s += moved; };
    step(__builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, s, 0x142, 0xA, 0xF, false));
    step(__builtin_amdgcn_update_dpp(0, s, 0x143, 0xC, 0xF, false));
    total = __builtin_amdgcn_readlane(s, 63);
    return s - v;
}

// keeps the compiler from holding what one pass made of the vectors (the widened
// entries of 16-bit rows, twice their registers) for the next
template <int NV> __device__ __forceinline__ void opaque(u32x4 (&x)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(x[i]));
}

template <typename T, int NT, int NV, int Cap, bool Join>
__device__ __forceinline__ void top_row(const T* z, int V, int K, double inv_tau, const TopRow& out) {
    constexpr int E = kVec<T>, N = NV * E, NW = NT / 64;
    static_assert(N >= 8, "eight groups a thread");
    using Cand = Candidate<T, NT * N>;
    using Key = typename Cand::Key;
    constexpr int kBins = Cand::kBins;
    // (the digits' way keeps up to K 64-bit numbers there)
    constexpr int kRoom = (Cap + 8) * (int)sizeof(Key), kKept = (Cap < HBSJD_TOP_MAX ? Cap : HBSJD_TOP_MAX) * 8;
    __shared__ __attribute__((aligned(16))) char room[kRoom > kKept ? kRoom : kKept];
    Key* cand = (Key*)room;
    __shared__ int bins[kBins];
    __shared__ float red[5][NW];
    __shared__ int s_count[NW];
    __shared__ int word[4];
    __shared__ float s_last;
    const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
    const float c2 = (float)(inv_tau * kLog2e);

    // The thread's first vector. A join's vectors are nearly in order: they are
    // dealt out one by one, so that every wavefront has its share of the largest.
    const int t0 = Join ? lane * NW + wv : t;
    const Span sp = Span::of(z, V);
    const u32x4* z4 = (const u32x4*)(z + sp.head);
    u32x4 x[NV];
    float xe = -INFINITY;
    if (sp.vecs > 0)
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = vec_at(z4, min(t0 + NT * i, sp.vecs - 1));
    if (t < sp.edges()) xe = widen(z[sp.edge(t, V)]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t0 + NT * i >= sp.vecs) x[i] = masked_vec<T>();
    out.pad(K);

    const float part_rest = out.part_rest();

    // ---- 1. the pivot
    float p0 = -INFINITY;
    const bool sample = NT * 8 >= 2 * K;
    if (sample) {
        float g[8];
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            float m = -INFINITY;
#pragma unroll
            for (int n = b * N / 8; n < (b + 1) * N / 8; ++n) m = fmaxf(m, vec_get<T>(x[n / E], n % E));
            g[b] = m;
        }
        int groups = 8;
#pragma unroll
        for (int h = 4; h > 0; h /= 2)
            if (!Join && groups == 2 * h && NT * h >= 2 * K) {
#pragma unroll
                for (int b = 0; b < h; ++b) g[b] = fmaxf(g[b], g[b + h]);
                groups = h;
            }
        const int want = (K + NW - 1) / NW;
        uint32_t pivot = 0;
        // the upper 24 bits will do (a lower pivot is a pivot too), or all that the
        // images of 16-bit logits have
        constexpr int kLowest = std::is_same_v<T, Bf16> ? 16 : std::is_same_v<T, F16> ? 13 : 8;
        auto descend = [&](auto n) {
            uint32_t key[decltype(n)::value];
#pragma unroll
            for (int b = 0; b < decltype(n)::value; ++b) key[b] = order_of(g[b]);
            for (int bit = 31; bit >= kLowest; --bit) {
                const uint32_t next = pivot | 1u << bit;
                int have = 0;
#pragma unroll
                for (int b = 0; b < decltype(n)::value; ++b) have += __popcll(__ballot(key[b] >= next));
                if (have >= want) pivot = next;
            }
        };
        if (groups == 1) descend(std::integral_constant<int, 1>{});
        else if (groups == 2) descend(std::integral_constant<int, 2>{});
        else if (groups == 4) descend(std::integral_constant<int, 4>{});
        else descend(std::integral_constant<int, 8>{});
        p0 = pivot > 0x007FFFFFu ? value_of(pivot) : -INFINITY;
        if (NW > 1) {
            if (lane == 0) red[0][wv] = p0;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) p0 = fminf(p0, red[0][w]);
            p0 = uniform(p0);
        }
    }
    // -infinity is nobody's candidate
    const float from = fmaxf(p0, -3.4028234663852886e38f);
    const float ref = p0 == -INFINITY ? 0.f : p0, ref2 = -ref * c2;

    // ---- 2. candidates, and the mass below them
    opaque(x);
    int mine = 0;
    float below = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            const float y = vec_get<T>(x[i], q);
            const bool in = y >= from;
            const float e = __builtin_amdgcn_exp2f(fmaf(y, c2, ref2));
            mine += in;
            below += in ? 0.f : e;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    {
        const bool in = xe >= from;
        mine += in;
        below += in ? 0.f : __builtin_amdgcn_exp2f(fmaf(xe, c2, ref2));
    }
    int total;
    int slot = wave_prefix(mine, total);
    below = wave_all(below, AddOp());
    if (lane == 0) {
        s_count[wv] = total;
        red[1][wv] = below;
    }
    __syncthreads();
    int C = 0;
    below = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wv) slot += s_count[w];
        C += s_count[w];
        below += red[1][w];
    }
    C = uniform(C);
    below = uniform(below);
    if (C > Cap || (Join && C < K) || below != below || fabsf(ref2) == INFINITY) {
        __syncthreads();
        top_by_digits<NT>(z, V, K, inv_tau, out, (uint64_t*)room, bins, red[0], word);
        return;
    }
    opaque(x);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            const float y = vec_get<T>(x[i], q);
            if (y >= from) cand[slot++] = Cand::of(y, out.entry(sp.head + (t0 + NT * i) * E + q));
        }
    }
    if (xe >= from) cand[slot++] = Cand::of(xe, out.entry(sp.edge(t, V)));

    // fewer than K entries above -infinity: then the first of those at it
    for (int base = 0, filled = C; __builtin_expect(filled < K, 0) && base < V; base += NT) {
        __syncthreads();
        const int v = base + t;
        const uint64_t at = __ballot(v < V && widen(z[min(v, V - 1)]) == -INFINITY);
        if (lane == 0) s_count[wv] = __popcll(at);
        __syncthreads();
        int k = filled + __popcll(at & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wv) k += s_count[w];
            filled += s_count[w];
        }
        if ((at >> lane & 1) && k < K) out.put(k, -INFINITY, out.entry(v), K);
    }

    // ---- 3. places
    constexpr int M = Cap / NT;   // candidates a thread looks after
    static_assert(M >= 1 && M * NT == Cap, "");
    Key me[M];
    int place[M];                 // K where it is known only not to be lower
    if (C <= kPairs) {
        // zeros, below every candidate, to a whole number of steps
        if (t < 8) cand[C + t] = 0;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < M; ++n) {
            const int c = t + NT * n;
            me[n] = 0;
            place[n] = K;
            if (n * NT >= kPairs || c >= C) continue;
            me[n] = cand[c];
            int p = 0;
            for (int j = 0; j < C; j += 8)
#pragma unroll
                for (int i = 0; i < 8; i += 16 / (int)sizeof(Key)) {
                    typedef Key Vec __attribute__((ext_vector_type(16 / sizeof(Key))));
                    const Vec other = *(const Vec*)(cand + j + i);
#pragma unroll
                    for (int q = 0; q < 16 / (int)sizeof(Key); ++q) p += other[q] > me[n];
                }
            place[n] = p;
            if (p < K) out.put(p, Cand::logit(me[n]), Cand::index(me[n]), K);
            if (p == K - 1) s_last = Cand::logit(me[n]);
        }
        __syncthreads();
    } else {
        for (int i = t; i < kBins; i += NT) bins[i] = 0;
        if (t == 0) word[2] = 0;   // most entries in a bin
        __syncthreads();
        float ends[2] = {-INFINITY, -INFINITY};   // of the candidates: least, negated, and largest
#pragma unroll
        for (int n = 0; n < M; ++n) {
            const int c = t + NT * n;
            me[n] = c < C ? cand[c] : 0;
            if (c < C) {
                ends[0] = fmaxf(ends[0], -Cand::logit(me[n]));
                ends[1] = fmaxf(ends[1], Cand::logit(me[n]));
            }
        }
        block_all<NT, 2>(ends, &red[2], MaxOp());
        const float lo = -ends[0], hi = ends[1];
        const uint32_t least = Cand::least(lo), most = Cand::most(hi);
        // Bins on the images where all candidates have one sign: even an outlier
        // among them only costs some octaves. Across zero, where the images of
        // small numbers would take most bins, on the logits themselves.
        const bool images = lo > 0.f || hi < 0.f || !(hi - lo < INFINITY);
        constexpr int kBits = 31 - __builtin_clz(kBins);
        const int shift = max(32 - kBits - __clz((int)(most - least)), 0);
        const float scale = (kBins - 1) / (hi - lo);
        auto bin_of = [&](Key c) {   // from the largest down
            const int b = images ? (int)((Cand::image(c) - least) >> shift)
                                 : (int)((Cand::logit(c) - lo) * scale);
            return kBins - 1 - min(max(b, 0), kBins - 1);
        };
#pragma unroll
        for (int n = 0; n < M; ++n)
            if (t + NT * n < C) atomicAdd(&bins[bin_of(me[n])], 1);
        __syncthreads();
        // exclusive prefix sums: thread t has its consecutive bins
        constexpr int B = kBins / NT;
        int own[B], sum = 0, big = 0;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            own[b] = bins[t * B + b];
            sum += own[b];
            big = max(big, own[b]);
        }
        int all;
        int start = wave_prefix(sum, all);
        if (lane == 0) s_count[wv] = all;
        if (big > kBinMost) word[2] = 1;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w)
            if (w < wv) start += s_count[w];
        if (uniform(word[2])) {
            __syncthreads();
            top_by_digits<NT>(z, V, K, inv_tau, out, (uint64_t*)room, bins, red[0], word);
            return;
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            bins[t * B + b] = start;
            start += own[b];
        }
        __syncthreads();
        // the candidates by bin, in the list's place; afterwards bins[b] is where
        // bin b + 1 starts
#pragma unroll
        for (int n = 0; n < M; ++n)
            if (t + NT * n < C) cand[atomicAdd(&bins[bin_of(me[n])], 1)] = me[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < M; ++n) {
            place[n] = K;
            if (t + NT * n >= C) continue;
            const int b = bin_of(me[n]), first = b ? bins[b - 1] : 0, end = bins[b];
            if (first >= K) continue;
            int p = first;
            for (int j = first; j < end; j += 4)
#pragma unroll
                for (int i = 0; i < 4; ++i) p += (j + i < end) & (cand[j + i] > me[n]);
            place[n] = p;
            if (p == K - 1) s_last = Cand::logit(me[n]);
        }
        __syncthreads();
        // in order, for whole lines to be written
#pragma unroll
        for (int n = 0; n < M; ++n)
            if (place[n] < K) cand[place[n]] = me[n];
        __syncthreads();
        for (int k = t; k < min(K, C); k += NT) out.put(k, Cand::logit(cand[k]), Cand::index(cand[k]), K);
    }
    // ---- the mass of the others: below the pivot, and the candidates left over
    const float last = uniform(s_last);
    const uint32_t last_image = order_of(last);
    if (last == INFINITY && C > K) {
        __syncthreads();
        top_by_digits<NT>(z, V, K, inv_tau, out, (uint64_t*)room, bins, red[0], word);
        return;
    }
    float over = 0.f;
    if (C > K) {
#pragma unroll
        for (int n = 0; n < M; ++n)
            if (t + NT * n < C && place[n] >= K)
                over += __builtin_amdgcn_exp2f((Cand::logit(me[n]) - last) * c2);
        over = block_all<NT>(over, red[2], AddOp());
    }
    // A sum far below its reference, where the exponents' roundings are coarse:
    // again, relative to the largest term. (With candidates left over the mass
    // below the pivot is at most V times the least of them, so only without any
    // does it matter.)
    float ref_below = ref, ref_over = last;
    if (C > K ? over < 0x1p-6f : below < 0x1p-6f) {
        const uint64_t bound = C > K ? (uint64_t)last_image << 32 : (uint64_t)order_of(from) << 32;
        float m = -INFINITY, s = 0.f;
        for (int v = t; v < V; v += NT) {
            const float y = widen(z[v]);
            m = fmaxf(m, ranked(y, 0) < bound ? y : -INFINITY);
        }
        __syncthreads();
        m = block_all<NT>(m, red[0], MaxOp());
        for (int v = t; v < V; v += NT) {
            const float y = widen(z[v]);
            s += ranked(y, 0) < bound && m > -INFINITY ? __builtin_amdgcn_exp2f((y - m) * c2) : 0.f;
        }
        s = block_all<NT>(s, red[4], AddOp());
        ref_below = m;
        below = s;
        over = 0.f;
    }
    if (t < 64) {
        const double a = log_mass(ref_below, inv_tau, below), b = log_mass(ref_over, inv_tau, over);
        const double m = fmax(a, b);
        const float sum = __expf((float)(a - m)) + __expf((float)(b - m));
        out.put_rest(m == -INFINITY ? m : m + (double)__logf(sum), part_rest);
    }
}

template <typename T, int NT, int NV, int Cap>
__global__ __launch_bounds__(NT) void k_top(TopArgs a, int64_t r0) {
    const int64_t r = r0 + blockIdx.x;
    const TopRow out{a.values + r * a.K, a.index + r * a.K, a.rest + r, nullptr, nullptr, 0, 0, 0};
    top_row<T, NT, NV, Cap, false>((const T*)a.logits + r * a.ld, a.V, a.K, a.inv_tau, out);
}

// Long rows: every part's K largest and the mass of its others go to the
// workspace, and the row's are the K largest of the parts'.
struct PartsArgs {
    int parts, len;
    float* values;   // [rows of the slab][list_room(K) * parts]
    int32_t* index;
    float* rest;     // [rows of the slab][parts]
};
__host__ __device__ inline int list_room(int K) { return (K + 3) / 4 * 4; }

template <typename T, int NT, int NV, int Cap>
__global__ __launch_bounds__(NT) void k_top_part(TopArgs a, PartsArgs p, int64_t r0) {
    const int row = blockIdx.x / p.parts, c = blockIdx.x - row * p.parts;
    const int first = c * p.len;
    const int64_t at = (int64_t)row * list_room(a.K) * p.parts + 4 * c;
    const TopRow out{p.values + at, p.index + at, p.rest + blockIdx.x, nullptr, nullptr, 0, first, p.parts};
    top_row<T, NT, NV, Cap, false>((const T*)a.logits + (r0 + row) * a.ld + first,
                                   min(p.len, a.V - first), a.K, a.inv_tau, out);
}

template <int NT, int NV, int Cap>
__global__ __launch_bounds__(NT) void k_top_join(TopArgs a, PartsArgs p, int64_t r0) {
    const int64_t row = blockIdx.x, r = r0 + row, n = (int64_t)list_room(a.K) * p.parts;
    const TopRow out{a.values + r * a.K,     a.index + r * a.K, a.rest + r, p.index + row * n,
                     p.rest + row * p.parts, p.parts,           0,          0};
    top_row<float, NT, NV, Cap, true>(p.values + row * n, (int)n, a.K, a.inv_tau, out);
}

// How a call runs: whole rows, or in parts with workspace for `slab` rows.
struct Plan {
    int parts = 0, len = 0;
    int64_t slab = 0;
};
inline size_t part_row_bytes(const Plan& p, int K) { return (size_t)p.parts * (8 * (size_t)list_room(K) + 4); }

// Rows of more than kWhole entries go in parts, and many fp32 ones of more than
// kPart (2000 of 25000, K 64: 74 us, whole 87; 100 of 30000: 20 and 13); where rows are few,
// in more and smaller ones, as long as the join stays the smaller work.
Plan plan_of(int64_t rows, int V, int K, int32_t elem) {
    Plan p;
    if (V <= kPart || (V <= kWhole && (elem != HBSJD_ELEM_F32 || rows <= 512))) return p;
    p.parts = (V + kPart - 1) / kPart;
    while (rows * p.parts < 256 && V / (2 * p.parts) >= std::max(4096, 8 * K) && 2 * p.parts * K <= 8192)
        p.parts *= 2;
    p.len = ((V + p.parts - 1) / p.parts + 7) / 8 * 8;
    p.parts = (V + p.len - 1) / p.len;
    p.slab = std::max<int64_t>(1, (64 << 20) / (int64_t)part_row_bytes(p, K));
    p.slab = std::min(p.slab, rows);
    return p;
}

// f(threads, vectors a thread, room for candidates) for the smallest workgroup of
// at least `least` threads that holds the row. Up to K = 256 the maxima of 64
// threads leave few enough candidates; a larger K takes workgroups with at least
// 2 K groups, unless all of the row's entries may be candidates.
template <typename T, typename F> void by_size(int V, int K, int least, F f) {
    using std::integral_constant;
    auto fits = [&](auto nt, auto nv) {
        constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
        return NT >= least && V <= NT * NV * kVec<T> && (NT * 8 >= 2 * K || V <= (NT == 64 ? kFew : kMany));
    };
#define FITS(nt, nv) fits(integral_constant<int, nt>{}, integral_constant<int, nv>{})
#define CALL(nt, nv, cap) \
    f(integral_constant<int, nt>{}, integral_constant<int, nv>{}, integral_constant<int, cap>{})
    const bool few = K <= 256 || V <= kFew;
    if (FITS(64, 2)) CALL(64, 2, kFew);
    else if (FITS(64, 8)) CALL(64, 8, kFew);
    else if (FITS(256, 4)) { if (few) CALL(256, 4, kFew); else CALL(256, 4, kMany); }
    else if (FITS(512, 4)) { if (few) CALL(512, 4, kFew); else CALL(512, 4, kMany); }
    else if (FITS(512, 8)) { if (few) CALL(512, 8, kFew); else CALL(512, 8, kMany); }
    else if constexpr (sizeof(T) == 4) CALL(1024, 8, kMany);
#undef FITS
#undef CALL
}

template <typename T> void go(const TopArgs& a, void* ws, hipStream_t s) {
    const Plan plan = plan_of(a.rows, a.V, a.K, a.elem);
    if (!plan.parts) {
        by_size<T>(a.V, a.K, 64, [&](auto nt, auto nv, auto cap) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value, Cap = decltype(cap)::value;
            by_slabs(a.rows, [&](int64_t r0, dim3 grid) {
                hipLaunchKernelGGL((k_top<T, NT, NV, Cap>), grid, dim3(NT), 0, s, a, r0);
            });
        });
        return;
    }
    PartsArgs p{plan.parts, plan.len, (float*)ws, nullptr, nullptr};
    const int64_t lists = plan.slab * plan.parts * list_room(a.K);
    p.index = (int32_t*)(p.values + lists);
    p.rest = (float*)(p.index + lists);
    for (int64_t r0 = 0; r0 < a.rows; r0 += plan.slab) {
        const int64_t n = std::min(plan.slab, a.rows - r0);
        by_size<T>(p.len, a.K, 256, [&](auto nt, auto nv, auto cap) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value, Cap = decltype(cap)::value;
            if constexpr (NT >= 256 && NT * NV * kVec<T> <= kPart)
                hipLaunchKernelGGL((k_top_part<T, NT, NV, Cap>), dim3((unsigned)(n * p.parts)), dim3(NT),
                                   0, s, a, p, r0);
        });
        by_size<float>(p.parts * list_room(a.K), a.K, 256, [&](auto nt, auto nv, auto cap) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value, Cap = decltype(cap)::value;
            if constexpr (NT >= 256)
                hipLaunchKernelGGL((k_top_join<NT, NV, Cap>), dim3((unsigned)n), dim3(NT), 0, s, a, p, r0);
        });
    }
}

}  // namespace

size_t top_logits_workspace(int64_t rows, int V, int K, int32_t elem) {
    const Plan p = plan_of(rows, V, K, elem);
    return p.parts ? p.slab * part_row_bytes(p, K) : 0;
}

void top_logits(const TopArgs& a, void* workspace, hipStream_t s) {
    if (a.elem == HBSJD_ELEM_F32) go<float>(a, workspace, s);
    else if (a.elem == HBSJD_ELEM_BF16) go<Bf16>(a, workspace, s);
    else go<F16>(a, workspace, s);
}

}  // namespace hbsjd
