// nvq_sample: the next token of each row of logits.
//
// Every question is one of the descending order of a row's tokens: which token brings the count to top_k, the sum of
// the weights to top_p, to u times the kept sum.  It is answered without sorting the row, in two launches (or in one, rows that a
// workgroup takes alone):
//   1. Workgroups share a row's logits, a part each: the part's largest, and relative to it a histogram of counts and
//      weights over bins of 1 / 32 in the logit.  The one that arrives last adds the parts' bins up
//      and sees in which bins the answers can lie: the weight of a bin that a border falls into is known, which of its
//      tokens are in is not, so the later borders are ranges of a bin or a few.
//   2. The tokens of those bins are collected (a few hundred of 128256), and the workgroup that arrives last sorts
//      them by logit and index and answers every question to the token.
// Weights are 64-bit fixed point relative to the largest, so that sums do not depend on their order.  A row whose bins
// hold too many tokens (nearly equal logits), or whose logits are out of the bins' range, is looked at by one workgroup
// alone, eleven bits of the sort words after the other (choose_slowly, in the last launch).
//
// Neither bytes nor operations bound a few rows but the chain of trips to memory and through LDS: one row of 128256 in 20.5 us (14
// and 6.5 in the kernels: logits 1.5, bins 2.6, the parts' arrival 1, their bins 3.5 (196 KB through one compute unit), sums
// 0.9, search 1.4; logits and list 3.5, the choice 1.5), five of 32003 in 16 bits 19.8, 32 of 128256 29.7 (16.4 MB).
#include <type_traits>

#include "mfma_act.h"

namespace nvq {

namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kPoint = 43;  // bits after the point: 2^20 weights of at most 1 stay below 2^63
constexpr double kOne = (double)(1ull << kPoint);

struct SampleArgs {
    const void *logits;
    int64_t ld;
    int M, V;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *ids;
    int parts, part;  // workgroups to a row, logits of each
    uint32_t *arrived;  // workspace
    struct RowState *rows;
    struct PartHead *heads;
    struct PartBins *bins;
};

// Words in the order of the logits; minus infinity and NaN: 0, both zeros alike.
__device__ __forceinline__ uint32_t sort_word(float f) {
    if (!(f > -INFINITY)) return 0u;
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_sort_word(uint32_t w) {
    return __uint_as_float(w & 0x80000000u ? w & 0x7fffffffu : ~w);
}

// (The type is a template's: a branch on it at every load made the compiler wait for each before the next.)
template <bool BF16>
struct Row {
    typedef std::conditional_t<BF16, uint16_t, float> Value;
    const Value *at;
    int V;
    __device__ Row(const SampleArgs &a, int m) : at(static_cast<const Value *>(a.logits) + m * a.ld), V(a.V) {}
    __device__ float logit(int i) const {
        const Value v = *as_global<Value>(at + i);
        if constexpr (BF16)
            return bf16_bits_to_float(v);
        else
            return v;
    }
    __device__ uint32_t word(int i) const { return sort_word(logit(i)); }
    // Logits b + tid + 1024 j, those past `end` minus infinity (the first is loaded there: no load behind a branch).
    __device__ void load(int b, int end, float (&to)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = b + j * 1024 + (int)threadIdx.x;
            to[j] = logit(i < end ? i : 0);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j] = b + j * 1024 + (int)threadIdx.x < end ? to[j] : -INFINITY;
    }
};

// exp(x) as fixed point, x = (logit - top) / temperature <= 0: 2^(k / 64), its fraction from a table, times the
// exponential series of the rest, |rest| <= ln 2 / 128, to six terms (the next is 4e-17 of the sum; without the table it
// takes thirteen, and the weights of a row of 128256 in sixteen parts 4.4 us instead of 3.1).
constexpr int kRoots = 64;
__constant__ const double kRoot[kRoots] = {
    1.0, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284, 1.0442737824274138, 1.0556451783605572,
    1.0671404006768237, 1.0787607977571199, 1.0905077326652577, 1.102382583307841, 1.1143867425958924, 1.1265216186082418,
    1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812, 1.189207115002721, 1.202156731452703,
    1.215247359980469, 1.22848053610687, 1.241857812073484, 1.255380757024691, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.339667524053303, 1.3542555469368927, 1.3690024229745905,
    1.383909881963832, 1.3989796725383112, 1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647,
    1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384, 1.5422108254079407, 1.559004400237837,
    1.5759808451078865, 1.593142151342267, 1.6104903319492543, 1.6280274218573478, 1.645755478153965, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.718619298122478, 1.7373338352737062, 1.7562521603732995, 1.7753764925265212,
    1.7947090750031072, 1.8142521755003989, 1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656,
    1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.978456026387951};
struct Weights {
    double top, rate;  // 64 log2(e) / temperature
    const double *root;  // kRoot, or a copy in LDS
    __device__ Weights(float most, float temperature, const double *roots)
        : top(most), rate(kRoots * 1.4426950408889634074 / (double)temperature), root(roots) {}
    __device__ uint64_t of(float logit) const {
        double t = ((double)logit - top) * rate;
        t = t > -64.0 * kRoots ? t : -64.0 * kRoots;  // (nothing is left of the weight long before)
        const double k = rint(t), x = (t - k) * (0.69314718055994530942 / kRoots);
        const int i = (int)k;
        double e = 1.0 / 120;
        e = fma(e, x, 1.0 / 24);
        e = fma(e, x, 1.0 / 6);
        e = fma(e, x, 0.5);
        e = fma(e, x, 1.0);
        e = fma(e, x, 1.0) * root[i & (kRoots - 1)];
        // e times 2^(k / 64 + kPoint), below 2^44; beside 2^52 its whole part is the low bits
        const double scaled = __longlong_as_double(__double_as_longlong(e) + ((int64_t)((i >> 6) + kPoint) << 52));
        return (uint64_t)__double_as_longlong(scaled + 4503599627370496.0) & 0xfffffffffffffull;
    }
    __device__ uint64_t of_word(uint32_t word) const { return of(of_sort_word(word)); }
};

// What choose_slowly needs of LDS.
constexpr int kDigits = 2048;  // of the sort words, eleven bits at a time (ten at last)
struct Shared {
    unsigned long long mass[kDigits];
    uint32_t count[kDigits];
    unsigned long long wave[kSampleWaves];
    unsigned long long before;
    uint32_t bin;
};

// ---- over a wave and over the workgroup, by moves between lanes (shuffles go through LDS: 16 waves of six 64-bit steps
// and sixteen reads each took about 1.2 us where these take 0.5)
struct MaxU32 {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct MinU32 {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a < b ? a : b; }
};
template <int LANES, typename OP>  // 16 or 64
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, OP op) {
    if constexpr (LANES == 64) {
        v = with_lane_xor<32>(v, op);
        v = with_lane_xor<16>(v, op);
    }
    v = with_lane_xor<8>(v, op);
    v = with_lane_xor<4>(v, op);
    v = with_lane_xor<2>(v, op);
    return with_lane_xor<1>(v, op);
}
// Sum over the threads before this one; *all: over all.  By the first W waves.
template <int W, typename T>
__device__ __forceinline__ T scan_block(T *wave, T v, T *all) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T sum = scan_wave(v);
    __syncthreads();
    if (lane == 63) wave[w] = sum;
    __syncthreads();
    const T waves = scan_row(wave[(lane & 15) < W ? lane & 15 : W - 1]);
    *all = of_lane(waves, W - 1);
    return (w ? of_lane(waves, w ? w - 1 : 0) : 0) + sum - v;
}
__device__ uint64_t sum_block(unsigned long long *wave, uint64_t v) {
    unsigned long long all;
    scan_block<kSampleWaves>(wave, (unsigned long long)v, &all);
    return all;
}

// The first token of a row or a part of it: sort word and index.  Of a wave, or of sixteen lanes that lie side by side.
struct First {
    uint32_t word, index;
};
template <int LANES>
__device__ __forceinline__ First first_of(First f) {
    const uint32_t top = over_lanes<LANES>(f.word, MaxU32());
    return First{top, over_lanes<LANES>(f.word == top ? f.index : ~0u, MinU32())};
}

// The token at which the running count (or sum of weights) of the descending order first exceeds x: its word, and the
// count (sum) before all tokens of that word.  x is below the row's whole count (sum).
template <bool MASS, typename ROW>
__device__ void find(Shared &s, const ROW &row, const Weights &w, uint64_t x, uint32_t *word, uint64_t *before) {
    uint32_t prefix = 0;
    uint64_t base = 0;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 1 ? 21 : 10;
        const uint32_t digits = pass == 2 ? kDigits / 2 : kDigits;
        __syncthreads();
        for (int i = threadIdx.x; i < kDigits; i += kSampleThreads) {
            s.count[i] = 0;
            s.mass[i] = 0;
        }
        __syncthreads();
        for (int b = 0; b < row.V; b += 8 * kSampleThreads) {
            float l[8];
            row.load(b, row.V, l);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t v = sort_word(l[j]);
                if (v == 0 || (pass > 0 && v >> above != prefix)) continue;
                if (MASS)
                    atomicAdd(&s.mass[v >> shift & (digits - 1)], (unsigned long long)w.of(l[j]));
                else
                    atomicAdd(&s.count[v >> shift & (digits - 1)], 1u);
            }
        }
        __syncthreads();
        // Two digits a thread, in descending order.
        const uint32_t high = kDigits - 1 - 2 * threadIdx.x, low = high - 1;
        const unsigned long long a = MASS ? s.mass[high] : s.count[high], b = MASS ? s.mass[low] : s.count[low];
        unsigned long long all;
        const uint64_t at = base + scan_block<kSampleWaves>(s.wave, a + b, &all);
        if (x >= at && x < at + a + b) {  // (one thread)
            s.bin = x < at + a ? high : low;
            s.before = x < at + a ? at : at + a;
        }
        __syncthreads();
        prefix = prefix << (pass == 2 ? 10 : 11) | s.bin;
        base = s.before;
    }
    *word = prefix;
    *before = base;
}

// The n-th token (from 0, by index) of a word; -1 if there are fewer.
template <typename ROW>
__device__ int nth_of_word(Shared &s, const ROW &row, uint32_t word, uint64_t n) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int part = (row.V + kSampleThreads - 1) / kSampleThreads * 64;  // of a wave, in one piece
    const int i0 = w * part, i1 = i0 + part < row.V ? i0 + part : row.V;
    uint64_t mine = 0;
    for (int i = i0; i < i1; i += 64) mine += __popcll(__ballot(i + lane < i1 && row.word(i + lane) == word));
    __syncthreads();
    if (lane == 0) s.wave[w] = mine;
    if (threadIdx.x == 0) s.bin = ~0u;
    __syncthreads();
    uint64_t before = 0;
    for (int i = 0; i < w; ++i) before += s.wave[i];
    if (n >= before && n < before + mine) {  // (one wave)
        uint64_t seen = before;
        for (int i = i0; i < i1; i += 64) {
            const uint64_t hits = __ballot(i + lane < i1 && row.word(i + lane) == word);
            const uint64_t c = (uint64_t)__popcll(hits);
            if (n < seen + c) {
                const bool me = (hits >> lane & 1) && (uint64_t)__popcll(hits & ((1ull << lane) - 1)) == n - seen;
                if (me) s.bin = (uint32_t)(i + lane);
                break;
            }
            seen += c;
        }
    }
    __syncthreads();
    return (int)s.bin;
}

// What a row asks for.
struct Ask {
    float temperature, top_p, min_p, u;
    int top_k;
};
// (What is not given is read from u instead, so that no load stands behind a branch.)
__device__ __forceinline__ Ask ask_of(const SampleArgs &a, int m) {
    const float t = (a.temperature ? a.temperature : a.u)[m], p = (a.top_p ? a.top_p : a.u)[m], q = (a.min_p ? a.min_p : a.u)[m];
    const int k = (a.top_k ? a.top_k : reinterpret_cast<const int32_t *>(a.u))[m];
    return Ask{a.temperature ? t : 1.0f, a.top_p ? p : 1.0f, a.min_p ? q : 0.0f, a.u[m], a.top_k ? k : 0};
}
// Where in a kept sum the random number points.
__device__ __forceinline__ uint64_t point_of(float u, uint64_t kept) {
    const uint64_t x = !(u > 0.0f) ? 0 : u >= 1.0f ? kept - 1 : (uint64_t)((double)u * (double)kept);
    return x < kept ? x : kept - 1;
}
// The sum that top_p asks for, at least 1 and at most all.
__device__ __forceinline__ uint64_t reach_of(float top_p, uint64_t all) {
    const double share = top_p > 0.0f ? ceil((double)top_p * (double)all) : 0.0;
    return share < 1.0 ? 1 : share < (double)all ? (uint64_t)share : all;
}

// f of every logit of a row, by the workgroup.
template <typename ROW, typename F>
__device__ void over_row(const ROW &row, F f) {
    for (int b = 0; b < row.V; b += 8 * kSampleThreads) {
        float l[8];
        row.load(b, row.V, l);
#pragma unroll
        for (int j = 0; j < 8; ++j) f(l[j]);
    }
}

// The answer for a row of n tokens to choose from, by one workgroup and any logits.  (128256 logits from which no bin is left out: 320 us.)
template <typename ROW>
__device__ int choose_slowly(Shared &s, const ROW &row, const Ask &k, float most, uint64_t n) {
    const Weights w(most, k.temperature, kRoot);
    uint32_t word;
    uint64_t before, kept;
    if (k.top_k > 0 && (uint64_t)k.top_k < n) {
        find<false>(s, row, w, (uint64_t)k.top_k - 1, &word, &before);
        uint64_t above = 0;
        over_row(row, [&](float l) { above += sort_word(l) > word ? w.of(l) : 0; });
        kept = sum_block(s.wave, above) + ((uint64_t)k.top_k - before) * w.of_word(word);
    } else {
        uint64_t all = 0;
        over_row(row, [&](float l) { all += sort_word(l) ? w.of(l) : 0; });
        kept = sum_block(s.wave, all);
    }
    if (!(k.top_p >= 1.0f)) {
        const uint64_t reach = reach_of(k.top_p, kept);
        find<true>(s, row, w, reach - 1, &word, &before);
        const uint64_t each = w.of_word(word);
        kept = before + (reach - before + each - 1) / each * each;
    }
    if (k.min_p > 0.0f) {
        uint64_t enough = 0;
        over_row(row, [&](float l) {
            const uint64_t x = sort_word(l) ? w.of(l) : 0;
            enough += (double)x >= (double)k.min_p * kOne ? x : 0;
        });
        enough = sum_block(s.wave, enough);
        kept = enough < kept ? enough : kept;
    }
    kept = kept < 1ull << kPoint ? 1ull << kPoint : kept;  // (the first token's weight is 1)
    const uint64_t x = point_of(k.u, kept);
    find<true>(s, row, w, x, &word, &before);
    return nth_of_word(s, row, word, (x - before) / w.of_word(word));
}

// ---- bins
constexpr int kBins = kSampleThreads;   // the last one: everything below the others
constexpr int kBlock = 8 * kSampleThreads;  // logits that a workgroup has in flight together
constexpr int kList = 4096;             // tokens that can be collected
constexpr int kMostParts = 32;
constexpr float kSteps = 32.0f;         // bins to a unit of the logit
constexpr float kFar = 16777216.0f;     // bin numbers are whole floats up to here
static_assert(NVQ_SAMPLE_CLEAR_BYTES >= 4 * NVQ_SAMPLE_MAX_M, "a counter per row");

// Bins of a row: number floor(32 logit), and from the largest one down the place among kBins.  The width does not go by the
// temperature: a bin has to hold few tokens, whatever their weights (bins of a thirty-second of a temperature of 0.1 reached
// 3.2 below the largest, and top_k = 50 of 128256 went behind them, 640 us instead of 20).
struct Grid {
    float top;  // the largest logit's number
    __device__ static float number(float logit) { return fminf(fmaxf(floorf(logit * kSteps), -kFar), kFar); }
    __device__ int bin(float logit) const { return (int)fminf(fmaxf(top - number(logit), 0.0f), (float)(kBins - 1)); }
};

// Of a part: its first token, and its bins, each at its number modulo kBins, which is the same place for every part.
struct PartHead {
    unsigned long long first;  // sort word (0: none) and index
};
struct PartBins {
    double mass[kBins];  // relative to the part's largest
    uint32_t count[kBins];
};
// What the second launch has to know of a row.
struct RowState {
    uint32_t gather;   // 0: the row has its answer, 1: in these bins, 2: they do not serve
    uint32_t listed, arrived;
    float top, most;
    int lo[4], hi[4];  // bins whose tokens are collected: ranges in ascending order that share no bin
    unsigned long long all;  // of the weights
    uint32_t count;
    int cut;           // min_p: bins before have the weight, those from cut + 3 on have not
    unsigned long long before[kBins];  // weights of the bins before
    uint32_t ranked[kBins + 1];        // tokens of the bins before
    unsigned long long list[kList];
};

__device__ __forceinline__ void put64(unsigned long long *p, uint64_t v) {
    __hip_atomic_store(p, (unsigned long long)v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get64(const unsigned long long *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put32(uint32_t *p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t get32(const uint32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Tokens in ranges of bins, of the bins before b; lo and hi: ranges in ascending order that share no bin.
__device__ __forceinline__ uint32_t listed_before(const int *lo, const int *hi, const uint32_t *ranked, int b) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int end = hi[i] + 1 < b ? hi[i] + 1 : b;
        if (end > lo[i]) n += ranked[end] - ranked[lo[i]];
    }
    return n;
}

__device__ __forceinline__ bool listed_bin(const int (&lo)[4], const int (&hi)[4], int bin) {
    bool is = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) is |= bin >= lo[i] && bin <= hi[i];
    return is;
}

// Where a row's answers can lie, from the sums before its bins (before[kBins], ranked[kBins]: all), by one wave.
struct Search {
    int lo[4], hi[4], cut;  // bins
};
__device__ Search search(const Ask &k, const Grid &grid, float most, const unsigned long long *before, const uint32_t *ranked) {
    const int lane = threadIdx.x & 63;
    constexpr int kSkip = kBins / 64;
    // The first bin with which what is counted reaches x, or the last one: the lane's sixteen bins, then the bin of those.
    auto reached = [&](auto x, auto upto, const auto *counted) {
        const uint64_t some = __ballot(upto >= x);
        const int b0 = some ? kSkip * __builtin_ctzll(some) : kBins - kSkip;
        const uint64_t any = __ballot(lane < kSkip && (decltype(upto))counted[b0 + 1 + (lane & (kSkip - 1))] >= x);
        return any ? b0 + __builtin_ctzll(any) : kBins - 1;
    };
    const double upto = (double)before[kSkip * lane + kSkip];
    const uint32_t ranks = ranked[kSkip * lane + kSkip];
    auto reaching = [&](double x) { return reached(x, upto, before); };
    // Bounds of the sums are a little wide: a bin's weight has been rounded otherwise than its tokens' (by less than two units
    // a token, so by 2^13 for the kList that can be listed), and a sum that does not end in the first token is of 2^kPoint or more.
    static_assert(2 * kList <= 1 << (kPoint - 30), "room for their rounding");
    const double wide = 1.0 + 0x1p-30, all = (double)before[kBins];
    double least = all, greatest = all;
    Search r;
    auto bounds = [&](int i) {  // of a kept sum that ends in these bins
        least = fmin(least, (double)before[r.lo[i]]);
        greatest = fmin(greatest, (double)before[r.hi[i] + 1]);
    };
    for (int i = 0; i < 4; ++i) {
        r.lo[i] = kBins;
        r.hi[i] = -1;
    }
    r.cut = 0;
    // Tokens of the last bin do not matter where they weigh nothing (a mask of the lowest number on most of a row).
    const int end = before[kBins] > before[kBins - 1] ? kBins - 1 : kBins - 2;
    if (k.top_k > 0 && (uint32_t)k.top_k < ranked[kBins]) {
        const int b = reached((uint32_t)k.top_k, ranks, ranked);
        if (b <= end) {
            r.lo[0] = r.hi[0] = b;
            bounds(0);
        }
    }
    if (!(k.top_p >= 1.0f)) {
        const double p = k.top_p > 0.0f ? (double)k.top_p : 0.0;
        r.lo[1] = reaching(fmax(p * least / wide, 1.0));
        r.hi[1] = reaching(fmin(fmax(p * greatest * wide + 2.0, 1.0), all));
        r.hi[1] = r.hi[1] > r.lo[1] ? r.hi[1] : r.lo[1];
        bounds(1);
    }
    if (k.min_p > 0.0f) {
        const double at = (double)most + (double)k.temperature * log((double)k.min_p);
        const int cut = grid.bin((float)at);  // (its rounding moves it to a neighbouring bin at most)
        r.cut = r.lo[2] = cut > 0 ? cut - 1 : 0;
        r.hi[2] = r.cut + 2 < end ? r.cut + 2 : end;
        bounds(2);
    }
    least = fmax(least, kOne);
    greatest = fmax(greatest, kOne);
    const double u = k.u > 0.0f ? (k.u < 1.0f ? (double)k.u : 1.0) : 0.0;
    r.lo[3] = reaching(fmax(u * least / wide - 2.0, 1.0));
    r.hi[3] = reaching(fmin(u * greatest * wide + 2.0, all));
    r.hi[3] = r.hi[3] > r.lo[3] ? r.hi[3] : r.lo[3];
    // in ascending order, ranges that meet as one (the other empty, behind the last bin)
#pragma unroll
    for (int pass = 0; pass < 3; ++pass)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (r.lo[i] <= r.lo[i + 1]) continue;
            const int l = r.lo[i], h = r.hi[i];
            r.lo[i] = r.lo[i + 1];
            r.hi[i] = r.hi[i + 1];
            r.lo[i + 1] = l;
            r.hi[i + 1] = h;
        }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (r.lo[i + 1] <= r.hi[i]) {  // the second becomes both, the first empty where it stands
            r.hi[i + 1] = r.hi[i] > r.hi[i + 1] ? r.hi[i] : r.hi[i + 1];
            r.lo[i + 1] = r.lo[i];
            r.hi[i] = r.lo[i] - 1;
        }
    return r;
}

// A workgroup's part of a row: logits [*i0, *i1).
__device__ __forceinline__ void part_of(const SampleArgs &a, int part, int *i0, int *i1) {
    *i0 = part * a.part < a.V ? part * a.part : a.V;
    *i1 = *i0 + a.part < a.V ? *i0 + a.part : a.V;
}

// Into the last bin, a wave's together.  (Hundreds of additions to one place take microseconds.)
__device__ __forceinline__ void add_last(unsigned long long *mass, uint32_t *count, uint32_t c, unsigned long long w) {
    if (!__any(c != 0)) return;
    const uint32_t wave_count = scan_wave(c);
    const unsigned long long wave_mass = scan_wave(w);
    if ((threadIdx.x & 63) == 63) {
        atomicAdd(&count[kBins - 1], wave_count);
        atomicAdd(&mass[kBins - 1], wave_mass);
    }
}

// Of logits [i0, i1) of a row the first token, and relative to it the bins, for a temperature above 0; l: the first N
// blocks of them (the first of these: the last one of all, if there are more).  The workgroup's, who has to meet before the bins are read.
template <int N, bool BF16>
__device__ __forceinline__ First fill_bins(const Row<BF16> &row, const Ask &k, int i0, int i1, float (&l)[N][8], unsigned long long *mass,
                                           uint32_t *count, double *roots, First *firsts) {
    const int tid = threadIdx.x, lane = tid & 63;
    // The first N blocks of logits stay in registers from here to the bins, others (of parts that have more) are read
    // twice.
    First best = {0, ~0u};
    auto look = [&](int b, const float (&at)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = sort_word(at[j]);
            const int i = b + j * kSampleThreads + tid;
            if (v > best.word || (v == best.word && (uint32_t)i < best.index)) best = First{v, (uint32_t)i};
        }
    };
#pragma unroll
    for (int q = 0; q < N; ++q) row.load(i0 + q * kBlock, i1, l[q]);
    for (int b = i0 + N * kBlock; b < i1; b += kBlock) {
        float more[8];
        row.load(b, i1, more);
        look(b, more);
    }
#pragma unroll
    for (int q = 0; q < N; ++q) look(i0 + q * kBlock, l[q]);
    mass[tid] = 0;
    count[tid] = 0;
    if (tid < kRoots) roots[tid] = kRoot[tid];
    best = first_of<64>(best);
    if (lane == 0) firsts[tid >> 6] = best;
    __syncthreads();
    best = first_of<16>(firsts[lane & 15]);
    if (k.temperature > 0.0f && best.word) {
        const float most = of_sort_word(best.word);
        const Weights w(most, k.temperature, roots);
        const Grid grid = {Grid::number(most)};
        uint32_t far = 0;  // the last bin's
        unsigned long long far_mass = 0;
        auto add = [&](const float (&at)[8]) {
#pragma unroll
            for (int j0 = 0; j0 < 8; j0 += 4) {
                uint64_t weight[4];
                int bin[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bin[j] = grid.bin(at[j0 + j]);
                    weight[j] = w.of(at[j0 + j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!(at[j0 + j] > -INFINITY)) continue;
                    if (bin[j] == kBins - 1) {
                        ++far;
                        far_mass += weight[j];
                        continue;
                    }
                    atomicAdd(&count[bin[j]], 1u);
                    atomicAdd(&mass[bin[j]], (unsigned long long)weight[j]);
                }
            }
        };
#pragma unroll
        for (int q = 0; q < N; ++q) add(l[q]);
        for (int b = i0 + N * kBlock; b < i1; b += kBlock) {
            row.load(b, i1, l[0]);
            add(l[0]);
        }
        add_last(mass, count, far, far_mass);
    }
    return best;
}

// The sums of the weights and tokens of the bins before a thread's own; *all, *n: of all bins.
__device__ __forceinline__ void scan_bins(unsigned long long own_mass, uint32_t own_count, unsigned long long *wave64, uint32_t *wave32,
                                          unsigned long long *own_before, uint32_t *own_ranked, unsigned long long *all, uint32_t *n) {
    const int tid = threadIdx.x, lane = tid & 63;
    // scan_block of both at once
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned long long sum = scan_wave(own_mass);
    const uint32_t num = scan_wave(own_count);
    if (lane == 63) {
        wave64[w] = sum;
        wave32[w] = num;
    }
    __syncthreads();
    const unsigned long long sums = scan_row(wave64[lane & 15]);
    const uint32_t nums = scan_row(wave32[lane & 15]);
    *all = of_lane(sums, 15);
    *n = of_lane(nums, 15);
    *own_before = (w ? of_lane(sums, w ? w - 1 : 0) : 0) + sum - own_mass;
    *own_ranked = (w ? of_lane(nums, w ? w - 1 : 0) : 0) + num - own_count;
}

template <bool BF16>
__global__ __launch_bounds__(kSampleThreads, 8) void sample_bins_kernel(SampleArgs a) {
    __shared__ unsigned long long mass[kBins], before[kBins + 1], wave64[kSampleWaves];
    __shared__ uint32_t count[kBins], ranked[kBins + 1], wave32[kSampleWaves];
    __shared__ First firsts[kSampleWaves];
    __shared__ double roots[kRoots];
    __shared__ uint32_t last;
    const int m = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x, lane = tid & 63;
    const Row<BF16> row(a, m);
    const Ask k = ask_of(a, m);
    RowState &state = a.rows[m];
    int i0, i1;
    part_of(a, part, &i0, &i1);

    float l[1][8];
    First best = fill_bins(row, k, i0, i1, l, mass, count, roots, firsts);
    const bool ordinary = k.temperature > 0.0f;  // (else the first token is the answer)
    __syncthreads();
    float most = of_sort_word(best.word);
    {  // the parts' bins, joined
        PartBins &to = a.bins[(int64_t)m * a.parts + part];
        const int place = ((int)Grid::number(most) - tid) & (kBins - 1);
        put64(reinterpret_cast<unsigned long long *>(&to.mass[place]), (uint64_t)__double_as_longlong((double)mass[tid]));
        put32(&to.count[place], count[tid]);
        if (tid == 0) put64(&a.heads[(int64_t)m * a.parts + part].first, (uint64_t)best.word << 32 | best.index);
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): written through to where all XCDs see it
        __syncthreads();
        if (tid == 0) {
            const uint32_t arrived = __hip_atomic_fetch_add(a.arrived + m, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = arrived == (uint32_t)a.parts - 1;
            if (last) put32(a.arrived + m, 0);
        }
        __syncthreads();
        if (!last) return;
        // Every part's bin at this place, and by a lane each the parts' first tokens; without branches between the loads.
        constexpr int kAtOnce = 8;
        double ms[kAtOnce];
        uint32_t cs[kAtOnce];
        auto ask = [&](int p0) {
#pragma unroll
            for (int p = 0; p < kAtOnce; ++p) {
                const PartBins &from = a.bins[(int64_t)m * a.parts + (p0 + p < a.parts ? p0 + p : 0)];
                ms[p] = __longlong_as_double((long long)get64(reinterpret_cast<const unsigned long long *>(&from.mass[tid])));
                cs[p] = get32(&from.count[tid]);
            }
        };
        const uint64_t head = get64(&a.heads[(int64_t)m * a.parts + (lane < a.parts ? lane : 0)].first);
        ask(0);
        First mine = {(uint32_t)(head >> 32), (uint32_t)head};
        if (lane >= a.parts) mine = First{0, ~0u};
        best = first_of<64>(mine);
        most = of_sort_word(best.word);
        // A part's weights, relative to the row's largest; its bins, so many places further down.
        const float own = of_sort_word(mine.word), top = Grid::number(most);
        const double factor = mine.word ? exp(((double)own - (double)most) / (double)k.temperature) : 0.0;
        const int shift = (int)fminf(top - Grid::number(own), (float)kBins), bin = ((int)top - tid) & (kBins - 1);
        // What a part has at this place is in the row's bin, or was moved past the last one, to which it belongs.
        double sum = 0.0, past = 0.0;
        uint32_t num = 0, rest = 0;
        for (int p0 = 0; p0 < a.parts; p0 += kAtOnce) {
            if (p0 > 0) ask(p0);
#pragma unroll
            for (int p = 0; p < kAtOnce; ++p) {
                if (p0 + p >= a.parts) break;
                const double v = __longlong_as_double((long long)of_lane((uint64_t)__double_as_longlong(factor), p0 + p)) * ms[p];
                const bool in = bin >= of_lane(shift, p0 + p);
                sum += in ? v : 0.0;
                past += in ? 0.0 : v;
                num += in ? cs[p] : 0;
                rest += in ? 0 : cs[p];
            }
        }
        mass[bin] = (unsigned long long)sum;
        count[bin] = num;
        __syncthreads();
        add_last(mass, count, rest, (unsigned long long)past);
        __syncthreads();
    }
    if (best.word == 0 || !ordinary || most == INFINITY) {  // (the same for the whole row)
        if (tid == 0) {
            a.ids[m] = best.word == 0 ? -1 : (int)best.index;
            state.gather = 0;
        }
        return;
    }
    const Grid grid = {Grid::number(most)};
    unsigned long long all, own_before;
    uint32_t n, own_ranked;
    scan_bins(mass[tid], count[tid], wave64, wave32, &own_before, &own_ranked, &all, &n);
    state.before[tid] = before[tid] = own_before;
    state.ranked[tid] = ranked[tid] = own_ranked;
    if (tid == 0) {
        before[kBins] = all;
        ranked[kBins] = n;
    }
    __syncthreads();
    if (tid >= 64) return;
    const Search found = search(k, grid, most, before, ranked);
    const uint32_t listed = listed_before(found.lo, found.hi, ranked, kBins);
    if (tid == 0) {
        state.ranked[kBins] = n;
        state.gather = listed > (uint32_t)kList || !(fabsf(grid.top) < kFar) ? 2 : 1;
        state.listed = 0;
        state.arrived = 0;
        state.top = grid.top;
        state.most = most;
        for (int i = 0; i < 4; ++i) {
            state.lo[i] = found.lo[i];
            state.hi[i] = found.hi[i];
        }
        state.all = all;
        state.count = n;
        state.cut = found.cut;
    }
}

constexpr int kFound = 6;  // words of LDS that finish looks for tokens with; the last one: whether a slot is crowded
// Tokens of a slot that are too many to be ranked by counting.  (Each counts for 0.036 us in a list of up to 1024 tokens, 0.13 in a
// longer one; sorting these by exchanges takes 14 and 38 us.)
constexpr uint32_t kCrowd = 320;

// What is known of a row whose tokens have been listed.
struct Listed {
    float most;
    int cut;
    uint32_t count;
    unsigned long long all;
};

// The answer from the n listed tokens, by the first W waves, which are all that is left of the workgroup (kEach tokens to
// a thread).  list(i): token i of them; key, sum: room for kList each, sum also where they may come from.
template <int W, int kEach, typename LIST>
__device__ int finish(const Listed &state, LIST list, const Ask &k, const Grid &grid, const int (&lo)[4], const int (&hi)[4], int n,
                      unsigned long long *key, unsigned long long *sum, unsigned long long *wave64, uint32_t *wave32, uint32_t *found,
                      unsigned long long *kept_at, const unsigned long long *before, const uint32_t *ranked, const double *roots,
                      float per_index) {
    constexpr int kThreads = 64 * W, kSlots = kThreads * kEach;
    const int tid = threadIdx.x;
    // Before the keys are in order: tokens per slot, and of the slots before.  Before the sums: keys by slot.
    uint32_t *const count = reinterpret_cast<uint32_t *>(key), *const begin = count + kSlots;
    // Sorted by interpolation: a bin's tokens have as many slots as they are, a logit's slot goes by its place within the
    // bin, and the few that share one are ranked by counting.  Where all logits are bf16 values, of which a bin has few and a
    // row many that are equal, the index counts as well, over half the distance of two values (128256 of them, a spread of
    // 1.5 at a temperature of 2: 84 us without, 32 with).
    uint64_t mine[kEach];
    uint32_t slot[kEach], nth[kEach];
    bool fine = false;
    if (tid == 0) found[kFound - 1] = 0;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        const int i = q * kThreads + tid;
        mine[q] = i < n ? list(i) : 0;
        count[i] = 0;
        fine |= i < n && (__float_as_uint(of_sort_word((uint32_t)(mine[q] >> 32))) & 0xffffu);
    }
    fine = __any(fine);
    if ((tid & 63) == 0) wave32[tid >> 6] = fine;
    __syncthreads();
    fine = __any(wave32[(tid & 15) < W ? tid & 15 : 0] != 0);
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        if (q * kThreads + tid >= n) continue;
        const float l = of_sort_word((uint32_t)(mine[q] >> 32));
        const int b = grid.bin(l);
        const uint32_t from = listed_before(lo, hi, ranked, b), room = ranked[b + 1] - ranked[b];
        const float v = l * kSteps;
        float down = b + 1 < kBins ? floorf(v) + 1.0f - v : 0.0f;  // (0, 1]; the last bin: one slot
        if (!fine && b + 1 < kBins) {
            const uint32_t e = __float_as_uint(l) >> 23 & 255;
            const float half = fminf(e > 8 ? __uint_as_float((e - 8) << 23) * kSteps : 0.0f, 1.0f);  // (half a step of bf16)
            down = down - half + half * ((float)~(uint32_t)mine[q] * per_index);
        }
        const uint32_t in = (uint32_t)(down * (float)room);
        slot[q] = from + (in < room ? in : room - 1);
        nth[q] = atomicAdd(&count[slot[q]], 1u);
        if (nth[q] >= kCrowd) found[kFound - 1] = 1;
    }
    __syncthreads();
    if (kSlots > (int)kCrowd && __builtin_amdgcn_readfirstlane(found[kFound - 1])) {
        // Equal logits beside one that bf16 does not hold, nearly equal ones, and those of the last bin share a slot, where every
        // token would read all the others.  Exchanges at halving distances take the same time whatever the tokens are (4000 times
        // 0.1: 57 us instead of 540).
        int slots = 64;
        while (slots < n) slots *= 2;
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid < slots) key[q * kThreads + tid] = mine[q];
        __syncthreads();
        for (int size = 2; size <= slots; size *= 2)
            for (int far = size / 2; far; far /= 2) {
                for (int p = tid; p < slots / 2; p += kThreads) {
                    const int i = 2 * p - (p & (far - 1)), j = i + far;
                    const uint64_t a = key[i], b = key[j];
                    if ((a < b) == !(i & size)) {
                        key[i] = b;
                        key[j] = a;
                    }
                }
                __syncthreads();
            }
    } else {
        {
            uint32_t c[kEach], sum4 = 0, all;
#pragma unroll
            for (int q = 0; q < kEach; ++q) {
                c[q] = count[kEach * tid + q];
                sum4 += c[q];
            }
            uint32_t at = scan_block<W>(wave32, sum4, &all);
#pragma unroll
            for (int q = 0; q < kEach; ++q) {
                begin[kEach * tid + q] = at;
                at += c[q];
            }
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid < n) sum[begin[slot[q]] + nth[q]] = mine[q];
        __syncthreads();
        uint32_t to[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            if (q * kThreads + tid >= n) continue;
            const uint32_t j0 = begin[slot[q]], j1 = j0 + count[slot[q]];
            to[q] = j0;
            for (uint32_t j = j0; j < j1; ++j) to[q] += sum[j] > mine[q];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid < n) key[to[q]] = mine[q];
        __syncthreads();
    }
    // Per token: its weight, the sum of the weights up to it (itself included) in the row, and its rank there.
    const Weights w(state.most, k.temperature, roots);
    uint64_t weight[kEach], upto[kEach], carry = 0;
    uint32_t rank[kEach];
    int bin[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        weight[q] = 0;
        if (q * kThreads >= n) continue;
        const int i = q * kThreads + tid;
        if (i < n) weight[q] = w.of_word((uint32_t)(key[i] >> 32));
        unsigned long long all;
        const uint64_t at = scan_block<W>(wave64, (unsigned long long)weight[q], &all);
        if (i < n) sum[i] = carry + at;
        carry += all;
    }
    if (tid < kFound) found[tid] = ~0u;
    if (tid == 0) *kept_at = state.all;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        const int i = q * kThreads + tid;
        if (i >= n) continue;
        bin[q] = grid.bin(of_sort_word((uint32_t)(key[i] >> 32)));
        const uint32_t first = listed_before(lo, hi, ranked, bin[q]);
        upto[q] = before[bin[q]] + (sum[i] + weight[q] - sum[first]);
        rank[q] = ranked[bin[q]] + ((uint32_t)i - first);
    }
    // The first token for which `is` holds, as it does for all behind it; n if there is none.  `at`: a word of LDS.
    auto first_token = [&](uint32_t *at, auto is) {
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const uint64_t any = __ballot(q * kThreads + tid < n && is(q));
            if (any && (tid & 63) == 0) atomicMin(at, (uint32_t)(q * kThreads + tid + __builtin_ctzll(any)));
        }
        __syncthreads();
        return *at < (uint32_t)n ? (int)*at : n;
    };
    // The sum of the weights with which a token is reached: by the thread that has it.
    auto keep = [&](uint64_t v) { if (v < *kept_at) *kept_at = v; };
    if (k.top_k > 0 && (uint32_t)k.top_k < state.count) {
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid < n && rank[q] == (uint32_t)k.top_k - 1) {
                keep(upto[q]);
                found[3] = (uint32_t)(q * kThreads + tid + 1);
            }
        __syncthreads();
    }
    int end = n;  // the listed tokens before it are those that top_p and min_p keep, those before found[3] top_k
    if (!(k.top_p >= 1.0f)) {
        const uint64_t reach = reach_of(k.top_p, *kept_at);
        const int i = first_token(&found[0], [&](int q) { return upto[q] >= reach; });
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid == i) keep(upto[q]);
        end = i < n ? i + 1 : n;
        __syncthreads();
    }
    if (k.min_p > 0.0f) {
        // (of the bins from `cut` on; before them all have the weight)
        const int i = first_token(&found[1], [&](int q) { return bin[q] >= state.cut && !((double)weight[q] >= (double)k.min_p * kOne); });
        if (i == 0 && tid == 0) keep(before[state.cut]);
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if (q * kThreads + tid == i - 1) keep(bin[q] >= state.cut ? upto[q] : before[state.cut]);
        end = i < end ? i : end;
        __syncthreads();
    }
    const uint64_t kept = *kept_at < 1ull << kPoint ? 1ull << kPoint : *kept_at;  // (the first token's weight is 1)
    const uint64_t x = point_of(k.u, kept);
    int i = first_token(&found[2], [&](int q) { return weight[q] && upto[q] > x; });
    end = found[3] < (uint32_t)end ? (int)found[3] : end;
    if (i >= end) {  // (a bin's sum and its tokens' have been rounded apart: the last token that is kept and has a weight)
        i = first_token(&found[4], [&](int q) { return weight[q] == 0; });
        i = (i < end ? i : end) - 1;
    }
    return (int)~(uint32_t)key[i > 0 ? i : 0];
}

// The same from up to 64 tokens by one wave, a token to a lane, which takes no LDS but for what it looks up.
template <typename LIST>
__device__ int finish_few(const Listed &state, LIST list, const Ask &k, const Grid &grid, const int (&lo)[4], const int (&hi)[4], int n,
                          const unsigned long long *before, const uint32_t *ranked, const double *roots) {
    const int lane = threadIdx.x & 63;
    const uint64_t mine = lane < n ? list(lane) : 0;
    const uint64_t all = state.all;
    const uint32_t row_count = state.count;
    const float most = state.most;
    const int row_cut = state.cut;
    int to = lane < n ? 0 : lane;
    for (int j = 0; j < n; ++j) to += of_lane(mine, j) > mine && lane < n;
    const uint32_t word = (uint32_t)__builtin_amdgcn_ds_permute(4 * to, (int)(mine >> 32));
    const uint32_t index = ~(uint32_t)__builtin_amdgcn_ds_permute(4 * to, (int)(uint32_t)mine);
    const Weights w(most, k.temperature, roots);
    const uint64_t weight = lane < n ? w.of_word(word) : 0, sum = scan_wave(weight) - weight;
    const int bin = lane < n ? grid.bin(of_sort_word(word)) : kBins - 1;
    const uint32_t first = listed_before(lo, hi, ranked, bin) & 63;  // (the first listed token of the bin; of no token: any lane)
    const uint64_t upto = before[bin] + (sum + weight - (uint64_t)__shfl((unsigned long long)sum, (int)first));
    const uint32_t rank = ranked[bin] + ((uint32_t)lane - first);
    const uint64_t live = n < 64 ? (1ull << n) - 1 : ~0ull;
    uint64_t kept = all;
    int end = n;  // the tokens before it are those that are kept
    auto keep = [&](uint64_t v) { kept = v < kept ? v : kept; };
    if (k.top_k > 0 && (uint32_t)k.top_k < row_count) {
        const uint64_t at = __ballot(rank == (uint32_t)k.top_k - 1) & live;
        if (at) {
            end = __builtin_ctzll(at) + 1;
            keep(of_lane(upto, end - 1));
        }
    }
    if (!(k.top_p >= 1.0f)) {
        const uint64_t reach = reach_of(k.top_p, kept), at = __ballot(upto >= reach) & live;
        if (at) {
            const int i = __builtin_ctzll(at);
            end = i + 1 < end ? i + 1 : end;
            keep(of_lane(upto, i));
        }
    }
    if (k.min_p > 0.0f) {
        // (of the bins from `cut` on; before them all have the weight)
        const uint64_t below = __ballot(bin >= row_cut && !((double)weight >= (double)k.min_p * kOne)) & live;
        const int i = below ? __builtin_ctzll(below) : n;
        if (i == 0 || of_lane(bin, i ? i - 1 : 0) < row_cut)
            keep(before[row_cut]);
        else
            keep(of_lane(upto, i - 1));
        end = i < end ? i : end;
    }
    kept = kept < 1ull << kPoint ? 1ull << kPoint : kept;  // (the first token's weight is 1)
    const uint64_t x = point_of(k.u, kept), weighty = __ballot(weight != 0) & live, at = __ballot(upto > x) & weighty;
    int i = at ? __builtin_ctzll(at) : n;
    if (i >= end) {  // (as in finish; those with a weight are the first)
        i = __builtin_popcountll(weighty);
        i = (i < end ? i : end) - 1;
    }
    return (int)of_lane(index, i > 0 ? i : 0);
}

// The same by whoever is needed, the answer in the first thread.
template <typename LIST>
__device__ __forceinline__ int choose(const Listed &row, LIST list, const Ask &k, const Grid &grid, const int (&lo)[4], const int (&hi)[4], int n, int V,
                                      unsigned long long *key, unsigned long long *sum, unsigned long long *wave64, uint32_t *wave32,
                                      uint32_t *found, unsigned long long *kept, const unsigned long long *before, const uint32_t *ranked,
                                      const double *roots) {
    const int tid = threadIdx.x;
    // By as few waves as hold the tokens, at first one to a thread: the others have ended, so that barriers wait for few.
    // (Four to a thread where one would do: 33.4 instead of 32.6 us for 32 rows of 128256.)
    const float per_index = 1.0f / (float)V;
    int id = 0;
    if (n <= 64) {
        if (tid < 64) id = finish_few(row, list, k, grid, lo, hi, n, before, ranked, roots);
    } else if (n <= 256) {
        if (tid < 256) id = finish<4, 1>(row, list, k, grid, lo, hi, n, key, sum, wave64, wave32, found, kept, before, ranked, roots, per_index);
    } else if (n <= 1024) {
        if (tid < 1024) id = finish<16, 1>(row, list, k, grid, lo, hi, n, key, sum, wave64, wave32, found, kept, before, ranked, roots, per_index);
    } else {
        id = finish<kSampleWaves, kList / kSampleThreads>(row, list, k, grid, lo, hi, n, key, sum, wave64, wave32, found, kept, before, ranked, roots, per_index);
    }
    return id;
}

template <bool BF16>
__global__ __launch_bounds__(kSampleThreads) void sample_list_kernel(SampleArgs a) {
    __shared__ unsigned long long key[kList], sum[kList], wave64[kSampleWaves];
    __shared__ uint32_t wave32[kSampleWaves], last;
    __shared__ unsigned long long kept, before[kBins];
    __shared__ uint32_t found[kFound], ranked[kBins + 1];
    __shared__ double roots[kRoots];
    const int m = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x, lane = tid & 63;
    RowState &state = a.rows[m];
    const Row<BF16> row(a, m);
    int i0, i1;
    part_of(a, part, &i0, &i1);
    // (asked for together: what the row's answer is made of, its first logits, and what the last workgroup looks up)
    const uint32_t gather = state.gather;
    const Ask k = ask_of(a, m);
    const Grid grid = {state.top};
    int lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = state.lo[i];
        hi[i] = state.hi[i];
    }
    float l[8];
    row.load(i0, i1, l);
    const unsigned long long own_before = state.before[tid];
    const uint32_t own_ranked = state.ranked[tid], all_ranked = state.ranked[kBins];
    const double own_root = kRoot[lane];
    if (gather == 0 || (gather == 2 && part > 0)) return;
    static_assert(sizeof(Shared) <= sizeof(key), "room for it");
    if (gather == 2) {  // (the second launch has the registers: in the first they would halve its workgroups)
        const int id = choose_slowly(*reinterpret_cast<Shared *>(key), row, k, state.most, state.count);
        if (tid == 0) a.ids[m] = id;
        return;
    }
    for (int b = i0; b < i1; b += kBlock) {
        if (b > i0) row.load(b, i1, l);
        uint64_t hits[8];
        uint32_t all = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int bin = grid.bin(l[j]);
            hits[j] = __ballot(listed_bin(lo, hi, bin) && l[j] > -INFINITY);
            all += (uint32_t)__builtin_popcountll(hits[j]);
        }
        if (all == 0) continue;  // (the wave's: most have none)
        uint32_t at = 0;
        if (lane == 0) at = __hip_atomic_fetch_add(&state.listed, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t to = at + (uint32_t)__builtin_popcountll(hits[j] & ((1ull << lane) - 1));
            if ((hits[j] >> lane & 1) && to < (uint32_t)kList)
                put64(&state.list[to], (uint64_t)sort_word(l[j]) << 32 | (uint32_t)~(b + j * kSampleThreads + tid));
            at += (uint32_t)__builtin_popcountll(hits[j]);
        }
    }
    before[tid] = own_before;
    ranked[tid] = own_ranked;
    if (tid == 0) ranked[kBins] = all_ranked;
    if (tid < kRoots) roots[tid] = own_root;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): written through to where all XCDs see it
    __syncthreads();
    if (tid == 0) last = __hip_atomic_fetch_add(&state.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.parts - 1;
    __syncthreads();
    if (!last) return;

    const int n = (int)get32(&state.listed) < kList ? (int)get32(&state.listed) : kList;
    const int id = choose(Listed{state.most, state.cut, state.count, state.all}, [&](int i) { return get64(&state.list[i]); }, k, grid, lo, hi, n, a.V,
                          key, sum, wave64, wave32, found, &kept, before, ranked, roots);
    if (tid == 0) a.ids[m] = id;
}

// Both in one launch, a workgroup to a row of one part.  N > 1: of up to N blocks, which stay in registers; 1: of any number.  (A
// row of 1000 10.4 us instead of 12.9, 64 of 8000 14.6 instead of 17.6; one of 16000 16.5, read again 17.7.)  More rows than compute
// units go two workgroups to one, which is worth more than the registers that one could have: 1024 rows of 8000 35 us, with one 42.5.
template <bool BF16, int N>
__global__ __launch_bounds__(kSampleThreads, N == 1 ? 8 : 4) void sample_row_kernel(SampleArgs a) {
    __shared__ unsigned long long key[kList], sum[kList], wave64[kSampleWaves];
    __shared__ unsigned long long kept, before[kBins + 1];
    __shared__ uint32_t wave32[kSampleWaves], found[kFound], ranked[kBins + 1], listed;
    __shared__ First firsts[kSampleWaves];
    __shared__ double roots[kRoots];
    __shared__ Search where;
    __shared__ bool serve;
    // (until they are summed)
    unsigned long long *const mass = key;
    uint32_t *const count = reinterpret_cast<uint32_t *>(key + kBins);
    const int m = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const Row<BF16> row(a, m);
    const Ask k = ask_of(a, m);
    float l[N][8];
    const First best = fill_bins(row, k, 0, a.V, l, mass, count, roots, firsts);
    const float most = of_sort_word(best.word);
    if (best.word == 0 || !(k.temperature > 0.0f) || most == INFINITY) {  // (the same for the whole row)
        if (tid == 0) a.ids[m] = best.word == 0 ? -1 : (int)best.index;
        return;
    }
    __syncthreads();
    const Grid grid = {Grid::number(most)};
    unsigned long long all, own_before;
    uint32_t tokens, own_ranked;
    scan_bins(mass[tid], count[tid], wave64, wave32, &own_before, &own_ranked, &all, &tokens);
    before[tid] = own_before;
    ranked[tid] = own_ranked;
    if (tid == 0) {
        before[kBins] = all;
        ranked[kBins] = tokens;
        listed = 0;
    }
    __syncthreads();
    if (tid < 64) {
        const Search at = search(k, grid, most, before, ranked);
        const bool can = listed_before(at.lo, at.hi, ranked, kBins) <= (uint32_t)kList && fabsf(grid.top) < kFar;
        if (tid == 0) {
            where = at;
            serve = can;
        }
    }
    __syncthreads();
    if (!serve) {
        const int id = choose_slowly(*reinterpret_cast<Shared *>(key), row, k, most, tokens);
        if (tid == 0) a.ids[m] = id;
        return;
    }
    int lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = where.lo[i];
        hi[i] = where.hi[i];
    }
    auto collect = [&](int b, const float (&from)[8]) {
        uint64_t hits[8];
        uint32_t mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            hits[j] = __ballot(listed_bin(lo, hi, grid.bin(from[j])) && from[j] > -INFINITY);
            mine += (uint32_t)__builtin_popcountll(hits[j]);
        }
        if (mine == 0) return;  // (the wave's)
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&listed, mine);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t to = at + (uint32_t)__builtin_popcountll(hits[j] & ((1ull << lane) - 1));
            if ((hits[j] >> lane & 1) && to < (uint32_t)kList)
                sum[to] = (uint64_t)sort_word(from[j]) << 32 | (uint32_t)~(b + j * kSampleThreads + tid);
            at += (uint32_t)__builtin_popcountll(hits[j]);
        }
    };
    if constexpr (N > 1) {
#pragma unroll
        for (int q = 0; q < N; ++q) collect(q * kBlock, l[q]);
    } else {
        for (int b = 0; b < a.V; b += kBlock) {
            if (a.V > kBlock) row.load(b, a.V, l[0]);
            collect(b, l[0]);
        }
    }
    __syncthreads();
    const int n = (int)listed < kList ? (int)listed : kList;
    const int id = choose(Listed{most, where.cut, tokens, all}, [&](int i) { return (uint64_t)sum[i]; }, k, grid, lo, hi, n, a.V, key, sum, wave64,
                          wave32, found, &kept, before, ranked, roots);
    if (tid == 0) a.ids[m] = id;
}

// Parts of a row, of whole blocks of kBlock logits and as many each: as many workgroups in all as there are compute units, or twice
// as many where they would have more than two blocks each.  (In the last workgroup of a row the parts' bins cost as much as a part's:
// 32 rows of 128256, 256 and 512 workgroups, 31 and 34 us; 64 45 and 43, 100 79 and 63, 150 98 and 79, 200 107 and 101, 255 115 and
// 121.  28 rows in ten parts, two of them empty, 38.4, in eight 30.3.)
// Two blocks are one part, in one launch: a row of 10000 14.7 us instead of 17.6, of 16000 16.6 and 18.0, 200 of these 19.7 and 28;
// and so are three and four, of rows that would have fewer workgroups: 100 of 32000 30.1 and 37.3, 200 of 24000 27.5 and 39.7 (but
// with one to a block, one of 20000 22.4 and 18.1, 50 of 30000 28.8 and 21.5, 86 of 20000 25.9 and 23.3).
constexpr int kMostUnits = 256;
int parts_of(int M, int V) {
    const int units = device_cu_count() < kMostUnits ? device_cu_count() : kMostUnits;
    const int blocks = (V + kBlock - 1) / kBlock, share = (units + M - 1) / M;
    const int more = share > 1 && blocks > 2 * share ? (2 * units + M - 1) / M : share, most = more < kMostParts ? more : kMostParts;
    if (blocks <= 2 || (blocks <= 4 && share < blocks)) return 1;
    const int each = (blocks + most - 1) / most;  // (no part without a block)
    return (blocks + each - 1) / each;
}
// Parts that calls of up to M rows of up to V logits have in all, on a device of any size.
size_t most_parts(int M, int V) {
    const size_t blocks = (size_t)((V + kBlock - 1) / kBlock), per = blocks < kMostParts ? blocks : kMostParts;
    const size_t rows = (size_t)M * per, share = 4 * kMostUnits + (size_t)M;
    return rows < share ? rows : share;
}

bool sample_shape(int M, int V) { return M >= 1 && M <= NVQ_SAMPLE_MAX_M && V >= 1 && V <= NVQ_SAMPLE_MAX_V; }

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_sample_workspace_bytes(int M, int V) {
    using namespace nvq;
    if (!sample_shape(M, V)) return 0;
    return NVQ_SAMPLE_CLEAR_BYTES + sizeof(RowState) * (size_t)M + (sizeof(PartHead) + sizeof(PartBins)) * most_parts(M, V);
}

extern "C" int nvq_sample(const void *logits, int dtype, int64_t ld, int M, int V, const float *u, const float *temperature,
                          const int32_t *top_k, const float *top_p, const float *min_p, int32_t *ids, void *workspace,
                          size_t workspace_bytes, void *stream) {
    using namespace nvq;
    if (!logits || !u || !ids || (dtype != NVQ_F32 && dtype != NVQ_BF16)) return NVQ_ERR_INVALID_ARG;
    if (!sample_shape(M, V) || ld < V) return NVQ_ERR_SHAPE;
    if (!aligned(logits, dtype == NVQ_F32 ? 4 : 2) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
        !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(ids, 4))
        return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_sample_workspace_bytes(M, V)) return NVQ_ERR_WORKSPACE;
    SampleArgs a;
    a.logits = logits;
    a.ld = ld;
    a.M = M;
    a.V = V;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.ids = ids;
    a.parts = parts_of(M, V);
    a.part = ((V + a.parts - 1) / a.parts + kBlock - 1) / kBlock * kBlock;
    char *const ws = static_cast<char *>(workspace);
    a.arrived = reinterpret_cast<uint32_t *>(ws);
    a.rows = reinterpret_cast<RowState *>(ws + NVQ_SAMPLE_CLEAR_BYTES);
    a.bins = reinterpret_cast<PartBins *>(a.rows + M);
    a.heads = reinterpret_cast<PartHead *>(a.bins + (size_t)M * a.parts);
    const dim3 grid((unsigned)(M * a.parts)), block(kSampleThreads);
    const hipStream_t st = (hipStream_t)stream;
    if (a.parts == 1) {
        const int held = M > device_cu_count() || V <= kBlock || V > 4 * kBlock ? 1 : V <= 2 * kBlock ? 2 : 4;
        auto launch = [&](auto bf16) {
            constexpr bool kBf16 = decltype(bf16)::value;
            if (held == 1)
                hipLaunchKernelGGL((sample_row_kernel<kBf16, 1>), grid, block, 0, st, a);
            else if (held == 2)
                hipLaunchKernelGGL((sample_row_kernel<kBf16, 2>), grid, block, 0, st, a);
            else
                hipLaunchKernelGGL((sample_row_kernel<kBf16, 4>), grid, block, 0, st, a);
        };
        if (dtype == NVQ_BF16)
            launch(std::true_type());
        else
            launch(std::false_type());
        NVQ_HIP_TRY(hipGetLastError());
        return NVQ_OK;
    }
    if (dtype == NVQ_BF16)
        hipLaunchKernelGGL(sample_bins_kernel<true>, grid, block, 0, st, a);
    else
        hipLaunchKernelGGL(sample_bins_kernel<false>, grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    if (dtype == NVQ_BF16)
        hipLaunchKernelGGL(sample_list_kernel<true>, grid, block, 0, st, a);
    else
        hipLaunchKernelGGL(sample_list_kernel<false>, grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
