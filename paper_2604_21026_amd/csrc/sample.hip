// nvq_sample: the next token of each row of logits.
//
// Every question is one of the descending order of a row's tokens: which token brings the count to top_k, the sum of
// the weights to top_p, to u times the kept sum.  It is answered without sorting: the logits are words whose unsigned
// order is theirs, a histogram over eight bits of them (counts, or sums of weights) says in which bin the answer
// lies, and the next eight bits are looked at inside that bin alone.  Weights are 64-bit fixed point, so that sums do
// not depend on their order and all passes agree to the last bit.
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kPoint = 43;  // bits after the point: 2^20 weights of at most 1 stay below 2^63
constexpr double kOne = (double)(1ull << kPoint);

struct SampleArgs {
    const void *logits;
    int dtype;
    int64_t ld;
    int M, V;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *ids;
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

struct Row {
    const void *at;
    int dtype, V;
    __device__ uint32_t word(int i) const {
        return sort_word(dtype == NVQ_F32 ? static_cast<const float *>(at)[i]
                                          : bf16_bits_to_float(static_cast<const uint16_t *>(at)[i]));
    }
};

struct Weights {
    double top, temperature;
    __device__ uint64_t of(uint32_t word) const {
        return (uint64_t)(exp(((double)of_sort_word(word) - top) / temperature) * kOne + 0.5);
    }
};

struct Shared {
    uint32_t count[256];
    unsigned long long mass[256];
    unsigned long long wave[kSampleWaves];
    unsigned long long before;
    uint32_t bin;
};

template <typename OP>
__device__ uint64_t over_block(Shared &s, uint64_t v, OP op) {
    for (int d = 32; d; d >>= 1) v = op(v, (uint64_t)__shfl_xor((unsigned long long)v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s.wave[0];
    for (int i = 1; i < kSampleWaves; ++i) v = op(v, (uint64_t)s.wave[i]);
    return v;
}
struct Most64 {
    __device__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; }
};
struct Add64 {
    __device__ uint64_t operator()(uint64_t a, uint64_t b) const { return a + b; }
};

// The token at which the running count (or sum of weights) of the descending order first exceeds x: its word, and the
// count (sum) before all tokens of that word.  x is below the row's whole count (sum).
template <bool MASS>
__device__ void find(Shared &s, const Row &row, const Weights &w, uint64_t x, uint32_t *word, uint64_t *before) {
    uint32_t prefix = 0;
    uint64_t base = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += kSampleThreads) {
            s.count[i] = 0;
            s.mass[i] = 0;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < row.V; i += kSampleThreads) {
            const uint32_t v = row.word(i);
            if (v == 0 || (shift < 24 && v >> (shift + 8) != prefix)) continue;
            if (MASS)
                atomicAdd(&s.mass[v >> shift & 255], (unsigned long long)w.of(v));
            else
                atomicAdd(&s.count[v >> shift & 255], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint64_t sum = base;
            int bin = 255;
            for (; bin > 0; --bin) {
                const uint64_t here = MASS ? s.mass[bin] : s.count[bin];
                if (sum + here > x) break;
                sum += here;
            }
            s.bin = (uint32_t)bin;
            s.before = sum;
        }
        __syncthreads();
        prefix = prefix << 8 | s.bin;
        base = s.before;
    }
    *word = prefix;
    *before = base;
}

// The n-th token (from 0, by index) of a word; -1 if there are fewer.
__device__ int nth_of_word(Shared &s, const Row &row, uint32_t word, uint64_t n) {
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

__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    const int m = blockIdx.x;
    Row row;
    row.at = a.dtype == NVQ_F32 ? (const void *)(static_cast<const float *>(a.logits) + m * a.ld)
                                : (const void *)(static_cast<const uint16_t *>(a.logits) + m * a.ld);
    row.dtype = a.dtype;
    row.V = a.V;
    uint64_t best = 0, n = 0;
    for (int i = threadIdx.x; i < a.V; i += kSampleThreads) {
        const uint32_t v = row.word(i);
        const uint64_t k = (uint64_t)v << 32 | (uint32_t)~i;
        best = k > best ? k : best;
        n += v != 0;
    }
    best = over_block(s, best, Most64());
    n = over_block(s, n, Add64());
    const uint32_t top = (uint32_t)(best >> 32);
    const float temperature = a.temperature ? a.temperature[m] : 1.0f, most = of_sort_word(top);
    if (top == 0 || !(temperature > 0.0f) || most == INFINITY) {  // (the same for the whole row)
        if (threadIdx.x == 0) a.ids[m] = top == 0 ? -1 : (int)~(uint32_t)best;
        return;
    }
    const Weights w{(double)most, (double)temperature};
    const int top_k = a.top_k ? a.top_k[m] : 0;
    const float top_p = a.top_p ? a.top_p[m] : 1.0f, min_p = a.min_p ? a.min_p[m] : 0.0f;
    uint32_t word;
    uint64_t before, kept;
    if (top_k > 0 && (uint64_t)top_k < n) {
        find<false>(s, row, w, (uint64_t)top_k - 1, &word, &before);
        uint64_t above = 0;
        for (int i = threadIdx.x; i < a.V; i += kSampleThreads) {
            const uint32_t v = row.word(i);
            above += v > word ? w.of(v) : 0;
        }
        kept = over_block(s, above, Add64()) + ((uint64_t)top_k - before) * w.of(word);
    } else {
        uint64_t all = 0;
        for (int i = threadIdx.x; i < a.V; i += kSampleThreads) {
            const uint32_t v = row.word(i);
            all += v ? w.of(v) : 0;
        }
        kept = over_block(s, all, Add64());
    }
    if (!(top_p >= 1.0f)) {
        const double share = top_p > 0.0f ? ceil((double)top_p * (double)kept) : 0.0;
        const uint64_t reach = share < 1.0 ? 1 : share < (double)kept ? (uint64_t)share : kept;
        find<true>(s, row, w, reach - 1, &word, &before);
        const uint64_t each = w.of(word);
        kept = before + (reach - before + each - 1) / each * each;
    }
    if (min_p > 0.0f) {
        uint64_t enough = 0;
        for (int i = threadIdx.x; i < a.V; i += kSampleThreads) {
            const uint32_t v = row.word(i);
            const uint64_t x = v ? w.of(v) : 0;
            enough += (double)x >= (double)min_p * kOne ? x : 0;
        }
        enough = over_block(s, enough, Add64());
        kept = enough < kept ? enough : kept;
    }
    kept = kept < 1ull << kPoint ? 1ull << kPoint : kept;  // (the first token's weight is 1)
    const float u = a.u[m];
    const uint64_t x = !(u > 0.0f) ? 0 : u >= 1.0f ? kept - 1 : (uint64_t)((double)u * (double)kept);
    find<true>(s, row, w, x < kept ? x : kept - 1, &word, &before);
    const uint64_t at = x < kept ? x : kept - 1;
    const int id = nth_of_word(s, row, word, (at - before) / w.of(word));
    if (threadIdx.x == 0) a.ids[m] = id;
}

bool sample_shape(int M, int V) { return M >= 1 && M <= NVQ_SAMPLE_MAX_M && V >= 1 && V <= NVQ_SAMPLE_MAX_V; }

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_sample_workspace_bytes(int M, int V) {
    using namespace nvq;
    return sample_shape(M, V) ? NVQ_SAMPLE_CLEAR_BYTES : 0;
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
    a.dtype = dtype;
    a.ld = ld;
    a.M = M;
    a.V = V;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.ids = ids;
    hipLaunchKernelGGL(sample_kernel, dim3((unsigned)M), dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
