// nvq_moe_route: the router of a mixture of experts for 1 to 32 tokens, in one launch: logits = x R^T (bf16 operands,
// fp32 sums), the top_k largest of each token in descending order (the lowest index first among equals) and their
// softmax weights.
//
// A few tokens' router is latency, not bytes: the grid is tiles of 16 experts times parts of K, so that a few
// hundred waves ask for everything at once; each leaves its partial logits in the workspace, and the workgroup that
// arrives last (a counter that wraps to zero by itself) adds them in the order of the parts and chooses.
//
// Measured: one token of 64 experts, 2048 inputs 5.2 us (an empty launch 2.4); 32 tokens of 128 experts, 4096
// inputs 7.8 us.
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;
constexpr int kRouteMaxParts = 4;

struct RouteArgs {
    const uint16_t *x, *router;
    int M, E, K, top_k, renormalise;
    int32_t *ids;
    float *weights;
    uint32_t *arrived;  // workspace
    float *partial;     // [tiles][parts][M][16]: a workgroup's in one piece
    int tiles, parts, cols;  // columns of 32 inputs per part
};

// Logits as words whose unsigned order is theirs; equal numbers (both zeros) give equal words, NaN the lowest.
constexpr uint32_t kNanWord = 1u;
__device__ __forceinline__ uint32_t order_word(float f) {
    if (f != f) return kNanWord;
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The logit of such a word (minus zero: zero).
__device__ __forceinline__ float of_order_word(uint32_t w) { return __uint_as_float(w & 0x80000000u ? w & 0x7fffffffu : ~w); }

struct MaxWord {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct MinWord {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a < b ? a : b; }
};
// Over groups of L lanes.
template <int L, typename T, typename OP>
__device__ __forceinline__ T over_group(T v, OP op) {
    if (L == 64) {
        v = with_lane_xor<32>(v, op);
        v = with_lane_xor<16>(v, op);
    }
    v = with_lane_xor<8>(v, op);
    v = with_lane_xor<4>(v, op);
    v = with_lane_xor<2>(v, op);
    return with_lane_xor<1>(v, op);
}

// The chosen experts of token m, by L lanes: lane i of them holds the logits of experts i, L + i .., P in all.
// Their parts are requested up to eight experts at once (one after the other they were 14 of the 25 us that 32
// tokens and 128 experts took).  A choice is instructions on one compute unit, not bytes.
template <int L, int P>
__device__ __forceinline__ void choose(const RouteArgs &a, int m) {
    const int i = threadIdx.x & (L - 1);
    const bool here = m < a.M;
    const float *const own = a.partial + (here ? m : a.M - 1) * 16;
    uint32_t key[P];
    constexpr int kAtOnce = P < 8 ? P : 8;
#pragma unroll
    for (int j0 = 0; j0 < P; j0 += kAtOnce) {
        float v[kAtOnce][kRouteMaxParts];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int e = L * (j0 + j) + i, in = e < a.E ? e : a.E - 1;
            const float *const at = own + (int64_t)(in >> 4) * a.parts * a.M * 16 + (in & 15);
#pragma unroll
            for (int p = 0; p < kRouteMaxParts; ++p)
                v[j][p] = __hip_atomic_load(at + (int64_t)(p < a.parts ? p : 0) * a.M * 16, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            float l = 0.0f;
#pragma unroll
            for (int p = 0; p < kRouteMaxParts; ++p) l += p < a.parts ? v[j][p] : 0.0f;
            key[j0 + j] = L * (j0 + j) + i < a.E ? order_word(l) : 0u;
        }
    }
    float all = 0.0f, top = 0.0f, chosen = 0.0f, mine = 0.0f;
    int my_id = 0;
    for (int k = 0; k < a.top_k; ++k) {
        uint32_t best = key[0];
        int at = i;  // the expert (of equal ones the lowest)
#pragma unroll
        for (int j = 1; j < P; ++j) {
            const bool more = key[j] > best;
            best = more ? key[j] : best;
            at = more ? L * j + i : at;
        }
        const uint32_t most = over_group<L>(best, MaxWord());
        const uint32_t id = P == 1 && L == 64 ? (uint32_t)__builtin_ctzll(__ballot(best == most))
                                              : over_group<L>(best == most ? (uint32_t)at : ~0u, MinWord());
        const float value = of_order_word(most);
        if (k == 0) {
            top = value;
            if (!a.renormalise) {
                // (experts past the last have words of zero; a NaN, the smallest, adds nothing)
#pragma unroll
                for (int j = 0; j < P; ++j) all += key[j] > kNanWord ? expf(of_order_word(key[j]) - top) : 0.0f;
                all = over_group<L>(all, AddOp());
            }
        }
#pragma unroll
        for (int j = 0; j < P; ++j)
            if ((uint32_t)(L * j + i) == id) key[j] = 0u;
        const float w = expf(value - top);
        chosen += w;
        if (i == k) {
            my_id = (int)id;
            mine = w;
        }
    }
    if (here && i < a.top_k) {
        a.ids[m * a.top_k + i] = my_id;
        a.weights[m * a.top_k + i] = mine / (a.renormalise ? chosen : all);
    }
}

// T token tiles; L lanes per token and P experts per lane in the choice.
template <int T, int L, int P>
__global__ __launch_bounds__(kRouteThreads) void moe_route_kernel(RouteArgs a) {
    __shared__ float red[kRouteWaves][T * 4][64];
    __shared__ uint32_t last;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int n = lane & 15, kb = lane >> 4;
    const int tile = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int e0 = 16 * tile;
    const int all_cols = a.K / 32, col0 = part * a.cols;
    const int col1 = col0 + a.cols < all_cols ? col0 + a.cols : all_cols;

    const char *const r =
        reinterpret_cast<const char *>(a.router) + (int64_t)(e0 + n < a.E ? e0 + n : a.E - 1) * a.K * 2 + kb * 16;
    const char *x[T];
    float4v sum[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int m = 16 * t + n;
        x[t] = reinterpret_cast<const char *>(a.x) + (int64_t)(m < a.M ? m : 0) * a.K * 2 + kb * 16;
        sum[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // Two columns at a time, a line of 128 bytes of every row.  (K of an odd number of columns: the last one by
    // itself.)
    for (int c = col0 + 2 * w; c < col1; c += 2 * kRouteWaves) {
        const bool both = c + 1 < col1;  // (uniform)
        uint4v b[2] = {}, v[2][T] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k == 1 && !both) break;
            b[k] = load_stream(reinterpret_cast<const uint4 *>(r + (int64_t)(c + k) * 64));
#pragma unroll
            for (int t = 0; t < T; ++t) v[k][t] = load_stream(reinterpret_cast<const uint4 *>(x[t] + (int64_t)(c + k) * 64));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int t = 0; t < T; ++t)
                sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[k][t]),
                                                                __builtin_bit_cast(bf16x8, b[k]), sum[t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        wait_written(sum[t]);
#pragma unroll
        for (int j = 0; j < 4; ++j) red[w][4 * t + j][lane] = sum[t][j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < T * 4 * 64; i += kRouteThreads) {
        const int reg = i >> 6, l = i & 63;
        const int m = 16 * (reg >> 2) + 4 * (l >> 4) + (reg & 3), e = e0 + (l & 15);
        float v = red[0][reg][l];
#pragma unroll
        for (int k = 1; k < kRouteWaves; ++k) v += red[k][reg][l];
        if (m < a.M && e < a.E)
            __hip_atomic_store(a.partial + ((int64_t)blockIdx.x * a.M + m) * 16 + (l & 15), v, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's partial logits are written
    __syncthreads();
    if (threadIdx.x == 0) {
        // The workgroup's partial logits are written through to where all XCDs see them (agent-scope stores,
        // waited for) before it arrives; the last one's loads are of that scope too and pass its caches by.  So
        // no cache has to be written back or emptied here, as a fence of that scope would.
        const uint32_t before = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = before == gridDim.x - 1;
        if (last) __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    const int m = threadIdx.x / L;
    if (m - m % (64 / L) < a.M) choose<L, P>(a, m);  // (whole waves)
}

template <int T, int L>
int launch_route(const RouteArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.tiles * a.parts)), block(kRouteThreads);
    if (a.E <= 64)
        hipLaunchKernelGGL((moe_route_kernel<T, L, 64 / L>), grid, block, 0, st, a);
    else if (a.E <= 128)
        hipLaunchKernelGGL((moe_route_kernel<T, L, 128 / L>), grid, block, 0, st, a);
    else if (a.E <= 256)
        hipLaunchKernelGGL((moe_route_kernel<T, L, 256 / L>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((moe_route_kernel<T, L, 512 / L>), grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

constexpr size_t kRouteCounterBytes = 256;

bool route_shape(int M, int E) { return M >= 1 && M <= NVQ_MAX_M && E >= 1 && E <= NVQ_MOE_MAX_EXPERTS; }

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_moe_route_workspace_bytes(int M, int E) {
    using namespace nvq;
    if (!route_shape(M, E)) return 0;
    return kRouteCounterBytes + sizeof(float) * kRouteMaxParts * (size_t)M * ((E + 15) / 16 * 16);
}

extern "C" int nvq_moe_route(const uint16_t *x_bf16, const uint16_t *router_bf16, int M, int E, int K, int top_k,
                             int renormalise, int32_t *ids, float *weights, void *workspace, size_t workspace_bytes,
                             void *stream) {
    using namespace nvq;
    if (!x_bf16 || !router_bf16 || !ids || !weights || (renormalise != 0 && renormalise != 1)) return NVQ_ERR_INVALID_ARG;
    if (!route_shape(M, E) || top_k < 1 || top_k > NVQ_MOE_MAX_TOP_K || top_k > E || K <= 0 || K % 32 || K > NVQ_MAX_K)
        return NVQ_ERR_SHAPE;
    if (!aligned(x_bf16, 16) || !aligned(router_bf16, 16) || !aligned(ids, 4) || !aligned(weights, 4)) return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_moe_route_workspace_bytes(M, E))
        return NVQ_ERR_WORKSPACE;
    RouteArgs a;
    a.x = x_bf16;
    a.router = router_bf16;
    a.M = M;
    a.E = E;
    a.K = K;
    a.top_k = top_k;
    a.renormalise = renormalise;
    a.ids = ids;
    a.weights = weights;
    a.arrived = static_cast<uint32_t *>(workspace);
    a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + kRouteCounterBytes);
    a.tiles = (E + 15) / 16;
    // a part: two columns per wave or more
    const int cols = K / 32;
    int parts = (cols + 2 * kRouteWaves - 1) / (2 * kRouteWaves);
    parts = parts < kRouteMaxParts ? parts : kRouteMaxParts;
    a.cols = ((cols + parts - 1) / parts + 1) / 2 * 2;  // (whole lines)
    a.parts = (cols + a.cols - 1) / a.cols;
    const hipStream_t st = (hipStream_t)stream;
    // Lanes per token in the choice: of many tokens four share a wave, sixteen lanes each (32 tokens of 128
    // experts 7.8 us against 9.4, of 6 experts 5.5 against 7.7); few tokens have a wave each (one of 256
    // experts 6.6 against 8.5, of 64 5.2 against 5.9).
    if (M <= 8) return launch_route<1, 64>(a, st);
    return M <= 16 ? launch_route<1, 16>(a, st) : launch_route<2, 16>(a, st);
}
