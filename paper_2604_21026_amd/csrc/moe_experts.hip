// nvq_moe_experts: the experts' feed-forward layers of 1 to 32 tokens and the weighted sum of their outputs,
// y[m] = sum_s w[m][s] * D_e (silu(G_e x[m]) * (U_e x[m])), e = ids[m][s], in two launches.
//
// The first one makes h = bf16(silu(g) * u) for every pair of a token and an expert: a workgroup takes 16 * R gate
// rows and the up rows beside them of one expert, for all tokens that chose it, so that every weight is read once.  The
// second one makes y: a workgroup takes 16 * R output rows over all experts, its waves in turn the experts (or parts of
// one, where there are fewer experts than waves), and the sums over experts stay in LDS, one copy per wave, added in wave
// order.  Products: mx_rows.h.
#include "mx_rows.h"
#include "transform.h"

namespace nvq {

namespace {

struct MoeArgs {
    const uint8_t *gu_q, *dn_q;
    const void *gu_s, *dn_s;
    int E, K, F;
    const uint16_t *x;
    const int32_t *ids;
    const float *weights;
    int M, top_k, pairs;
    uint32_t per_token;  // 65536 / top_k, rounded up: pair / top_k = pair * per_token >> 16 below 512 pairs
    uint16_t *h;         // [M * top_k][F], row m * top_k + the first slot of the expert
    void *y;
    int y_dtype;
};

__device__ __forceinline__ int token_of(const MoeArgs &a, int pair) { return (int)((uint32_t)pair * a.per_token >> 16); }

// The tokens of one expert in ascending order, spread over a wave: lane n of a lane-row has number 16 t + n of them
// for tile t (past the end: the first one's), and the pair of its first slot.
template <int T>
struct ExpertTokens {
    int count, token[T], pair[T];
};

// From the ids in memory; `first`: the lowest pair of the expert.
template <int T>
__device__ __forceinline__ ExpertTokens<T> tokens_of(const MoeArgs &a, int e, int &first) {
    const int lane = threadIdx.x & 63, n = lane & 15;
    ExpertTokens<T> et;
    et.count = 0;
    first = -1;
    int previous = -1;
    for (int base = 0; base < a.pairs; base += 64) {
        const int id = base + lane < a.pairs ? a.ids[base + lane] : -1;
        uint64_t here = __ballot(id == e);
        while (here) {  // (uniform)
            const int p = base + __builtin_ctzll(here);
            here &= here - 1;
            const int m = token_of(a, p);
            if (m == previous) continue;
            previous = m;
            if (et.count == 0) {
                first = p;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    et.token[t] = m;
                    et.pair[t] = p;
                }
            }
#pragma unroll
            for (int t = 0; t < T; ++t)
                if (16 * t + n == et.count) {
                    et.token[t] = m;
                    et.pair[t] = p;
                }
            ++et.count;
        }
    }
    return et;
}

template <int FMT, int R, int T, int W, int B>
__device__ __forceinline__ void gate_up(const MoeArgs &a, int e, int row0, const ExpertTokens<T> &et, float *red,
                                        const int *pair_of) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int n = lane & 15, G = a.K / 32;
    RowAt at[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t row = (int64_t)e * 2 * a.F + row0 + 16 * r + n;
        at[r] = row_at<FMT>(a.gu_q, a.gu_s, row, G);
        at[R + r] = row_at<FMT>(a.gu_q, a.gu_s, row + a.F, G);
    }
    const char *x[T];
    float4v sum[2 * R][T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        x[t] = reinterpret_cast<const char *>(a.x) + (int64_t)et.token[t] * a.K * 2;
#pragma unroll
        for (int r = 0; r < 2 * R; ++r) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    rows_times_tokens<FMT, 2 * R, T, B>(at, x, G, w, W, sum);
    constexpr int kRegs = 2 * R * T * 4;
#pragma unroll
    for (int r = 0; r < 2 * R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) red[(w * kRegs + (r * T + t) * 4 + j) * 64 + lane] = sum[r][t][j];
    __syncthreads();
    for (int i = threadIdx.x; i < R * T * 4 * 64; i += 64 * W) {
        const int reg = i >> 6, l = i & 63;
        const int t = (reg >> 2) % T, r = (reg >> 2) / T;
        const int number = 16 * t + 4 * (l >> 4) + (reg & 3);
        float g = 0.0f, u = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            g += red[(k * kRegs + reg) * 64 + l];
            u += red[(k * kRegs + R * T * 4 + reg) * 64 + l];
        }
        if (number < et.count)
            a.h[(int64_t)pair_of[number] * a.F + row0 + 16 * r + (l & 15)] = float_to_bf16_bits(silu_mul_one(g, u));
    }
}

template <int FMT, int R, int T, int W, int B>
__global__ __launch_bounds__(64 * W) void moe_gate_up_kernel(MoeArgs a) {
    __shared__ float red[W * 2 * R * T * 4 * 64];
    __shared__ int pair_of[32];
    const int row0 = blockIdx.x * (16 * R);
    // the second grid axis: experts, or pairs where there are fewer (a pair that is not the first of its expert has
    // nothing to do)
    const bool by_expert = a.E <= a.pairs;
    const int e = by_expert ? (int)blockIdx.y : a.ids[blockIdx.y];
    if ((uint32_t)e >= (uint32_t)a.E) return;
    int first;
    const ExpertTokens<T> et = tokens_of<T>(a, e, first);
    if (et.count == 0 || (!by_expert && first != (int)blockIdx.y)) return;
    if (threadIdx.x < 16) {
#pragma unroll
        for (int t = 0; t < T; ++t) pair_of[16 * t + threadIdx.x] = et.pair[t];
    }
    if (T == 1 || et.count > 16) {  // (the barrier inside comes before pair_of is read)
        gate_up<FMT, R, T, W, B>(a, e, row0, et, red, pair_of);
    } else {
        const ExpertTokens<1> one = {et.count, {et.token[0]}, {et.pair[0]}};
        gate_up<FMT, R, 1, W, B>(a, e, row0, one, red, pair_of);
    }
}

// One expert's part of a wave: columns first, first + step, ... of its inputs h, added to the wave's sums out[token][row].
template <int FMT, int R, int T, int B>
__device__ __forceinline__ void add_expert(const MoeArgs &a, const RowAt (&at)[R], const int (&token)[T],
                                           const int (&pair)[T], const float (&weight)[T], int count, int first, int step,
                                           float *out) {
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const char *h[T];
    float4v sum[R][T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        h[t] = reinterpret_cast<const char *>(a.h) + (int64_t)pair[t] * a.F * 2;
#pragma unroll
        for (int r = 0; r < R; ++r) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    rows_times_tokens<FMT, R, T, B>(at, h, a.F / 32, first, step, sum);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = __shfl(token[t], 4 * kb + j, 64);
            const float w = __shfl(weight[t], 4 * kb + j, 64);
            if (16 * t + 4 * kb + j < count) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float *const o = out + (m * R + r) * 16 + n;
                    *o = fmaf(w, sum[r][t][j], *o);
                }
            }
        }
}

template <int FMT, int R, int T, int W, int B>
__global__ __launch_bounds__(64 * W) void moe_down_kernel(MoeArgs a) {
    constexpr int kOut = 16 * T * R * 16;  // a wave's sums
    __shared__ float out[W * kOut];
    __shared__ uint32_t chosen[NVQ_MOE_MAX_EXPERTS];  // tokens of each expert
    __shared__ uint16_t active[NVQ_MOE_MAX_EXPERTS];
    __shared__ int ids[NVQ_MAX_M * NVQ_MOE_MAX_TOP_K];
    __shared__ float weights[NVQ_MAX_M * NVQ_MOE_MAX_TOP_K];
    __shared__ int nactive;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15;
    const int row0 = blockIdx.x * (16 * R);
    for (int i = threadIdx.x; i < a.E; i += 64 * W) chosen[i] = 0;
    for (int i = threadIdx.x; i < W * kOut; i += 64 * W) out[i] = 0.0f;
    __syncthreads();
    for (int i = threadIdx.x; i < a.pairs; i += 64 * W) {
        const int id = a.ids[i];
        ids[i] = id;
        weights[i] = a.weights[i];
        if ((uint32_t)id < (uint32_t)a.E) atomicOr(&chosen[id], 1u << token_of(a, i));
    }
    __syncthreads();
    if (w == 0) {
        int count = 0;
        for (int base = 0; base < a.E; base += 64) {
            const bool is = base + lane < a.E && chosen[base + lane] != 0;
            const uint64_t b = __ballot(is);
            if (is) active[count + __popcll(b & ((1ull << lane) - 1))] = (uint16_t)(base + lane);
            count += __popcll(b);
        }
        if (lane == 0) nactive = count;
    }
    __syncthreads();
    const int G = a.F / 32;
    // experts in `split` parts of their columns where there are fewer experts than waves
    const int split = nactive == 0 || nactive >= W ? 1 : (W + nactive - 1) / nactive;
    for (int item = w; item < nactive * split; item += W) {  // (uniform)
        const int e = __builtin_amdgcn_readfirstlane(active[item / split]);
        const uint32_t tokens = (uint32_t)__builtin_amdgcn_readfirstlane((int)chosen[e]);
        const int count = __popc(tokens);
        int token[T], pair[T];
        float weight[T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            // the lane's token: bit number 16 t + n of those set (the first one's past the end)
            uint32_t left = tokens;
            const int skip = 16 * t + n < count ? 16 * t + n : 0;
            for (int k = 0; k < skip; ++k) left &= left - 1;
            token[t] = __builtin_ctz(left);
            weight[t] = 0.0f;
            pair[t] = 0;
            for (int s = a.top_k - 1; s >= 0; --s) {
                const int p = token[t] * a.top_k + s;
                if (ids[p] == e) {
                    pair[t] = p;
                    weight[t] += weights[p];
                }
            }
        }
        RowAt at[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            at[r] = row_at<FMT>(a.dn_q, a.dn_s, (int64_t)e * a.K + row0 + 16 * r + n, G);
        if (T == 1 || count > 16) {
            add_expert<FMT, R, T, B>(a, at, token, pair, weight, count, item % split, split, out + w * kOut);
        } else {
            const int token1[1] = {token[0]}, pair1[1] = {pair[0]};
            const float weight1[1] = {weight[0]};
            add_expert<FMT, R, 1, B>(a, at, token1, pair1, weight1, count, item % split, split, out + w * kOut);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.M * R * 16; i += 64 * W) {
        float v = out[i];
#pragma unroll
        for (int k = 1; k < W; ++k) v += out[k * kOut + i];
        store_global(a.y, a.y_dtype, (int64_t)(i / (R * 16)) * a.K + row0 + i % (R * 16), v);
    }
}

template <int FMT, int T>
int launch_experts(const MoeArgs &a, hipStream_t st) {
#ifndef R1
#define R1 1
#define W1 4
#define C1 2
#define R2 1
#define W2 8
#define C2 4
#endif
    const unsigned experts = (unsigned)(a.E <= a.pairs ? a.E : a.pairs);
    hipLaunchKernelGGL((moe_gate_up_kernel<FMT, R1, T, W1, C1>), dim3(a.F / 16 / R1, experts), dim3(64 * W1), 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL((moe_down_kernel<FMT, R2, T, W2, C2>), dim3(a.K / 16 / R2), dim3(64 * W2), 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

// NVQ_OK, or what is wrong with the sizes.
int check_experts(const nvq_experts *e, int M, int top_k) {
    if (!e || (e->format != NVQ_FMT_INT4 && e->format != NVQ_FMT_MXFP4)) return NVQ_ERR_INVALID_ARG;
    if (e->E < 1 || e->E > NVQ_MOE_MAX_EXPERTS || e->K <= 0 || e->K % 32 || e->K > NVQ_MAX_K || e->F <= 0 || e->F % 32 ||
        e->F > NVQ_MAX_K || M < 1 || M > NVQ_MAX_M || top_k < 1 || top_k > NVQ_MOE_MAX_TOP_K)
        return NVQ_ERR_SHAPE;
    return NVQ_OK;
}

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_moe_workspace_bytes(const nvq_experts *experts, int M, int top_k) {
    if (nvq::check_experts(experts, M, top_k) != NVQ_OK) return 0;
    return ((size_t)M * top_k * experts->F * sizeof(uint16_t) + 255) / 256 * 256;
}

extern "C" int nvq_moe_experts(const nvq_experts *experts, const uint16_t *x_bf16, const int32_t *ids,
                               const float *weights, int M, int top_k, void *y, int y_dtype, void *workspace,
                               size_t workspace_bytes, void *stream) {
    using namespace nvq;
    if (!experts || !x_bf16 || !ids || !weights || !y || (y_dtype != NVQ_F32 && y_dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (!experts->gate_up || !experts->gate_up_scales || !experts->down || !experts->down_scales)
        return NVQ_ERR_INVALID_ARG;
    const int bad = check_experts(experts, M, top_k);
    if (bad) return bad;
    const size_t scale = experts->format == NVQ_FMT_INT4 ? 2 : 1;
    if (!aligned(experts->gate_up, 16) || !aligned(experts->down, 16) || !aligned(experts->gate_up_scales, scale) ||
        !aligned(experts->down_scales, scale) || !aligned(x_bf16, 16) || !aligned(ids, 4) || !aligned(weights, 4) ||
        !aligned(y, y_dtype == NVQ_F32 ? 4 : 2))
        return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_moe_workspace_bytes(experts, M, top_k))
        return NVQ_ERR_WORKSPACE;
    MoeArgs a;
    a.gu_q = experts->gate_up;
    a.gu_s = experts->gate_up_scales;
    a.dn_q = experts->down;
    a.dn_s = experts->down_scales;
    a.E = experts->E;
    a.K = experts->K;
    a.F = experts->F;
    a.x = x_bf16;
    a.ids = ids;
    a.weights = weights;
    a.M = M;
    a.top_k = top_k;
    a.pairs = M * top_k;
    a.per_token = (65536u + top_k - 1) / top_k;
    a.h = static_cast<uint16_t *>(workspace);
    a.y = y;
    a.y_dtype = y_dtype;
    const hipStream_t st = (hipStream_t)stream;
    if (experts->format == NVQ_FMT_INT4)
        return M <= 16 ? launch_experts<NVQ_FMT_INT4, 1>(a, st) : launch_experts<NVQ_FMT_INT4, 2>(a, st);
    return M <= 16 ? launch_experts<NVQ_FMT_MXFP4, 1>(a, st) : launch_experts<NVQ_FMT_MXFP4, 2>(a, st);
}
