// nvq_moe_experts: the experts' feed-forward layers of 1 to 32 tokens and the weighted sum of their outputs,
// y[m] = sum_s w[m][s] * D_e (silu(G_e x[m]) * (U_e x[m])), e = ids[m][s], in two launches.
//
// The first one makes h = bf16(silu(g) * u) for every pair of a token and an expert: a workgroup takes gate
// rows and the up rows beside them of one expert, for all tokens that chose it, so that every weight is read
// once.  The second one makes y: a workgroup takes 16 or 64 output rows, its waves the experts in turn, or
// slices of one where there are fewer experts than waves; the sums over experts stay in LDS, one copy per wave,
// and are added in wave order.  Where a row tile's experts are more than its waves can do with little in
// flight, up to four workgroups share them: they leave their sums in the workspace, and the last to arrive adds
// them in their order.  No sum's order depends on timing.  Products: mx_rows.h.  A token or a few that share
// few experts take another way, by dot products (below).
//
// h is rounded to bf16, the operand type of the second product (as nvq_silu_mul_bf16 rounds it for the layers
// of single calls): a relative error of up to 2^-8 in each of its values, 0.0016 in y on the average (y in bf16
// 0.0023 with it, 0.0017 without).  Two bf16 terms would hold it, with twice the reads of h and twice the
// products of the second launch.
//
// Bound: the chosen experts' weights, each read once.  Captured calls, one after the other, the same weights
// each time (and weights that no cache holds).  Microscaled, 32 experts of 4096 x 1792, 32 tokens, four experts
// each: 373 MB in 82 us (83; first launch 52, second 33), 4.5 TB/s; int4 (396 MB) 99 us (99).  One token, eight
// experts of 2048 x 1024: 28 MB in 9.1 us (12.1; int4) and 27 MB in 7.9 (10.2; microscaled), two launches (an
// empty one 2.4 from the host), each a chain of ids -> weights -> sums.
#include "mx_rows.h"
#include "transform.h"

namespace nvq {

namespace {

constexpr int kMaxParts = 4, kMaxPairs = NVQ_MAX_M * NVQ_MOE_MAX_TOP_K, kMaxChunks = kMaxPairs / 64;

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
    int parts;           // of the second launch
    float *partial;      // [row tiles][parts][M][rows of a tile]
    uint32_t *arrived;   // [row tiles]
    void *y;
    int y_dtype;
};

__device__ __forceinline__ int token_of(const MoeArgs &a, int pair) { return (int)((uint32_t)pair * a.per_token >> 16); }

// The tokens of one expert in ascending order, spread over a wave: lane n of a lane-row has number 16 t + n of
// them for t = 0, 1 (past the end: the first one's), the pair of its first slot and the sum of its slots'
// weights.
struct ExpertTokens {
    int count, first;  // first: the lowest pair
    int token[2], pair[2];
    float weight[2];
};

// Up to 64 pairs, one in each lane: those of the expert one after the other.
__device__ __forceinline__ ExpertTokens tokens_of(const MoeArgs &a, int id, float weight, int e) {
    const int n = threadIdx.x & 15;
    ExpertTokens et = {0, -1, {0, 0}, {0, 0}, {0.0f, 0.0f}};
    int previous = -1;
    for (uint64_t here = __ballot(id == e); here; here &= here - 1) {  // (uniform)
        const int p = __builtin_ctzll(here), m = token_of(a, p);
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), p));
        if (m != previous) {
            previous = m;
            if (et.count == 0) {
                et.first = p;
                et.token[0] = et.token[1] = m;
                et.pair[0] = et.pair[1] = p;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (16 * k + n == et.count) {
                    et.token[k] = m;
                    et.pair[k] = p;
                }
            ++et.count;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) et.weight[k] += 16 * k + n == et.count - 1 ? w : 0.0f;
    }
    return et;
}

// More pairs, id_of(t) and weight_of(t) giving the lane's of chunk t: each that is its token's first with the
// expert finds its number by counting those below, and sends itself to the lane of that number.  (One after the
// other, 25 tokens' 200 pairs of twelve experts took a seventh of 29 us.)
template <typename IDS, typename WEIGHTS>
__device__ __forceinline__ ExpertTokens tokens_of(const MoeArgs &a, int e, IDS id_of, WEIGHTS weight_of) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // (what follows from it is not kept in registers from expert to expert)
    const int n = lane & 15;
    const uint64_t lower = ((uint64_t)1 << lane) - 1;
    int count = 0, listed = 0;  // listed: in lane i the i-th token's pair, plus one
    float weight = 0.0f;
    uint64_t previous = 0;
#pragma unroll
    for (int t = 0; t < kMaxChunks; ++t) {
        if (64 * t >= a.pairs) break;  // (uniform)
        const uint64_t here = __ballot(id_of(t, lane) == e);
        if (here) {  // (uniform)
            const int p = 64 * t + lane, start = token_of(a, p) * a.top_k - 64 * t;  // the lane of the token's first slot
            const bool again = (here & lower & (start > 0 ? ~(uint64_t)0 << start : ~(uint64_t)0)) != 0 ||
                               (start < 0 && previous >> (64 + start) != 0);
            const bool first = (here >> lane & 1) && !again;
            const uint64_t firsts = __ballot(first);
            const float w = weight_of(t, lane);
            const int to = first ? count + __builtin_popcountll(firsts & lower) : 63;  // (63: none; there are 32 tokens)
            listed |= __builtin_amdgcn_ds_permute(4 * to, p + 1);
            weight = __uint_as_float(__float_as_uint(weight) |
                                     (uint32_t)__builtin_amdgcn_ds_permute(4 * to, (int)__float_as_uint(w)));
            for (uint64_t more = here & ~firsts; more; more &= more - 1) {  // (an expert in several slots of a token)
                const int bit = __builtin_ctzll(more);
                const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), bit));
                if (lane == count + __builtin_popcountll(firsts & (((uint64_t)1 << bit) - 1)) - 1) weight += other;
            }
            count += __builtin_popcountll(firsts);
        }
        previous = here;
    }
    ExpertTokens et;
    et.count = count;
    et.first = __builtin_amdgcn_readfirstlane(listed) - 1;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int from = 16 * k + n < count ? 16 * k + n : 0;
        et.pair[k] = __shfl(listed, from, 64) - 1;
        et.token[k] = token_of(a, et.pair[k]);
        et.weight[k] = __shfl(weight, from, 64);
    }
    return et;
}

// The tokens of a first launch's expert.
template <bool SMALL>
__device__ __forceinline__ ExpertTokens own_tokens(const MoeArgs &a, int e) {
    const int lane = threadIdx.x & 63;
    if constexpr (SMALL) {
        return tokens_of(a, lane < a.pairs ? a.ids[lane] : -1, 0.0f, e);
    } else {
        int id[kMaxChunks];
#pragma unroll
        for (int t = 0; t < kMaxChunks; ++t) id[t] = 64 * t + lane < a.pairs ? a.ids[64 * t + lane] : -1;
        return tokens_of(a, e, [&](int t, int) { return id[t]; }, [](int, int) { return 0.0f; });
    }
}

// The second launch's arrival counters, zero before it begins.
__device__ __forceinline__ void clear_arrivals(const MoeArgs &a) {
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < a.K / 16; i += blockDim.x) a.arrived[i] = 0;
}

// A workgroup takes 16 gate rows and the up rows beside them, its KS waves share out K, T token tiles at a time.
template <int FMT, int T, int KS, int C, bool SMALL>
__global__ __launch_bounds__(64 * KS) void moe_gate_up_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int s = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    clear_arrivals(a);
    // the second grid axis: experts, or pairs where there are fewer (a pair that is not the first of its expert has
    // nothing to do)
    const bool by_expert = a.E <= a.pairs;
    const int e = by_expert ? (int)blockIdx.y : a.ids[blockIdx.y];
    if ((uint32_t)e >= (uint32_t)a.E) return;
    const ExpertTokens et = own_tokens<SMALL>(a, e);
    if (et.count == 0 || (!by_expert && et.first != (int)blockIdx.y)) return;
    const int row0 = blockIdx.x * 16, G = a.K / 32;
    const int64_t row = (int64_t)e * 2 * a.F + row0 + n;
    const RowAt at[2] = {row_at<FMT>(a.gu_q, a.gu_s, row, G), row_at<FMT>(a.gu_q, a.gu_s, row + a.F, G)};
    // (T == 1: an expert of more than 16 tokens reads its weights twice)
    for (int t0 = 0; 16 * t0 < et.count; t0 += T) {
        const char *x[T];
        float4v sum[2][T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            x[t] = reinterpret_cast<const char *>(a.x) + (int64_t)(t0 + t ? et.token[1] : et.token[0]) * a.K * 2;
            sum[0][t] = sum[1][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        }
        rows_times_tokens<FMT, 2, T, C, C>(at, x, G, s, KS, sum);
        __shared__ float4v red[KS - 1][2][T][64];
        if (s > 0) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                red[s - 1][0][t][lane] = sum[0][t];
                red[s - 1][1][t][lane] = sum[1][t];
            }
        }
        __syncthreads();
        if (s == 0) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
#pragma unroll
                for (int k = 0; k < KS - 1; ++k) {
                    sum[0][t] += red[k][0][t][lane];
                    sum[1][t] += red[k][1][t][lane];
                }
                const int mine = t0 + t ? et.pair[1] : et.pair[0];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int pair = __shfl(mine, 4 * kb + j, 64);
                    if (16 * (t0 + t) + 4 * kb + j < et.count)
                        a.h[(int64_t)pair * a.F + row0 + n] = float_to_bf16_bits(silu_mul_one(sum[0][t][j], sum[1][t][j]));
                }
            }
        }
        __syncthreads();
    }
}

// The same for experts of many rows: wave w of W keeps the activations of C columns of the expert's tokens in
// registers and the workgroup streams tiles of gate and up rows past them, two turns of both requested ahead;
// the grid's first axis shares out an expert's tiles.  The waves' sums meet in LDS, one barrier a turn; four
// waves add them, the other four in the next turn.
template <int FMT, int W, int C, bool SMALL>
__global__ __launch_bounds__(64 * W) void moe_gate_up_resident_kernel(MoeArgs a) {
    constexpr int D = 2;
    __shared__ float red[2][W][8][64];
    __shared__ int pair_of[32];
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    clear_arrivals(a);
    const bool by_expert = a.E <= a.pairs;
    const int e = by_expert ? (int)blockIdx.y : a.ids[blockIdx.y];
    if ((uint32_t)e >= (uint32_t)a.E) return;
    const ExpertTokens et = own_tokens<SMALL>(a, e);
    if (et.count == 0 || (!by_expert && et.first != (int)blockIdx.y)) return;
    if (threadIdx.x < 16) {
        pair_of[threadIdx.x] = et.pair[0];
        pair_of[16 + threadIdx.x] = et.pair[1];
    }
    const int G = a.K / 32, tiles = a.F / 16;
    const int share = 4 * C * w, b0 = share < G - 4 * C ? share : G - 4 * C;  // (G >= 4 C)
    Codes<C> codes[D][2];
    Scales<FMT, C> sc[D][2];
    auto tile_of = [&](int it) { return it * (int)gridDim.x + (int)blockIdx.x; };
    auto load = [&](int d, int it) {
        const int tile = tile_of(it) < tiles ? tile_of(it) : tiles - 1;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const RowAt at = row_at<FMT>(a.gu_q, a.gu_s, (int64_t)e * 2 * a.F + r * a.F + 16 * tile + n, G);
            const RowAt from = {at.q + b0, at.s + (int64_t)b0 * scale_bytes<FMT>()};
            load_codes<C>(codes[d][r], from, 0, kb);
            load_scales<FMT, C>(sc[d][r], from, 0);
        }
    };
    int done = 0;  // turns, for the two halves of `red`
    for (int t = 0; 16 * t < et.count; ++t) {
#pragma unroll
        for (int d = 0; d < D; ++d) load(d, d);
        const char *const xt = reinterpret_cast<const char *>(a.x) + (int64_t)(t ? et.token[1] : et.token[0]) * a.K * 2;
        bf16x8 x[C][1][4];
#pragma unroll
        for (int b = 0; b < C; ++b) {
            uint4v raw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int block = b0 + 4 * b + (FMT == NVQ_FMT_MXFP4 ? kb : i);
                raw[i] = uint4v{0, 0, 0, 0};
                if (block >= share && 16 * t + n < et.count)
                    raw[i] = *as_global<uint4v>(xt + (b0 + 4 * b) * 64 + piece_at<FMT>(i, kb));
            }
            to_operands<FMT>(raw, x[b][0]);
        }
        auto one = [&](int d, int it) {
            float4v sum[2][1] = {{float4v{0.0f, 0.0f, 0.0f, 0.0f}}, {float4v{0.0f, 0.0f, 0.0f, 0.0f}}};
            if (b0 < share) {  // (uniform)
                clear_scales<FMT, C>(sc[d][0], share - b0);
                clear_scales<FMT, C>(sc[d][1], share - b0);
            }
#pragma unroll
            for (int b = 0; b < C; ++b) multiply_column<FMT, 2, 1, C, C>(codes[d], b, sc[d], b, x[b], sum);
            load(d, it + D);
            float(&to)[W][8][64] = red[done & 1];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                wait_written(sum[r][0]);
#pragma unroll
                for (int j = 0; j < 4; ++j) to[w][4 * r + j][lane] = sum[r][0][j];
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int j = (w + W - (done * 4) % W) % W;  // (uniform)
            if (j < 4) {
                float g = 0.0f, u = 0.0f;
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    g += to[k][j][lane];
                    u += to[k][4 + j][lane];
                }
                const int number = 16 * t + 4 * kb + j;
                if (number < et.count)
                    a.h[(int64_t)pair_of[number] * a.F + 16 * tile_of(it) + n] = float_to_bf16_bits(silu_mul_one(g, u));
            }
            ++done;
        };
        for (int it = 0; tile_of(it) < tiles; it += D) {
            one(0, it);
            if (tile_of(it + 1) >= tiles) break;
            one(1, it + 1);
        }
    }
}

// A workgroup takes 16 R rows of the outputs; the row tiles' experts, or slices of them, are shared out among
// the waves of a.parts workgroups.  (R = T = 1: within 128 registers, so that two workgroups run on a compute
// unit; with 129 one token's eight experts took 17.4 us for 14.6.)
template <int FMT, int R, int T, int W, int C, bool SMALL>
__global__ __launch_bounds__(64 * W, R * T == 1 ? 4 : 1) void moe_down_kernel(MoeArgs a) {
    constexpr int kTokens = SMALL ? 16 : NVQ_MAX_M;
    constexpr int kOut = kTokens * R * 16;  // a wave's sums
    __shared__ float out[W][kOut];
    __shared__ uint32_t chosen[NVQ_MOE_MAX_EXPERTS / 32];
    __shared__ uint32_t last;
    constexpr int kListed = SMALL ? 1 : kMaxPairs;
    __shared__ int ids[kListed];
    __shared__ float weights[kListed];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    const int row0 = blockIdx.x * (16 * R), part = blockIdx.y;
    int my_id = -1;  // SMALL: the lane's pair
    float my_weight = 0.0f;
    if (SMALL && lane < a.pairs) {
        my_id = a.ids[lane];
        my_weight = a.weights[lane];
    }
    // the experts that some token chose, a bit for each
    if (threadIdx.x < NVQ_MOE_MAX_EXPERTS / 32) chosen[threadIdx.x] = 0;
    for (int i = lane; i < kOut; i += 64) out[w][i] = 0.0f;
    __syncthreads();
    if constexpr (SMALL) {
        if (w == 0 && (uint32_t)my_id < (uint32_t)a.E) atomicOr(&chosen[my_id >> 5], 1u << (my_id & 31));
    } else {
        for (int p = threadIdx.x; p < kMaxPairs; p += 64 * W) {
            const int e = p < a.pairs ? a.ids[p] : -1;
            ids[p] = e;
            weights[p] = p < a.pairs ? a.weights[p] : 0.0f;
            if ((uint32_t)e < (uint32_t)a.E) atomicOr(&chosen[e >> 5], 1u << (e & 31));
        }
    }
    __syncthreads();
    const uint32_t word = chosen[lane & (NVQ_MOE_MAX_EXPERTS / 32 - 1)];
    const int words = (a.E + 31) >> 5;
    int active = 0;
    for (int i = 0; i < words; ++i) active += __builtin_popcount((uint32_t)__builtin_amdgcn_readlane((int)word, i));
    // The workgroups of all parts share the experts out among their waves; where there are more waves than
    // experts, each in `split` slices of its inputs.
    const int workers = a.parts * W, G = a.F / 32;
    int split = active == 0 || active >= workers ? 1 : (workers + active - 1) / active;
    const int passes = (G + 4 * C - 1) / (4 * C);
    split = split < passes ? split : passes;
    for (int item = part * W + w; item < active * split; item += workers) {  // (uniform)
        int skip = item / split, e = 0;
        for (int i = 0; i < words; ++i) {
            uint32_t bits = (uint32_t)__builtin_amdgcn_readlane((int)word, i);
            const int count = __builtin_popcount(bits);
            if (skip >= count) {
                skip -= count;
                continue;
            }
            for (; skip > 0; --skip) bits &= bits - 1;
            e = 32 * i + __builtin_ctz(bits);
            break;
        }
        e = __builtin_amdgcn_readfirstlane(e);
        ExpertTokens et;
        if constexpr (SMALL)
            et = tokens_of(a, my_id, my_weight, e);
        else
            et = tokens_of(
                a, e, [&](int t, int l) { return ids[64 * t + l]; }, [&](int t, int l) { return weights[64 * t + l]; });
        RowAt at[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            at[r] = row_at<FMT>(a.dn_q, a.dn_s, (int64_t)e * a.K + row0 + 16 * r + n, G);
        for (int t0 = 0; 16 * t0 < et.count; t0 += T) {
            const char *h[T];
            float4v sum[R][T];
#pragma unroll
            for (int t = 0; t < T; ++t) {
                h[t] = reinterpret_cast<const char *>(a.h) + (int64_t)(t0 + t ? et.pair[1] : et.pair[0]) * a.F * 2;
#pragma unroll
                for (int r = 0; r < R; ++r) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            }
            rows_times_tokens<FMT, R, T, C, C>(at, h, G, item % split, split, sum);
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int m = __shfl(t0 + t ? et.token[1] : et.token[0], 4 * kb + j, 64);
                    const float wt = __shfl(t0 + t ? et.weight[1] : et.weight[0], 4 * kb + j, 64);
                    if (16 * (t0 + t) + 4 * kb + j < et.count) {
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            float *const o = &out[w][(m * R + r) * 16 + n];
                            *o = fmaf(wt, sum[r][t][j], *o);
                        }
                    }
                }
        }
    }
    __syncthreads();
    float *const mine = a.partial + ((int64_t)blockIdx.x * a.parts + part) * (a.M * R * 16);
    for (int i = threadIdx.x; i < a.M * R * 16; i += 64 * W) {
        float v = out[0][i];
#pragma unroll
        for (int k = 1; k < W; ++k) v += out[k][i];
        if (a.parts == 1)
            store_global(a.y, a.y_dtype, (int64_t)(i / (R * 16)) * a.K + row0 + i % (R * 16), v);
        else
            __hip_atomic_store(mine + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (a.parts == 1) return;
    // The parts' sums are added, in their order, by the workgroup that arrives last: they are written through
    // to where all XCDs see them before it arrives, and read past its caches.
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
    if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(&a.arrived[blockIdx.x], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
               (uint32_t)a.parts - 1;
    __syncthreads();
    if (!last) return;
    const float *const all = a.partial + (int64_t)blockIdx.x * a.parts * (a.M * R * 16);
    for (int i = threadIdx.x; i < a.M * R * 16; i += 64 * W) {
        float v[kMaxParts];
#pragma unroll
        for (int k = 0; k < kMaxParts; ++k)
            v[k] = __hip_atomic_load(all + (int64_t)(k < a.parts ? k : 0) * (a.M * R * 16) + i, __ATOMIC_RELAXED,
                                     __HIP_MEMORY_SCOPE_AGENT);
        float s = v[0];
#pragma unroll
        for (int k = 1; k < kMaxParts; ++k) s += k < a.parts ? v[k] : 0.0f;
        store_global(a.y, a.y_dtype, (int64_t)(i / (R * 16)) * a.K + row0 + i % (R * 16), s);
    }
}

// ---- few pairs: by dot products ----
//
// With a token or two the matrix cores' way reads activations for sixteen, four loads for each one of weights.
// Here a lane keeps the activations of its blocks in registers and takes its blocks of R rows, so that nothing
// but weights is asked for.  Every pair of a token and a slot is worked off by itself (an expert that two
// tokens chose is read twice).

// The dot product of a block's 32 weights with the lane's activations, x[k] inputs 2 k and 2 k + 1, added to
// `sum`.  int4: a nibble n stands for n - 8 and goes in as bf16 128 + n (exact); `offset`, -136 times the sum
// of the activations, takes the rest away.
template <int FMT>
__device__ __forceinline__ float block_dot(const uint4v &codes, uint32_t scale, const uint32_t (&x)[16], float offset,
                                           float sum) {
    auto dot = [](uint32_t a, uint32_t b, float c) {
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(nvq_bf16x2, a), __builtin_bit_cast(nvq_bf16x2, b), c, false);
    };
    if constexpr (FMT == NVQ_FMT_MXFP4) {
        const float s = __uint_as_float(scale << 23);  // (the conversions look at the exponent alone)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4v v = __builtin_bit_cast(uint4v, mx_values(codes[i], s));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t two = v[k];
                sum = dot(two, x[4 * i + k], sum);
            }
        }
        return sum;
    } else {
        float v = offset;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = codes[i] & 0x0f0f0f0fu, hi = (codes[i] >> 4) & 0x0f0f0f0fu;  // inputs 4 i .., 16 + 4 i ..
            v = dot(__builtin_amdgcn_perm(0x43434343u, lo, 0x04010400u), x[2 * i], v);
            v = dot(__builtin_amdgcn_perm(0x43434343u, lo, 0x04030402u), x[2 * i + 1], v);
            v = dot(__builtin_amdgcn_perm(0x43434343u, hi, 0x04010400u), x[8 + 2 * i], v);
            v = dot(__builtin_amdgcn_perm(0x43434343u, hi, 0x04030402u), x[9 + 2 * i], v);
        }
        return fmaf(half_bits_to_float((uint16_t)scale), v, sum);
    }
}
template <int FMT>
__device__ __forceinline__ float block_offset(const uint32_t (&x)[16]) {
    float s = 0.0f;
    if constexpr (FMT == NVQ_FMT_INT4) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(nvq_bf16x2, 0x3f803f80u), __builtin_bit_cast(nvq_bf16x2, x[k]),
                                                s, false);
        s *= -136.0f;
    }
    return s;
}
// A block's activations (64 bytes), or zeros.
__device__ __forceinline__ void load_block(const uint16_t *from, bool there, uint32_t (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4v v = {0, 0, 0, 0};
        if (there) v = as_global<uint4v>(from)[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * i + k] = v[k];
    }
}
// ... and a block's codes and scale, or zeros (which stand for zero, whatever the place holds).
template <int FMT>
__device__ __forceinline__ void load_weights(const uint8_t *q, const void *s, int64_t at, bool there, uint4v &codes,
                                             uint32_t &scale) {
    codes = uint4v{0, 0, 0, 0};
    scale = 0;
    if (there) {
        codes = load_stream(reinterpret_cast<const uint4 *>(q) + at);
        scale = FMT == NVQ_FMT_MXFP4 ? as_global<uint8_t>(s)[at] : as_global<uint16_t>(s)[at];
    }
}

// h of pair blockIdx.y: a wave takes R gate rows and the up rows beside them, a lane the blocks l, 64 + l ..
template <int FMT, int B, int R>
__global__ __launch_bounds__(256) void moe_gate_up_dot_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int pair = blockIdx.y, e = a.ids[pair], f0 = ((int)blockIdx.x * 4 + w) * R, G = a.K / 32;
    if ((uint32_t)e >= (uint32_t)a.E) return;
    uint4v c[2 * R][B];
    uint32_t sc[2 * R][B];
#pragma unroll
    for (int r = 0; r < 2 * R; ++r) {
        const int64_t row = (int64_t)e * 2 * a.F + (r & 1 ? a.F : 0) + f0 + (r >> 1);  // (F is a multiple of 4 R)
#pragma unroll
        for (int b = 0; b < B; ++b)
            load_weights<FMT>(a.gu_q, a.gu_s, row * G + 64 * b + lane, 64 * b + lane < G, c[r][b], sc[r][b]);
    }
    uint32_t x[B][16];
    float offset[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        load_block(a.x + ((int64_t)token_of(a, pair) * G + 64 * b + lane) * 32, 64 * b + lane < G, x[b]);
        offset[b] = block_offset<FMT>(x[b]);
    }
    float g = 0.0f, u = 0.0f;  // of row f0 + lane
#pragma unroll
    for (int r = 0; r < 2 * R; ++r) {
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < B; ++b) sum = block_dot<FMT>(c[r][b], sc[r][b], x[b], offset[b], sum);
        sum = group_sum<64>(sum);
        if (r & 1)
            u = lane == r >> 1 ? sum : u;
        else
            g = lane == r >> 1 ? sum : g;
    }
    if (lane < R) a.h[(int64_t)pair * a.F + f0 + lane] = float_to_bf16_bits(silu_mul_one(g, u));
}

// y of token blockIdx.y: the token's pairs as one product, whose blocks are those of h of all its slots, 256 B
// of them, shared out among the lanes of four waves.  Each block's product is weighted with its pair's weight
// on its way into the row's sum.
template <int FMT, int B, int R>
__global__ __launch_bounds__(256) void moe_down_dot_kernel(MoeArgs a) {
    __shared__ float red[4][R];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m = blockIdx.y, row0 = blockIdx.x * R, G = a.F / 32;
    uint4v c[R][B];
    uint32_t sc[R][B], h[B][16];
    float weight[B], offset[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int unit = 256 * b + (int)threadIdx.x, slot = unit / G, block = unit - slot * G;
        const int pair = m * a.top_k + (slot < a.top_k ? slot : 0);
        const int e = a.ids[pair];
        const bool there = slot < a.top_k && (uint32_t)e < (uint32_t)a.E;
        weight[b] = there ? a.weights[pair] : 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            load_weights<FMT>(a.dn_q, a.dn_s, ((int64_t)e * a.K + row0 + r) * G + block, there, c[r][b], sc[r][b]);
        load_block(a.h + ((int64_t)pair * G + block) * 32, there, h[b]);
        offset[b] = block_offset<FMT>(h[b]);
    }
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < B; ++b) sum = fmaf(weight[b], block_dot<FMT>(c[r][b], sc[r][b], h[b], offset[b], 0.0f), sum);
        sum = group_sum<64>(sum);
        mine = lane == r ? sum : mine;
    }
    if (lane < R) red[w][lane] = mine;
    __syncthreads();
    if (w == 0 && lane < R)
        store_global(a.y, a.y_dtype, (int64_t)m * a.K + row0 + lane,
                     red[0][lane] + red[1][lane] + red[2][lane] + red[3][lane]);
}

constexpr int kColumns = 2;    // of a pass (rows_times_tokens)
constexpr int kDownWaves = 8;  // of a workgroup of the second launch

// The second launch in tiles of 64 outputs (32 with two token tiles), four row tiles reading a token's h at
// once, where that leaves a workgroup to each compute unit: 4096 outputs of 32 experts 32 us against 44
// microscaled, 38 against 47 int4; 2048 outputs, half the workgroups: 26 against 17.
bool wide_down(const MoeArgs &a, int parts) {
    return a.K / 16 % 4 == 0 && (int64_t)(a.K / 64) * parts >= device_cu_count();
}

// Workgroups that share a row tile of the second launch: as many as leave each wave a pass (over the experts
// that the tokens can choose), or two passes where a pass would be more than two workgroups to each compute
// unit.  Two experts of 4096 outputs, 14 passes: 5.1 us with one, 6.2 with two, 7.7 with four; 23 of 28 experts
// of 992 outputs, 23 passes: both launches 18.2 with one, 13.5 with two; 43 of 64 experts of 2048, 172 passes:
// 26.5 with one, 18.3 with two, 16.9 with four.
int parts_of(const MoeArgs &a) {
    const int experts = a.E <= a.pairs ? a.E : a.pairs, passes = (a.F + 128 * kColumns - 1) / (128 * kColumns);
    const auto within = [](int v) { return v < 1 ? 1 : v < kMaxParts ? v : kMaxParts; };
    const int most = within(experts * passes / kDownWaves), least = within(experts * passes / (2 * kDownWaves));
    if (wide_down(a, most)) return most;
    const int room = 2 * device_cu_count() / (a.K / 16);
    return room < least ? least : room < most ? room : most;
}

// SMALL: up to 64 pairs and 16 tokens.  T: token tiles at a time.
template <int FMT, int T, bool SMALL>
int launch_experts(const MoeArgs &a, hipStream_t st) {
    const int experts = a.E <= a.pairs ? a.E : a.pairs, tiles = a.F / 16, out_tiles = a.K / 16;
    const int cus = device_cu_count();
    // Activations in registers: K <= 4096, which is what eight waves of four columns hold, and K > 2048, so
    // that each has most of them; an expert for most workgroups that are launched (three choices for each on
    // the average leave one in twenty without); eight tiles for each compute unit.  32 experts of 4096 x 1792,
    // 32 tokens: 53 us against 68 microscaled, 65 against 73 int4.  Not for fewer inputs: 64 experts of 2048 x
    // 1024 with half the columns to a wave took 24 us against 20.
    bool resident = false;
    if constexpr (T == 1) {
        resident = a.K > 2048 && a.K <= 4096 && 3 * a.E <= a.pairs && (int64_t)a.E * tiles >= 8 * cus;
        const unsigned slices = (unsigned)(a.E < cus ? cus / a.E : 1);
        if (resident)
            hipLaunchKernelGGL((moe_gate_up_resident_kernel<FMT, 8, 4, SMALL>), dim3(slices, a.E), dim3(512), 0, st, a);
    }
    if (!resident)
        hipLaunchKernelGGL((moe_gate_up_kernel<FMT, T, 4, kColumns, SMALL>), dim3(tiles, experts), dim3(256), 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    constexpr int kWide = T == 1 ? 4 : 2;
    const dim3 block(64 * kDownWaves);
    if (wide_down(a, a.parts))
        hipLaunchKernelGGL((moe_down_kernel<FMT, kWide, T, kDownWaves, kColumns, SMALL>), dim3(out_tiles / kWide, a.parts), block,
                           0, st, a);
    else
        hipLaunchKernelGGL((moe_down_kernel<FMT, 1, T, kDownWaves, kColumns, SMALL>), dim3(out_tiles, a.parts), block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

// Where dot products are worked off: up to eight tokens, few of whose experts are shared; K and a token's slots
// (blocks of h) that fit the lanes.  us, by dot products and on the matrix cores; tokens, experts of each and
// in all, inputs, F:
//                              int4          microscaled                                int4          microscaled
//   1, 8 of 64, 2048, 1024  10.7  13.8      8.0  12.5      4, 8 of 32, 2048, 1024  29.3  29.9     19.1  23.9
//   2, 8 of 64, 2048, 1024  18.7  20.8     13.0  17.8      4, 8 of 32, 4096, 1024  53.0  46.1     41.2  41.3
//   3, 8 of 64, 2048, 1024  24.1  27.5     17.4  23.4      5, 4 of 20, 2048, 1024  21.2  20.7     15.2  17.7
//   3, 4 of 12, 2048, 1024  12.4  17.0      9.6  12.6      6, 4 of 40, 2048, 1024  25.4  27.3     18.4  23.2
//   4, 8 of 64, 2048, 1024  30.1  31.0     20.6  29.5      7, 3 of 40, 1440, 992   21.8  26.5     15.5  18.0
//   4, 4 of 16, 2048, 768   13.4  16.4     10.8  14.1      8, 8 of 64, 2048, 1024  52.6  44.8     32.9  38.7
//   4, 6 of 24, 1024, 512   10.4  12.2      8.6  11.0      8, 4 of 32, 4096, 1792  77.5  71.4     59.1  55.3
// So int4 of up to four tokens and 2048 inputs, microscaled of all up to 2048.  (Three tokens of 4096 inputs
// that choose all of twelve experts lose, int4 39.2 and 32.6; eight tokens, two of eight 16.1 and 13.1: more
// pairs than experts; seven tokens whose slots are four blocks 12.5 and 9.7: fewer blocks than lanes.)
template <int FMT>
bool by_dot_products(const MoeArgs &a) {
    const int blocks = a.top_k * (a.F / 32);
    if (a.M > 8 || a.pairs > a.E || a.K > 4096 || blocks < 64 || blocks > 512) return false;
    return a.M <= 3 || 8 * a.pairs <= 5 * a.E || (a.K <= 2048 && (a.M == 4 || FMT == NVQ_FMT_MXFP4));
}

template <int FMT>
int launch_experts_dot(const MoeArgs &a, hipStream_t st) {
    // gate rows to a wave, outputs to a workgroup (one and two, or four and eight: 2 to 12 % more)
    constexpr int kRows = 2, kOut = 4;
    const dim3 grid(a.F / (4 * kRows), a.pairs), out(a.K / kOut, a.M), block(256);
    if (a.K <= 2048)
        hipLaunchKernelGGL((moe_gate_up_dot_kernel<FMT, 1, kRows>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((moe_gate_up_dot_kernel<FMT, 2, kRows>), grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    if (a.top_k * (a.F / 32) <= 256)
        hipLaunchKernelGGL((moe_down_dot_kernel<FMT, 1, kOut>), out, block, 0, st, a);
    else
        hipLaunchKernelGGL((moe_down_dot_kernel<FMT, 2, kOut>), out, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

template <int FMT>
int launch_experts(const MoeArgs &a, hipStream_t st) {
    if (by_dot_products<FMT>(a)) return launch_experts_dot<FMT>(a, st);
    if (a.pairs <= 64 && a.M <= 16) return launch_experts<FMT, 1, true>(a, st);
    // Two token tiles at once where most experts have more than 16 tokens: 16 experts of 4096 x 1792
    // microscaled, 16 tokens each on the average, 90 us against 101; with twelve 78 against 65.
    return a.pairs >= 14 * a.E ? launch_experts<FMT, 2, false>(a, st) : launch_experts<FMT, 1, false>(a, st);
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

namespace {

// The workspace: h, the parts' sums, the counters.
struct MoeRooms {
    size_t h, partial, arrived, all;
};
MoeRooms moe_rooms(const nvq_experts *e, int M, int top_k) {
    const auto whole = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    MoeRooms r;
    r.h = 0;
    r.partial = r.h + whole((size_t)M * top_k * e->F * sizeof(uint16_t));
    r.arrived = r.partial + whole(sizeof(float) * nvq::kMaxParts * (size_t)M * e->K);
    r.all = r.arrived + whole(sizeof(uint32_t) * (e->K / 16));
    return r;
}

}  // namespace

extern "C" size_t nvq_moe_workspace_bytes(const nvq_experts *experts, int M, int top_k) {
    if (nvq::check_experts(experts, M, top_k) != NVQ_OK) return 0;
    return moe_rooms(experts, M, top_k).all;
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
    const MoeRooms rooms = moe_rooms(experts, M, top_k);
    a.h = static_cast<uint16_t *>(workspace);
    a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + rooms.partial);
    a.arrived = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + rooms.arrived);
    a.parts = parts_of(a);
    a.y = y;
    a.y_dtype = y_dtype;
    const hipStream_t st = (hipStream_t)stream;
    return experts->format == NVQ_FMT_INT4 ? launch_experts<NVQ_FMT_INT4>(a, st) : launch_experts<NVQ_FMT_MXFP4>(a, st);
}
