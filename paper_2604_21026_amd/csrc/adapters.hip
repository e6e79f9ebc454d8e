// nvq_adapters_add: low-rank adapters beside a layer, each token its own.
//
// Two launches, h = A x and y + scale * B h, both on the matrix cores (or one, where a workgroup's own h costs less: one_launch).  Tokens go in groups of 64, a group by the
// distinct adapters of its tokens, and the tokens of one adapter, wherever they stand in the group, are sixteen to a
// product: an adapter's weights are read once per group however its tokens lie, and 64 tokens of 64 adapters read what
// they have to.  h stays fp32 between the launches, in as many partial sums as K is cut into; it enters the second
// product as three bf16 values whose sum it is, so nothing of it is lost; the products with the first and with the rest are
// summed apart and added at the end, where what an infinite weight makes of a rest of zero is left out.
//
// Small ones are chains of trips to memory (ids, weights, sums; ids, h, results): one token of 2048 x 2048, 16 ranks, 5.8 us in one
// launch, of 4096 x 4096 6.8 in two.  With many adapters the bytes of B bound it: 32 tokens of 12 adapters of 4096 x 28672, 64
// ranks, 53 MB in 18.7 us, 2.8 TB/s; 500 tokens of prompts, 4099 outputs, 15.4 us.
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr int kGroup = 64, kTile = 16, kWaves = 4, kThreads = 64 * kWaves;
constexpr int kMostSlices = 16;

struct AdaptersArgs {
    const uint16_t *a, *b, *x;
    const float *scales;
    const int32_t *ids;
    const void *y;
    void *out;
    int dtype;
    int n, K, N, R, M;
    float *h;             // workspace, [slices][M][R]
    int slices, columns;  // of K, 32 inputs each
    int workers;          // workgroups that take a group's tiles in turn
    int copiers;          // one more for its tokens without an adapter, or none: the same ones do
    int blocks;           // of ranks (first launch)
    int turns;            // workgroups that share the outputs (second)
};

// The adapter of a lane's token, -1: none.
__device__ __forceinline__ int adapter_of(const AdaptersArgs &g, int m0) {
    const int m = m0 + (threadIdx.x & 63);
    const int e = m < g.M ? g.ids[m] : -1;
    return (unsigned)e < (unsigned)g.n ? e : -1;
}

// A group's tiles, of sixteen tokens of one adapter or fewer, are counted through, and its workers take them in turn: however
// the tokens lie, all have work.
//
// The distinct adapters of a group one after the other: `left` has a bit per token that has not had its turn.
__device__ __forceinline__ uint64_t turn(int mine, uint64_t *left, int *e) {
    *e = __builtin_amdgcn_readlane(mine, __builtin_ctzll(*left));
    const uint64_t with = __ballot(mine == *e);
    *left &= ~with;
    return with;
}

// The place of the k-th bit that is set (k from 0, below their number).
__device__ __forceinline__ int nth_bit(uint64_t bits, int k) {
    int at = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1) {
        const int c = __builtin_popcountll(bits >> at & ((1ull << step) - 1));
        if (k >= c) {
            k -= c;
            at += step;
        }
    }
    return at;
}

// A wave's share of h of one tile: columns c0 + w, c0 + w + W, .. before c1 of 32 inputs each, x of the lane's token and a of its
// ranks; AT_ONCE columns whose loads are in flight together.
template <int RT, int W, int AT_ONCE>
__device__ __forceinline__ void down_products(const uint16_t *x, const uint16_t *const (&a)[RT], int c0, int c1, float4v (&sum)[RT]) {
#pragma unroll
    for (int t = 0; t < RT; ++t) sum[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = c0 + (int)(threadIdx.x >> 6); c < c1; c += AT_ONCE * W) {
        uint4v xv[AT_ONCE], av[AT_ONCE][RT];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int cc = c + k * W < c1 ? c + k * W : c;
            xv[k] = *as_global<uint4v>(x + 32 * cc);
#pragma unroll
            for (int t = 0; t < RT; ++t) av[k][t] = *as_global<uint4v>(a[t] + 32 * cc);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const bool in = c + k * W < c1;
            if (!in) xv[k] = uint4v{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (!in) av[k][t] = uint4v{0, 0, 0, 0};
                sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[k]),
                                                                __builtin_bit_cast(bf16x8, av[k][t]), sum[t], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) wait_written(sum[t]);
}

// h of a group's tokens: RT tiles of sixteen ranks, a slice of K, its columns in turn over the waves.
template <int RT>
__global__ __launch_bounds__(kThreads) void adapters_down_kernel(AdaptersArgs g) {
    __shared__ float red[kWaves][RT * 4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    int i = blockIdx.x;
    const int slice = i % g.slices;
    i /= g.slices;
    const int r0 = i % g.blocks * 16 * RT;
    i /= g.blocks;
    const int worker = i % g.workers, m0 = i / g.workers * kGroup;
    const int c0 = slice * g.columns, c1 = c0 + g.columns < g.K / 32 ? c0 + g.columns : g.K / 32;
    const int mine = adapter_of(g, m0);
    uint64_t left = __ballot(mine >= 0);
    for (int next = worker, base = 0, end; left; base = end) {
        int e;
        const uint64_t with = turn(mine, &left, &e);
        const int tokens = __builtin_popcountll(with);
        end = base + (tokens + kTile - 1) / kTile;
        if (next >= end) continue;
        const uint16_t *a[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int r = r0 + 16 * t + n < g.R ? r0 + 16 * t + n : g.R - 1;
            a[t] = g.a + ((int64_t)e * g.R + r) * g.K + 8 * kb;
        }
        for (; next < end; next += g.workers) {
            const int k0 = (next - base) * kTile;
            const int m = m0 + nth_bit(with, k0 + n < tokens ? k0 + n : k0);
            const uint16_t *const x = g.x + (int64_t)m * g.K + 8 * kb;
            float4v sum[RT];
            down_products<RT, kWaves, RT == 4 ? 2 : 4>(x, a, c0, c1, sum);
            __syncthreads();
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) red[w][4 * t + j][lane] = sum[t][j];
            __syncthreads();
            for (int o = threadIdx.x; o < RT * 256; o += kThreads) {
                const int reg = o >> 6, l = o & 63;
                const int k = k0 + 4 * (l >> 4) + (reg & 3), r = r0 + 16 * (reg >> 2) + (l & 15);
                float v = red[0][reg][l];
#pragma unroll
                for (int q = 1; q < kWaves; ++q) v += red[q][reg][l];
                if (k < tokens && r < g.R) g.h[((int64_t)slice * g.M + m0 + nth_bit(with, k)) * g.R + r] = v;
            }
        }
    }
}

// A value as three whose sum it is, each with eight bits (cut off, so that nothing grows to infinity).
__device__ __forceinline__ void split(float v, uint32_t *hi, uint32_t *mid, uint32_t *lo) {
    const uint32_t b = __float_as_uint(v) & 0xffff0000u;
    const float rest = __builtin_isfinite(v) ? v - __uint_as_float(b) : 0.0f;
    const uint32_t c = __float_as_uint(rest) & 0xffff0000u;
    *hi = b >> 16;
    *mid = c >> 16;
    *lo = __float_as_uint(rest - __uint_as_float(c)) >> 16;
}

// Results side by side as one access, at the alignment of a single one.
typedef uint4v uint4_apart __attribute__((aligned(2)));
typedef uint2v uint2_apart __attribute__((aligned(2)));
template <int COUNT>  // 4 or 16
__device__ __forceinline__ void load_results(const void *p, int dtype, int64_t at, float (&v)[COUNT]) {
    if (dtype == NVQ_F32) {
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) {
            const uint4v w = *reinterpret_cast<const uint4_apart *>(static_cast<const float *>(p) + at + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = __uint_as_float(w[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) {
            const uint2v w = *reinterpret_cast<const uint2_apart *>(static_cast<const uint16_t *>(p) + at + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
        }
    }
}
template <int COUNT>
__device__ __forceinline__ void store_results(void *p, int dtype, int64_t at, const float (&v)[COUNT]) {
    if (dtype == NVQ_F32) {
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) {
            const uint4v w = {__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
            *reinterpret_cast<uint4_apart *>(static_cast<float *>(p) + at + i) = w;
        }
    } else if constexpr (COUNT == 4) {
        const uint2v w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        *reinterpret_cast<uint2_apart *>(static_cast<uint16_t *>(p) + at) = w;
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; i += 8) {
            const uint4v w = {pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]), pack_bf16x2(v[i + 4], v[i + 5]),
                              pack_bf16x2(v[i + 6], v[i + 7])};
            *reinterpret_cast<uint4_apart *>(static_cast<uint16_t *>(p) + at + i) = w;
        }
    }
}

// Results of a group's tokens, NT tiles of sixteen outputs per wave and turn, outputs the rows of a product and tokens its
// columns.  Row 4 q + j of tile t is output 4 NT q + 4 t + j, so that a lane has 4 NT outputs side by side.  A workgroup
// takes blocks of outputs in turn with the h that it has split once, the next block's weights asked for before this
// one's results are stored.
//
// RT > 0: h, of RT tiles of sixteen ranks, is not there; every workgroup makes it for its tile, from all of A.
template <int NT, int RT, int W>
__global__ __launch_bounds__(64 * W) void adapters_up_kernel(AdaptersArgs g) {
    constexpr int kThreads = 64 * W;
    constexpr int kPitch = (RT ? 16 * RT : NVQ_MAX_RANK) + 8;  // (16 bytes more than a row, against bank conflicts)
    constexpr int kBlock = W * 16 * NT;
    __shared__ float red[RT ? W : 1][RT ? RT * 4 : 1][64];
    __shared__ __align__(16) uint16_t hs[3][kTile][kPitch];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    int first = (int)(blockIdx.x % g.turns) * kBlock, stride = g.turns * kBlock;
    int i = blockIdx.x / g.turns;
    const int all = g.workers + g.copiers, worker = i % all, m0 = i / all * kGroup;
    const int mine = adapter_of(g, m0);
    uint64_t left = __ballot(mine >= 0);
    if (g.out != g.y && (!g.copiers || worker == g.workers)) {  // tokens without an adapter stay as they are
        uint64_t none = ~left;
        if (g.M - m0 < kGroup) none &= (1ull << (g.M - m0)) - 1;
        const int count = __builtin_popcountll(none);
        const int stride_k = g.copiers ? 1 : g.workers;
        for (int k0 = g.copiers ? 0 : worker; k0 < count; k0 += 8 * stride_k) {
            int64_t row[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int at = k0 + k * stride_k;
                row[k] = at < count ? (int64_t)(m0 + nth_bit(none, at)) * g.N : -1;
            }
            for (int block = first; block < g.N; block += stride)
                for (int o = block + (int)threadIdx.x; o < block + kBlock && o < g.N; o += kThreads) {
                    uint32_t v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (row[k] < 0) continue;
                        v[k] = g.dtype == NVQ_F32 ? static_cast<const uint32_t *>(g.y)[row[k] + o] : static_cast<const uint16_t *>(g.y)[row[k] + o];
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (row[k] < 0) continue;
                        if (g.dtype == NVQ_F32)
                            static_cast<uint32_t *>(g.out)[row[k] + o] = v[k];
                        else
                            static_cast<uint16_t *>(g.out)[row[k] + o] = (uint16_t)v[k];
                    }
                }
        }
        if (g.copiers) return;
    }
    // Fewer tiles than half the workers: several workers to a tile, each with outputs of its own.
    int next = worker;
    if (!g.copiers) {
        int count = 0;
        for (uint64_t rest = left; rest;) {
            int e;
            count += (__builtin_popcountll(turn(mine, &rest, &e)) + kTile - 1) / kTile;
        }
        if (count > 0 && 2 * count <= g.workers) {
            const int each = g.workers / count, part = worker / count;
            next = part < each ? worker - part * count : count;
            first += part * stride;
            stride *= each;
        }
    }
    if (first >= g.N) return;
    const int64_t h_slice = (int64_t)g.M * g.R;
    for (int base = 0, end; left; base = end) {
        int e;
        const uint64_t with = turn(mine, &left, &e);
        const int tokens = __builtin_popcountll(with);
        end = base + (tokens + kTile - 1) / kTile;
        if (next >= end) continue;
        // The weights of two columns of 32 ranks at a time.
        uint4v bw[2][NT];
        auto load = [&](int block, int c) {
            const int n0 = block + w * 16 * NT + 4 * NT * (n >> 2) + (n & 3);
            const uint16_t *const b = g.b + (int64_t)e * g.N * g.R;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int o = n0 + 4 * t < g.N ? n0 + 4 * t : g.N - 1;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int r = c + 32 * k + 8 * kb;  // (past the last rank h is zero: any weight of the row will do that is there)
                    bw[k][t] = *as_global<uint4v>(b + (int64_t)o * g.R + (r < g.R ? r : 0));
                    if (r >= g.R) bw[k][t] = uint4v{0, 0, 0, 0};
                }
            }
        };
        load(first, 0);
        const float scale = g.scales ? g.scales[e] : 1.0f;
        for (bool again = false; next < end; next += g.workers, again = true) {
            const int k0 = (next - base) * kTile;
            const bool my = k0 + n < tokens;
            const int64_t row = (int64_t)(m0 + nth_bit(with, my ? k0 + n : k0)) * g.N;
            float y[4 * NT];
            auto load_y = [&](int block) {
                const int o0 = block + w * 16 * NT + 4 * NT * kb;
                if (my && o0 + 4 * NT <= g.N) load_results<4 * NT>(g.y, g.dtype, row + o0, y);
            };
            load_y(first);
            if constexpr (RT > 0) {
                const uint16_t *a[RT];
#pragma unroll
                for (int t = 0; t < RT; ++t) a[t] = g.a + ((int64_t)e * g.R + (16 * t + n < g.R ? 16 * t + n : g.R - 1)) * g.K + 8 * kb;
                float4v part[RT];
                down_products<RT, W, RT == 1 ? 8 : 4>(g.x + (int64_t)(m0 + nth_bit(with, my ? k0 + n : k0)) * g.K + 8 * kb, a, 0, g.K / 32, part);
                __syncthreads();
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) red[w][4 * t + j][lane] = part[t][j];
            }
            __syncthreads();
            // four ranks of a token per thread
            const int fours = g.R / 4;
            for (int u = threadIdx.x; u < kTile * fours; u += kThreads) {
                const int k = u / fours, r = 4 * (u - k * fours);
                if (k0 + k >= tokens) break;  // (the columns of no token are not looked at)
                float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (RT > 0) {
#pragma unroll
                    for (int q = 0; q < W; ++q)
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] += red[q][4 * (r >> 4) + (k & 3)][16 * (k >> 2) + (r & 15) + j];
                }
                const float *const h = g.h + (int64_t)(m0 + nth_bit(with, k0 + k)) * g.R + r;
                constexpr int kAtOnce = 8;  // (sixteen take registers that a third workgroup needs: 20 us for 15 of 32 tokens)
                for (int s0 = 0; RT == 0 && s0 < g.slices; s0 += kAtOnce) {
                    float4v part[kAtOnce];
#pragma unroll
                    for (int s = 0; s < kAtOnce; ++s) part[s] = *as_global<float4v>(h + (s0 + s < g.slices ? s0 + s : 0) * h_slice);
#pragma unroll
                    for (int s = 0; s < kAtOnce; ++s)
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] += s0 + s < g.slices ? part[s][j] : 0.0f;
                }
                uint32_t p[4][3];
#pragma unroll
                for (int j = 0; j < 4; ++j) split(v[j], &p[j][0], &p[j][1], &p[j][2]);
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    *reinterpret_cast<uint2v *>(&hs[q][k][r]) = uint2v{p[0][q] | p[1][q] << 16, p[2][q] | p[3][q] << 16};
            }
            __syncthreads();
            if (again) load(first, 0);  // (of the first tile it is there)
            for (int block = first; block < g.N; block += stride) {
                const int o0 = block + w * 16 * NT + 4 * NT * kb;  // the lane's outputs
                const bool whole = o0 + 4 * NT <= g.N;
                const int64_t at_y = row + o0;
                float4v sum[NT], rest[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = rest[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
                for (int c = 0; c < g.R; c += 64) {
                    if (c > 0) load(block, c);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = c + 32 * k + 8 * kb;
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            uint4v hw = {0, 0, 0, 0};
                            if (r < g.R) hw = *reinterpret_cast<const uint4v *>(&hs[q][n][r]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                float4v &to = q ? rest[t] : sum[t];
                                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, bw[k][t]),
                                                                             __builtin_bit_cast(bf16x8, hw), to, 0, 0, 0);
                            }
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) wait_written(sum[t], rest[t]);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[t][j] += __builtin_isfinite(sum[t][j]) ? rest[t][j] : 0.0f;
                const int next = block + stride;
                if (next < g.N) load(next, 0);
                if (my && whole) {
                    float v[4 * NT];
#pragma unroll
                    for (int j = 0; j < 4 * NT; ++j) v[j] = y[j] + sum[j >> 2][j & 3] * scale;
                    if (next < g.N) load_y(next);
                    store_results<4 * NT>(g.out, g.dtype, at_y, v);
                } else if (my) {
#pragma unroll
                    for (int j = 0; j < 4 * NT; ++j)
                        if (o0 + j < g.N) {
                            const float v = g.dtype == NVQ_F32 ? static_cast<const float *>(g.y)[at_y + j]
                                                               : bf16_bits_to_float(static_cast<const uint16_t *>(g.y)[at_y + j]);
                            store_global(g.out, g.dtype, at_y + j, v + sum[j >> 2][j & 3] * scale);
                        }
                }
            }
        }
    }
}

// Groups of a batch; the workers of one of them: as many as it can have tiles where there are up to four groups, then eight.
// (500 tokens, 4096 outputs, of 16 adapters in no order: four workers 27 us, eight 24; of three prompts: 10.2 and 12.6;
// 8000 tokens of prompts, 14336 outputs: 358 and 308.)
int groups_of(int M) { return (M + kGroup - 1) / kGroup; }
int workers_of(int M, int n) {
    const int tokens = M < kGroup ? M : kGroup, tiles = n + tokens / kTile, most = tokens < tiles ? tokens : tiles;
    const int cap = groups_of(M) <= 4 ? kGroup : 8;
    return most < cap ? most : cap;
}
// Tiles of a batch: all of them where one group's adapters have tokens of their own, about half as many as they could be
// where there are several groups (all: 256 tokens of 16 adapters in no order 18.3 us, in prompts 12.6; half: 19.3 and 11.0).
int tiles_of(int M, int n) {
    const int whole = (M + kTile - 1) / kTile, apart = groups_of(M) * (n < kGroup ? n : kGroup), most = apart < M ? apart : M;
    const int likely = groups_of(M) <= 1 ? most : most / 2;
    return whole > likely ? whole : likely;
}
// Blocks of 64, 32 or 16 ranks.
int rank_tiles(int R) { return R > 32 ? 4 : R > 16 ? 2 : 1; }
int rank_blocks(int R) { return (R + 16 * rank_tiles(R) - 1) / (16 * rank_tiles(R)); }
// Slices of K: as many as bring a thousand workgroups with work, of four columns (one per wave) or more.  Every workgroup of
// the second launch adds them up, so that more than eight pay where it has many outputs then (8 instead of 16: one token
// of 2048 outputs 7.3 -> 6.8 us, 500 of 4099 19.4 -> 17.3; 32 of 28672 21.2 -> 22.0).
int slices_of(const nvq_adapters &s, int M) {
    const int64_t others = (int64_t)tiles_of(M, s.n) * rank_blocks(s.R);
    int64_t want = 1024 / others;
    const int64_t most = (s.K / 32 + kWaves - 1) / kWaves;
    want = want < most ? want : most;
    const int64_t pay = s.N >= 16384 ? kMostSlices : kMostSlices / 2;
    want = want < pay ? want : pay;
    return want > 1 ? (int)want : 1;
}

// Whether a batch takes one launch: a group of tokens, adapters whose A a workgroup of eight waves asks for in one trip, and a tile
// with 128 outputs to a compute unit at most.  (Outputs of one token of 2048 inputs, 16 ranks: 2048 6.8 -> 5.8 us, 28672 7.6 -> 6.3;
// 32 tokens of 12 adapters 2048 8.4 -> 7.0, but 4096, 384 workgroups, 9.1 and 9.3, 8192 9.1 and 15.2.  One token of 4096 inputs, two
// trips, 6.8 and 8.1.)
constexpr int kOneWaves = 8, kOneInputs = 32768;
bool one_launch(const nvq_adapters &s, int M) {
    const int64_t blocks = (s.N + 16 * kOneWaves - 1) / (16 * kOneWaves);
    return groups_of(M) == 1 && s.R <= 32 && (int64_t)s.R * s.K <= kOneInputs && tiles_of(M, s.n) * blocks <= device_cu_count();
}

bool adapters_shape(const nvq_adapters *s, int M) {
    return s && s->n >= 1 && s->n <= 1 << 16 && s->K >= 32 && s->K % 32 == 0 && s->K <= NVQ_MAX_K && s->N >= 1 && s->N <= 1 << 24 &&
           s->R >= 8 && s->R % 8 == 0 && s->R <= NVQ_MAX_RANK && M >= 1 && M <= 1 << 16;
}

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_adapters_workspace_bytes(const nvq_adapters *adapters, int M) {
    using namespace nvq;
    if (!adapters_shape(adapters, M)) return 0;
    // (fewer tokens may take more slices: of no more than kMostSlices tiles in all, or of all M in one)
    const size_t rows = (size_t)M < 1024 ? (size_t)M * kMostSlices : (size_t)M + 1024 * kMostSlices;
    return rows * adapters->R * sizeof(float);
}

extern "C" int nvq_adapters_add(const nvq_adapters *adapters, const uint16_t *x_bf16, const int32_t *ids, int M, const void *y,
                                void *out, int dtype, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace nvq;
    if (!adapters || !adapters->a || !adapters->b || !x_bf16 || !ids || !y || !out || (dtype != NVQ_F32 && dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (!adapters_shape(adapters, M)) return NVQ_ERR_SHAPE;
    if (!aligned(adapters->a, 16) || !aligned(adapters->b, 16) || !aligned(adapters->scales, 4) || !aligned(x_bf16, 16) ||
        !aligned(ids, 4) || !aligned(y, 16) || !aligned(out, 16))
        return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_adapters_workspace_bytes(adapters, M))
        return NVQ_ERR_WORKSPACE;
    AdaptersArgs g;
    g.a = adapters->a;
    g.b = adapters->b;
    g.scales = adapters->scales;
    g.x = x_bf16;
    g.ids = ids;
    g.y = y;
    g.out = out;
    g.dtype = dtype;
    g.n = adapters->n;
    g.K = adapters->K;
    g.N = adapters->N;
    g.R = adapters->R;
    g.M = M;
    g.h = static_cast<float *>(workspace);
    g.slices = slices_of(*adapters, M);
    g.columns = (g.K / 32 + g.slices - 1) / g.slices;
    g.slices = (g.K / 32 + g.columns - 1) / g.columns;
    g.workers = workers_of(M, g.n);
    g.blocks = rank_blocks(g.R);
    const hipStream_t st = (hipStream_t)stream;
    const int groups = groups_of(M), tiles = tiles_of(M, g.n);
    g.copiers = out != y && groups <= 4;
    if (one_launch(*adapters, M)) {
        g.turns = (g.N + 16 * kOneWaves - 1) / (16 * kOneWaves);
        const dim3 grid((unsigned)((g.workers + g.copiers) * g.turns)), threads(64 * kOneWaves);
        if (rank_tiles(g.R) == 1)
            hipLaunchKernelGGL((adapters_up_kernel<1, 1, kOneWaves>), grid, threads, 0, st, g);
        else
            hipLaunchKernelGGL((adapters_up_kernel<1, 2, kOneWaves>), grid, threads, 0, st, g);
        NVQ_HIP_TRY(hipGetLastError());
        return NVQ_OK;
    }
    const dim3 block(kThreads), down((unsigned)(groups * g.workers * g.blocks * g.slices));
    if (rank_tiles(g.R) == 1)
        hipLaunchKernelGGL(adapters_down_kernel<1>, down, block, 0, st, g);
    else if (rank_tiles(g.R) == 2)
        hipLaunchKernelGGL(adapters_down_kernel<2>, down, block, 0, st, g);
    else
        hipLaunchKernelGGL(adapters_down_kernel<4>, down, block, 0, st, g);
    NVQ_HIP_TRY(hipGetLastError());
    // A wave to 64 outputs where that leaves four a compute unit (32 tokens of 12 adapters, 14336 outputs: 10.9 us, 16.3 with 16 to
    // a wave; one of 4096: 7.7 and 6.9).
    const bool wide = (int64_t)tiles * g.N >= 1024 * 64;
    const int per = (wide ? 64 : 16) * kWaves, blocks = (g.N + per - 1) / per;
    // As many workgroups as the device holds at once (three a compute unit) between the tiles, or the workers, which have
    // a part of a tile's outputs where there are few of them.
    const int resident = 3 * device_cu_count() / (groups <= 4 ? tiles : groups * g.workers);
    const int each = resident < 1 ? blocks : (blocks + resident - 1) / resident;
    g.turns = (blocks + each - 1) / each;
    const dim3 up((unsigned)(groups * (g.workers + g.copiers) * g.turns));
    if (wide)
        hipLaunchKernelGGL((adapters_up_kernel<4, 0, kWaves>), up, block, 0, st, g);
    else
        hipLaunchKernelGGL((adapters_up_kernel<1, 0, kWaves>), up, block, 0, st, g);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
