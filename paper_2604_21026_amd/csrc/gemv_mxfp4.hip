// nvq_gemv_mxfp4: microscaled 4-bit weights times the bf16 activations of 1 to 32 tokens.  y[m][n] = sum over the
// blocks g of 2^(scale - 127) * sum_j code[n][32g + j] * x[m][32g + j], weights and activations unrounded, sums in
// fp32.
//
// Bound by reading the weights once, 17 bytes per 32 of them, which is 4.25 bits; mx_rows.h has the product on
// the matrix cores.  Five kernels: one or two tokens by dot products; row tiles whose workgroups read the
// activations with the weights, for few inputs or rows; all activations of a few tokens in LDS; activations
// shared through LDS step by step; and, for many rows, activations that stay in registers.
//
// Measured in captured calls, one after the other, the same weights each time (and weights that no cache
// holds): 4096 x 4096 at one token 2.9 us (4.4; an empty launch 2.4 from the host), 128256 x 4096 at one token
// 42 us, 6.6 TB/s (47), at 32 tokens 54, 5.3 TB/s (61), 128256 x 14336 at one token 161, 6.1 TB/s (161); the
// choices at the end have more.
#include "mx_rows.h"

namespace nvq {

namespace {

// A workgroup takes R row tiles and T token tiles, its W waves share out K (rows_times_tokens: passes of Q
// columns, B at a time).
template <int R, int T, int W, int B, int Q>
__global__ __launch_bounds__(64 * W) void gemv_mxfp4_kernel(const uint8_t *__restrict__ q,
                                                            const uint8_t *__restrict__ scales, int N, int G,
                                                            const uint16_t *__restrict__ x, int M,
                                                            void *__restrict__ y, int y_dtype) {
    __shared__ float red[W][R * T * 4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int n = lane & 15;
    const int row0 = blockIdx.x * (16 * R);

    RowAt at[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + 16 * r + n;  // (rows past the end read the last one, their results go nowhere)
        at[r] = row_at<NVQ_FMT_MXFP4>(q, scales, row < N ? row : N - 1, G);
    }
    const char *xt[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int m = 16 * t + n;  // (tokens past the end read token 0: a product keeps tokens apart)
        xt[t] = reinterpret_cast<const char *>(x) + (size_t)(m < M ? m : 0) * G * 64;
    }
    float4v sum[R][T];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    rows_times_tokens<NVQ_FMT_MXFP4, R, T, B, Q>(at, xt, G, w, W, sum);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) red[w][(r * T + t) * 4 + j][lane] = sum[r][t][j];
    __syncthreads();
    // result i: lane-position i % 64 of register i / 64
    for (int i = threadIdx.x; i < R * T * 4 * 64; i += 64 * W) {
        const int reg = i >> 6, l = i & 63;
        const int t = (reg >> 2) % T, r = (reg >> 2) / T;
        const int m = 16 * t + 4 * (l >> 4) + (reg & 3), row = row0 + 16 * r + (l & 15);
        float v = red[0][reg][l];
#pragma unroll
        for (int k = 1; k < W; ++k) v += red[k][reg][l];
        if (m < M && row < N) store_global(y, y_dtype, (int64_t)m * N + row, v);
    }
}


// One or two tokens (M).  KS waves take R rows at a time, a lane of theirs the blocks l, 64 + l, .. (B in all),
// whose activations it keeps for all its rows, and ask for the next rows meanwhile.  A block's codes become
// bf16 values, scale and all, eight in four conversions, and go through the dot product of bf16 pairs.  (The
// matrix cores' way reads the activations for sixteen tokens: four loads for each one of weights, as much of
// the address path's time.  Of three tokens on the products themselves cost more.)
template <int M, int B, int R, int KS>
__global__ __launch_bounds__(256) void gemv_mxfp4_dot_kernel(const uint8_t *__restrict__ q,
                                                             const uint8_t *__restrict__ scales, int N, int G,
                                                             const uint16_t *__restrict__ x, void *__restrict__ y,
                                                             int y_dtype) {
    static_assert(KS == 1 || KS == 4, "a wave or the workgroup");
    constexpr int kTeams = 4 / KS;
    __shared__ float red[2][KS][M * R];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int team = blockIdx.x * kTeams + w / KS, teams = gridDim.x * kTeams, l0 = w % KS * (64 * B) + lane;
    const int groups = (N + R - 1) / R;
    if (team >= groups) return;  // (KS == 4: the whole workgroup)
    uint4v c[2][R][B];
    uint32_t sc[2][R][B];
    auto load = [&](int d, int group) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = group * R + r < N ? group * R + r : N - 1;
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int block = l0 + 64 * b < G ? l0 + 64 * b : G - 1;
                c[d][r][b] = load_stream(reinterpret_cast<const uint4 *>(q) + row * G + block);
                sc[d][r][b] = as_global<uint8_t>(scales)[row * G + block];
            }
        }
    };
    load(0, team);
    uint4v xr[M][B][4];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                xr[m][b][i] = uint4v{0, 0, 0, 0};
                if (l0 + 64 * b < G) xr[m][b][i] = as_global<uint4v>(x)[((int64_t)m * G + l0 + 64 * b) * 4 + i];
            }
    // Scales become exponents (the conversions look at nothing else); past the end, where activations are zero,
    // the smallest one, since values beyond bf16 would make them NaN.  (4096 x 14336 6.4 us for 6.25, others
    // equal; loads or products left out instead cost up to 10 %.)
    int up[B];
#pragma unroll
    for (int b = 0; b < B; ++b) up[b] = l0 + 64 * b < G ? 23 : 31;
    int turn = 0;
    auto one = [&](int d, int group) {
        float mine = 0.0f;  // lane m R + r: the result of row r, token m
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float sum[M] = {};
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const float s = __uint_as_float(sc[d][r][b] << up[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4v v = __builtin_bit_cast(uint4v, mx_values(c[d][r][b][i], s));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t w2 = v[k];
#pragma unroll
                        for (int m = 0; m < M; ++m) {
                            const uint32_t x2 = xr[m][b][i][k];
                            sum[m] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(nvq_bf16x2, w2),
                                                                     __builtin_bit_cast(nvq_bf16x2, x2), sum[m], false);
                        }
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const float all = group_sum<64>(sum[m]);
                mine = lane == m * R + r ? all : mine;
            }
        }
        if constexpr (KS > 1) {
            if (lane < M * R) red[turn & 1][w][lane] = mine;
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (w == 0 && lane < M * R) {
                mine = red[turn & 1][0][lane];
#pragma unroll
                for (int k = 1; k < KS; ++k) mine += red[turn & 1][k][lane];
            }
            ++turn;
        }
        const int row = group * R + lane % R;
        if (w % KS == 0 && lane < M * R && row < N) store_global(y, y_dtype, (int64_t)(lane / R) * N + row, mine);
    };
    // (the registers change roles, nothing is requested past the last rows)
    int g = team;
    while (true) {
        if (g + teams >= groups) {
            one(0, g);
            return;
        }
        load(1, g + teams);
        one(0, g);
        g += teams;
        if (g + teams >= groups) {
            one(1, g);
            return;
        }
        load(0, g + teams);
        one(1, g);
        g += teams;
    }
}

// The same for more tokens, whose activations outweigh the weights where every row tile reads them for itself:
// a workgroup of RG x S waves takes RG * R row tiles, and brings the activations of S passes of C columns into
// LDS for all of them, a pass ahead (through registers, the loads two passes ahead); wave (g, s) multiplies the
// row tiles of group g with pass s of each turn.  Piece c (16 bytes) of token n lies at position c ^ swapped(n %
// 16): a read takes lanes 0-3, 12-15 and 20-27 of a half wave together and then its other sixteen, and either
// sixteen touch every bank once.
__device__ __forceinline__ int swapped(int n) { return (n & 9) | (n & 2) << 1 | (n & 4) >> 1; }

template <int T, int R, int RG, int S, int C>
__global__ __launch_bounds__(64 * RG * S) void gemv_mxfp4_shared_kernel(const uint8_t *__restrict__ q,
                                                                        const uint8_t *__restrict__ scales, int N, int G,
                                                                        const uint16_t *__restrict__ x, int M,
                                                                        void *__restrict__ y, int y_dtype) {
    constexpr int kThreads = 64 * RG * S, kPieces = 16 * C;         // pieces of a token and pass
    constexpr int kAll = S * 16 * T * kPieces, kMine = kAll / kThreads;  // pieces of a turn, of a thread
    static_assert(kMine * kThreads == kAll, "whole pieces per thread");
    __shared__ __attribute__((aligned(1024))) uint4v xs[2][kAll];
    constexpr int kRegs = R * T * 4;
    static_assert(S == 1 || (S - 1) * RG * kRegs * 64 * 4 <= (int)sizeof(xs), "the partial tiles fit");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = wave / S, s = wave % S;
    const int n = lane & 15, kb = lane >> 4;
    const int row0 = (blockIdx.x * RG + g) * (16 * R);
    const int passes = G / (4 * C), turns = (passes + S - 1) / S;

    RowAt at[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + 16 * r + n;
        at[r] = row_at<NVQ_FMT_MXFP4>(q, scales, row < N ? row : N - 1, G);
    }
    // pieces of a turn, as they lie in LDS: [slice][token][position]
    auto ask = [&](uint4v (&v)[kMine], int turn) {
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int i = tid + k * kThreads, slice = i / (16 * T * kPieces), m = i / kPieces % (16 * T);
            const int piece = (i % kPieces) ^ swapped(m & 15);
            int pass = turn * S + slice;
            pass = pass < passes ? pass : passes - 1;
            v[k] = *as_global<uint4v>(reinterpret_cast<const char *>(x) + ((int64_t)(m < M ? m : 0) * G * 64 +
                                                                          (int64_t)pass * (256 * C) + piece * 16));
        }
    };
    auto keep = [&](const uint4v (&v)[kMine], int buf) {
#pragma unroll
        for (int k = 0; k < kMine; ++k) xs[buf][tid + k * kThreads] = v[k];
    };
    auto weights = [&](Codes<C> (&w)[R], Scales<NVQ_FMT_MXFP4, C> (&sc)[R], int turn) {
        const int pass = turn * S + s;  // (uniform; past the end: the last one, for nothing)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (pass < passes ? pass : passes - 1) * C;
            load_codes<C>(w[r], at[r], c, kb);
            load_scales<NVQ_FMT_MXFP4, C>(sc[r], at[r], c);
        }
    };
    float4v sum[R][T];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    if (turns > 0) {
        uint4v xr[kMine];
        Codes<C> w[2][R];
        Scales<NVQ_FMT_MXFP4, C> sc[2][R];
        ask(xr, 0);
        weights(w[0], sc[0], 0);
        keep(xr, 0);
        ask(xr, 1);
        auto arrive = [&]() {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's pieces are in LDS
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        auto one = [&](int d, int turn) {
            arrive();
            keep(xr, (turn + 1) & 1);
            ask(xr, turn + 2);
            weights(w[d ^ 1], sc[d ^ 1], turn + 1);
            __builtin_amdgcn_sched_barrier(0);
            const uint4v *const xb = &xs[turn & 1][s * (16 * T * kPieces)];
#pragma unroll
            for (int b = 0; b < C; ++b) {
                bf16x8 a[T][4];
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        a[t][i] = __builtin_bit_cast(bf16x8,
                                                     xb[(16 * t + n) * kPieces + ((16 * b + 4 * kb + i) ^ swapped(n))]);
                multiply_column<NVQ_FMT_MXFP4, R, T, C, C>(w[d], b, sc[d], b, a, sum);
            }
        };
        // (the registers of the weights change roles from turn to turn, they are not copied)
        const int mine = (passes - s + S - 1) / S;  // (uniform) all turns, or all but the last one
        for (int turn = 0; turn < mine; turn += 2) {
            one(0, turn);
            if (turn + 1 >= mine) break;
            one(1, turn + 1);
        }
        if (mine < turns) arrive();
    }
    const char *xt[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int m = 16 * t + n;  // (tokens past the end read token 0: a product keeps tokens apart)
        xt[t] = reinterpret_cast<const char *>(x) + (size_t)(m < M ? m : 0) * G * 64;
    }
    last_columns<NVQ_FMT_MXFP4, R, T>(at, xt, G, passes * C, 0, s, S, sum);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) wait_written(sum[r][t]);
    if constexpr (S > 1) {
        __syncthreads();
        float *const red = reinterpret_cast<float *>(&xs[0][0]);
        if (s > 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < T; ++t)
                    *reinterpret_cast<float4v *>(&red[(((g * (S - 1) + s - 1) * (R * T) + r * T + t) * 64 + lane) * 4]) =
                        sum[r][t];
        }
        __syncthreads();
        if (s > 0) return;
#pragma unroll
        for (int k = 0; k < S - 1; ++k)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < T; ++t)
                    sum[r][t] += *reinterpret_cast<const float4v *>(
                        &red[(((g * (S - 1) + k) * (R * T) + r * T + t) * 64 + lane) * 4]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int m = 16 * t + 4 * kb + j, row = row0 + 16 * r + n;
                if (m < M && row < N) store_global(y, y_dtype, (int64_t)m * N + row, sum[r][t][j]);
            }
}


// The activations stay in registers: wave w of W keeps those of C columns (4 C blocks of 32 inputs), of all
// tokens, for the whole kernel, and the workgroup streams its row tiles past them, one after the other, D of
// them requested ahead.  So nothing but weights and their scales is read in the loop (read again for every
// tile, one token's activations took 25 of 68 us at 128256 x 4096).  The last wave's blocks may begin earlier
// than its share, where activations and scales are zero.  Partial tiles are added through LDS in wave order, by
// waves that change from tile to tile, and wait there (`out`) until kGroup tiles' results leave as runs of 16
// kGroup rows: stored tile by tile, 32 bytes here and there among the loads, 32 tokens' took 64 us for 56.
template <int T, int W, int C, int D>
__global__ __launch_bounds__(64 * W) void gemv_mxfp4_resident_kernel(const uint8_t *__restrict__ q,
                                                                     const uint8_t *__restrict__ scales, int N, int G,
                                                                     const uint16_t *__restrict__ x, int M,
                                                                     void *__restrict__ y, int y_dtype) {
    constexpr int kGroup = 16, kRows = 16 * kGroup, kPitch = kRows + 4;
    __shared__ float red[2][W][T * 4][64];
    __shared__ __attribute__((aligned(16))) float out[2][16 * T][kPitch];
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // the workgroup's tiles (there are more than workgroups)
    const int64_t tiles = (N + 15) >> 4;
    const int begin = (int)(tiles * blockIdx.x / gridDim.x), mine = (int)(tiles * (blockIdx.x + 1) / gridDim.x) - begin;
    const int share = 4 * C * w, b0 = share < G - 4 * C ? share : G - 4 * C;  // (G >= 4 C)

    Codes<C> codes[D][1];
    Scales<NVQ_FMT_MXFP4, C> sc[D][1];
    auto load = [&](int d, int it) {
        const int row = 16 * (begin + (it < mine ? it : mine - 1)) + n;
        const RowAt at = row_at<NVQ_FMT_MXFP4>(q, scales, row < N ? row : N - 1, G);
        const RowAt from = {at.q + b0, at.s + b0};
        load_codes<C>(codes[d][0], from, 0, kb);
        load_scales<NVQ_FMT_MXFP4, C>(sc[d][0], from, 0);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, d);
    bf16x8 xr[C][T][4];
#pragma unroll
    for (int b = 0; b < C; ++b)
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int block = b0 + 4 * b + kb, m = 16 * t + n;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4v v = {0, 0, 0, 0};
                if (block >= share && m < M)
                    v = *as_global<uint4v>(reinterpret_cast<const char *>(x) + ((size_t)m * G + block) * 64 + 16 * i);
                xr[b][t][i] = __builtin_bit_cast(bf16x8, v);
            }
        }
    // rows of tiles first .. of the group that lies in out[half], four to a lane
    auto leave = [&](int half, int first, int count) {
        typedef uint2v uint2v_any __attribute__((aligned(2)));
        typedef float4v float4v_any __attribute__((aligned(4)));
        const int row0 = 16 * (begin + first), rows = 16 * count < N - row0 ? 16 * count : N - row0;
        for (int i = threadIdx.x; i < M * (kRows / 4); i += 64 * W) {
            const int m = i / (kRows / 4), r = i % (kRows / 4) * 4;
            if (r >= rows) continue;
            const float4v v = *reinterpret_cast<const float4v *>(&out[half][m][r]);
            const int64_t to = (int64_t)m * N + row0 + r;
            if (r + 4 <= rows) {
                if (y_dtype == NVQ_BF16)
                    *(__attribute__((address_space(1))) uint2v_any *)(static_cast<uint16_t *>(y) + to) =
                        uint2v{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                else
                    *(__attribute__((address_space(1))) float4v_any *)(static_cast<float *>(y) + to) = v;
            } else {
                for (int j = 0; r + j < rows; ++j) store_global(y, y_dtype, to + j, out[half][m][r + j]);
            }
        }
    };
    auto one = [&](int d, int it) {
        float4v sum[1][T];
#pragma unroll
        for (int t = 0; t < T; ++t) sum[0][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        if (b0 < share) clear_scales<NVQ_FMT_MXFP4, C>(sc[d][0], share - b0);  // (uniform)
#pragma unroll
        for (int b = 0; b < C; ++b) multiply_column<NVQ_FMT_MXFP4, 1, T, C, C>(codes[d], b, sc[d], b, xr[b], sum);
        load(d, it + D);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            wait_written(sum[0][t]);
#pragma unroll
            for (int j = 0; j < 4; ++j) red[it & 1][w][4 * t + j][lane] = sum[0][t][j];
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (the group before is whole since this barrier, its half is written again a group later)
        if (it % kGroup == 0 && it > 0) leave((it / kGroup - 1) & 1, it - kGroup, kGroup);
        const int reg = (w + W - (it * 4 * T) % W) % W;  // (uniform)
        if (reg < 4 * T) {
            float v = red[it & 1][0][reg][lane];
#pragma unroll
            for (int k = 1; k < W; ++k) v += red[it & 1][k][reg][lane];
            out[it / kGroup & 1][16 * (reg >> 2) + 4 * kb + (reg & 3)][16 * (it % kGroup) + n] = v;
        }
    };
    for (int it = 0; it < mine; it += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (d > 0 && it + d >= mine) break;
            one(d, it + d);
        }
    }
    __syncthreads();
    const int last = (mine - 1) / kGroup;
    leave(last & 1, last * kGroup, mine - last * kGroup);
}

// Up to three tokens, whose activations fit in LDS: a workgroup keeps them there for all its row tiles, its W
// waves share out a tile's columns, four at a time, and four times two are on their way, from tile to tile
// without a pause.  (Nothing is requested past the last one: that cost a quarter at 4096 x 4096.)
constexpr int kLdsTokens = 3, kLdsBytes = 56 * 1024;  // (two workgroups to a compute unit)
__device__ __host__ constexpr int lds_pitch(int G) { return ((G + 3) / 4 + 1) * 256 + 16; }

template <int W>
__global__ __launch_bounds__(64 * W, 4) void gemv_mxfp4_lds_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ scales,
                                                                   int N, int G, const uint16_t *__restrict__ x, int M,
                                                                   void *__restrict__ y, int y_dtype) {
    constexpr int C = 4;  // 16 scales, in one load
    __shared__ __attribute__((aligned(16))) unsigned char xs[kLdsBytes];
    __shared__ float red[2][W][4][64];
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int tiles = (N + 15) >> 4, cols = (G + 3) >> 2, per = (cols + W * C - 1) / (W * C);
    const int pitch = lds_pitch(G);  // of a token: its columns, one of zeros, 16 bytes that set the tokens' banks apart
    Codes<C> codes[2][1];
    uint4v sc[2];
    auto load = [&](int d, int tile, int part) {
        const int row = 16 * tile + n, c0 = (part * W + w) * C;
        const RowAt at = row_at<NVQ_FMT_MXFP4>(q, scales, row < N ? row : N - 1, G);
#pragma unroll
        for (int b = 0; b < C; ++b) {
            const int block = 4 * (c0 + b) + kb;
            codes[d][0].w[b] = load_stream(at.q + (block < G ? block : G - 1));
        }
        typedef uint4v uint4v_any __attribute__((aligned(1)));
        sc[d] = *(const __attribute__((address_space(1))) uint4v_any *)(at.s + (4 * c0 < G - 16 ? 4 * c0 : G - 16));
    };
    // (the loads' place runs ahead of the products'; a workgroup has two items or more, of two tiles or of one
    // tile's parts)
    const int items = ((tiles - 1 - (int)blockIdx.x) / (int)gridDim.x + 1) * per;
    int lt = blockIdx.x, lp = 0;
    auto ahead = [&](int d) {
        load(d, lt, lp);
        if (++lp == per) {
            lp = 0;
            lt += gridDim.x;
        }
    };
    ahead(0);
    ahead(1);
    for (int i = threadIdx.x; i < M * (cols + 1) * 16; i += 64 * W) {
        const int m = i / ((cols + 1) * 16), p = i - m * (cols + 1) * 16;
        uint4v v = {0, 0, 0, 0};
        if (p < 4 * G) v = *as_global<uint4v>(reinterpret_cast<const char *>(x) + ((size_t)m * G * 4 + p) * 16);
        *reinterpret_cast<uint4v *>(&xs[m * pitch + p * 16]) = v;
    }
    __syncthreads();
    const unsigned char *const mine = xs + (n < M ? n : 0) * pitch + 64 * kb;
    int ct = blockIdx.x, cp = 0, done = 0;
    float4v sum[1][1] = {{float4v{0.0f, 0.0f, 0.0f, 0.0f}}};
    auto one = [&](int d, bool more) {
        const int c0 = (cp * W + w) * C;
        const int past = 4 * c0 - (G - 16);  // bytes of the scales before the column's (uniform; past the end: zeros)
        uint4v v = sc[d];
        if (past > 0) {
            if (past >= 16) {
                v = uint4v{0, 0, 0, 0};
            } else {
                uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
                if (past & 8) {
                    lo = hi;
                    hi = 0;
                }
                const int bits = 8 * (past & 7);
                if (bits) {
                    lo = lo >> bits | hi << (64 - bits);
                    hi >>= bits;
                }
                v = uint4v{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
            }
        }
        Scales<NVQ_FMT_MXFP4, C> s[1];
#pragma unroll
        for (int b = 0; b < C; ++b) s[0].s[b] = v[b];
#pragma unroll
        for (int b = 0; b < C; ++b) {
            const int c = c0 + b < cols ? c0 + b : cols;
            bf16x8 a[1][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[0][i] = *reinterpret_cast<const bf16x8 *>(mine + c * 256 + 16 * i);
            multiply_column<NVQ_FMT_MXFP4, 1, 1, C, C>(codes[d], b, s, b, a, sum);
        }
        if (more) ahead(d);
        if (++cp < per) return;
        wait_written(sum[0][0]);
        float(&to)[W][4][64] = red[done & 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) to[w][j][lane] = sum[0][0][j];
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int j = (w + W - (done * 4) % W) % W;  // (uniform)
        if (j < 4) {
            float r = to[0][j][lane];
#pragma unroll
            for (int k = 1; k < W; ++k) r += to[k][j][lane];
            const int m = 4 * kb + j, row = 16 * ct + n;
            if (m < M && row < N) store_global(y, y_dtype, (int64_t)m * N + row, r);
        }
        ++done;
        cp = 0;
        ct += gridDim.x;
        sum[0][0] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    };
    int left = items;
    for (; left >= 4; left -= 2) {
        one(0, true);
        one(1, true);
    }
    if (left == 3) {
        one(0, true);
        one(1, false);
        one(0, false);
    } else {
        one(0, false);
        one(1, false);
    }
}

struct GemvArgs {
    const uint8_t *q, *s;
    const uint16_t *x;
    void *y;
    int N, G, M, y_dtype;
};

// Up to 16 tokens, R row tiles per workgroup.  (Four row tiles, passes of eight columns, two at a time: eight
// tokens of 14336 x 4096 9.6 us, of 128256 x 14336 198; passes of four 10.2 and 209, one column at a time 9.5
// and 238.  One row tile, passes of four columns at once: nothing else was better by 1 %.)
template <int R>
int gemv_rows(const GemvArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.N + 16 * R - 1) / (16 * R)));
    hipLaunchKernelGGL((gemv_mxfp4_kernel<R, 1, 4, R == 1 ? 4 : 2, R == 1 ? 4 : 8>), grid, dim3(256), 0, st, a.q, a.s, a.N, a.G,
                       a.x, a.M, a.y, a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

// 17 to 32 tokens, a row tile per workgroup.
int gemv_two_tiles(const GemvArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((gemv_mxfp4_kernel<1, 2, 8, 2, 2>), dim3((unsigned)(((int64_t)a.N + 15) / 16)), dim3(512), 0,
                       st, a.q, a.s, a.N, a.G, a.x, a.M, a.y, a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

template <int T, int C>
int gemv_resident(const GemvArgs &a, int cus, hipStream_t st) {
    hipLaunchKernelGGL((gemv_mxfp4_resident_kernel<T, 8, C, 2>), dim3((unsigned)cus), dim3(512), 0, st, a.q, a.s, a.N, a.G, a.x,
                       a.M, a.y, a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

template <int M, int B, int R, int KS>
int gemv_dot(const GemvArgs &a, int cus, hipStream_t st) {
    const int64_t wanted = ((int64_t)a.N * KS + 4 * R - 1) / (4 * R);
    const dim3 grid((unsigned)(wanted < 2 * cus ? wanted : 2 * cus));
    hipLaunchKernelGGL((gemv_mxfp4_dot_kernel<M, B, R, KS>), grid, dim3(256), 0, st, a.q, a.s, a.N, a.G, a.x, a.y,
                       a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

int gemv_lds(const GemvArgs &a, int grid, hipStream_t st) {
    hipLaunchKernelGGL((gemv_mxfp4_lds_kernel<8>), dim3((unsigned)grid), dim3(512), 0, st, a.q, a.s, a.N, a.G, a.x, a.M, a.y,
                       a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

template <int T, int R, int RG, int S, int C>
int gemv_shared(const GemvArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.N + 16 * R * RG - 1) / (16 * R * RG)));
    hipLaunchKernelGGL((gemv_mxfp4_shared_kernel<T, R, RG, S, C>), grid, dim3(64 * RG * S), 0, st, a.q, a.s, a.N, a.G, a.x, a.M,
                       a.y, a.y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_gemv_mxfp4(const uint8_t *qweight, const uint8_t *scales, int N, int K, const uint16_t *x_bf16,
                              int M, void *y, int y_dtype, void *stream) {
    using namespace nvq;
    if (!qweight || !scales || !x_bf16 || !y || (y_dtype != NVQ_F32 && y_dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (N <= 0 || N > (1 << 29) || M < 1 || M > NVQ_MAX_M || K <= 0 || K % 32 || K > NVQ_MAX_K) return NVQ_ERR_SHAPE;
    if (!aligned(qweight, 16) || !aligned(x_bf16, 16) || !aligned(y, y_dtype == NVQ_F32 ? 4 : 2)) return NVQ_ERR_ALIGN;
    const hipStream_t st = (hipStream_t)stream;
    const GemvArgs a = {qweight, scales, x_bf16, y, N, K / 32, M, y_dtype};
    const int cus = device_cu_count();
    const int64_t tiles = ((int64_t)N + 15) / 16;
    // One token, us against what follows: 4096 x 4096 2.9 (3.9), 14336 x 4096 5.3 (8.1), 1024 x 4096 2.5 (3.8),
    // 4096 x 14336 6.5 (8.7), 2048 x 8192 3.4 (5.2), 10240 x 8192 9.3 (11.0), 128256 x 4096 42 (44), 14336 x
    // 1024 3.9 (4.4); not 32768 x 512 5.9 (4.0), and 4096 x 1024 2.3 (2.3).  Two rows at a time, or four where
    // that is one turn of one workgroup to each compute unit (4096 x 4096 3.2 against 3.5, 14336 x 4096 6.6
    // against 6.0); from 4096 inputs on the four waves share them, four rows at a time (10240 x 8192 9.5
    // against 10.6).
    if (M == 1) {
        if (a.G >= 32 && a.G <= 64 && (int64_t)N * a.G >= 1024 * cus) return gemv_dot<1, 1, 4, 1>(a, cus, st);
        if (a.G > 64 && a.G <= 128)
            return N > 8 * cus && N <= 16 * cus ? gemv_dot<1, 2, 4, 1>(a, cus, st) : gemv_dot<1, 2, 2, 1>(a, cus, st);
        if (a.G > 128 && a.G <= 256) return gemv_dot<1, 1, 4, 4>(a, cus, st);
        if (a.G > 256 && a.G <= 512) return gemv_dot<1, 2, 4, 4>(a, cus, st);
    }
    // Two: 4096 x 4096 3.8 (4.1), 14336 x 4096 7.3 (8.2), 1024 x 4096 3.1 (4.0), 4096 x 14336 8.8 (9.5, but
    // with weights that no cache holds 11.9 and 11.2); not 28672 x 4096 12.9 (12.3).
    if (M == 2 && tiles < 4 * cus) {
        if (a.G > 64 && a.G <= 128)
            return N > 8 * cus && N <= 16 * cus ? gemv_dot<2, 2, 4, 1>(a, cus, st) : gemv_dot<2, 2, 2, 1>(a, cus, st);
        if (a.G > 128 && a.G <= 256) return gemv_dot<2, 1, 4, 4>(a, cus, st);
        if (a.G > 256 && a.G <= 512) return gemv_dot<2, 2, 4, 4>(a, cus, st);
    }
    // Many row tiles, K that eight waves hold: (2, 128256, 4096) 44 us, at 16 tokens 47, at 32 54; below, a
    // tile or two per workgroup, its start costs more ((1, 14336, 4096) 9.4).
    if (tiles >= 16 * cus && a.G >= 16 && a.G <= 128) {
        if (a.G <= 64) return M <= 16 ? gemv_resident<1, 2>(a, cus, st) : gemv_resident<2, 2>(a, cus, st);
        return M <= 16 ? gemv_resident<1, 4>(a, cus, st) : gemv_resident<2, 4>(a, cus, st);
    }
    // Up to three tokens, many row tiles, or several and more K than the waves take at once, or K in whole
    // steps of them (4096 inputs).  us against what follows, of three tokens (18830, 6624) 16.6 and 24.3,
    // (28672, 4096) 13.3 and 14.1, (10240, 8192) 12.4 and 14.2, (8209, 4224) 7.8 and 9.6, (2048, 8192) 6.1 and
    // 6.6, (33000, 2080) 11.0 and 11.4; of two (28672, 4096) 12.3 and 13.8; of one (8209, 16672) 19.4 and 27.2,
    // (4096, 24576) 12.4 and 14.4; not of three (4096, 9152) 7.3 and 7.0, of four (14336, 4096) 9.8 and 8.8.
    if (M <= kLdsTokens && a.G > 64 && M * lds_pitch(a.G) <= kLdsBytes &&
        (tiles >= 4 * cus || (a.G > 128 && (tiles > 2 * cus || a.G % 128 == 0))))
        return gemv_lds(a, (int)(tiles < 2 * cus ? tiles : 2 * cus), st);
    // Up to 16 tokens.  us at (tokens, rows, inputs), R row tiles per workgroup with each wave reading its
    // activations, or activations shared by the RG groups of S waves; a workgroup to each compute unit where
    // row tiles allow:
    //                       rows 1  rows 4  shared 1, 8  shared 2, 4  shared 4, 2
    //   (1, 4096, 4096)       3.9     7.7        5.6         6.2         8.3
    //   (16, 4096, 4096)      6.4    10.2        5.9         6.5         8.5
    //   (8, 4096, 14336)     13.2    24.5       11.6        16.0        23.0
    //   (4, 4096, 14336)     11.1    22.3       11.1        15.1        22.9
    //   (2, 8192, 4096)       6.2     8.2       10.2         6.9         8.8
    //   (4, 8192, 4096)       7.1     8.6       10.4         7.0         9.0
    //   (8, 8192, 4096)       8.3     9.2       10.2         7.2         9.1
    //   (8, 14336, 4096)     15.1     9.2       20.5        11.5         9.2
    //   (16, 14336, 4096)    20.2    10.5       21.0        11.7         9.2
    // and at (16, 128256, 14336), too many inputs for registers, 16 row tiles 193 against 238 with 4.
    if (M <= 16) {
        if (tiles <= cus) return M * a.G >= 2048 ? gemv_shared<1, 1, 1, 8, 2>(a, st) : gemv_rows<1>(a, st);
        if (tiles <= 2 * cus) return M > 4 ? gemv_shared<1, 1, 2, 4, 2>(a, st) : gemv_rows<1>(a, st);
        if (M <= 8) return gemv_rows<4>(a, st);
        return tiles < 16 * cus ? gemv_shared<1, 1, 4, 2, 2>(a, st) : gemv_shared<1, 2, 8, 1, 4>(a, st);
    }
    // us at (32 tokens, rows, inputs)    (4096, 4096) (4096, 14336) (8192, 4096) (14336, 4096) (128256, 4096)
    //   a row tile, K in eight slices         8.0         20.4         15.0         29.7          249
    //   2 row tiles, K in four                8.4         23.2          9.8         17.8          144
    //   4 row tiles, K in two                 9.9         30.9         11.1         11.4           87
    //   16 row tiles                         26.6         83.1         26.7         27.4           65
    // (Up to 2 row tiles the activations bound it: every compute unit reads all of them, 0.9 MB at 14336
    // inputs.  Asked for two turns ahead, each workgroup beginning at another place of K, or with more weights
    // in flight it took as long.)  And with few inputs, each wave reading its activations, against a row tile in
    // eight slices: (25, 1236, 1760) 4.3 and 5.4, (32, 4096, 1024) 3.9 and 4.2, (20, 300, 3520) 7.0 and 6.9,
    // (32, 2048, 2560) 6.8 and 5.7 (from about 2000 inputs on slices would do as well or better); not (32,
    // 1024, 4096) 10.0 and 7.4.
    if (tiles <= cus && a.G < 128) return gemv_two_tiles(a, st);
    if (tiles <= cus && a.G >= 128) return gemv_shared<2, 1, 1, 8, 1>(a, st);
    if (tiles <= 2 * cus) return gemv_shared<2, 1, 2, 4, 2>(a, st);
    if (tiles < 16 * cus) return gemv_shared<2, 1, 4, 2, 2>(a, st);
    return gemv_shared<2, 2, 8, 1, 4>(a, st);
}
