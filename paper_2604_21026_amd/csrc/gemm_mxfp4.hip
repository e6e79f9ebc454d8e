// nvq_gemm_mxfp4: both operands microscaled 4-bit floating point, for prompts.  The matrix cores take codes and
// scales as they are: one 16x16x128 scaled MFMA multiplies four blocks of 16 rows with those of 16 tokens, lane
// (i, kb) = (lane % 16, lane / 16) holding the 16 bytes of codes of one block of row or token i and that block's scale
// byte.  Sums in fp32.
//
// Bound by the matrix units where there is enough to multiply, by the L2's rate into LDS in smaller tiles.
// Measured (M x N x K): 4096 x 28672 x 4096 265 us = 3.6 PFLOP/s (the products alone, in a loop: 158), 512 x
// 4096 x 14336 31 us, 77 x 1003 x 2080 6 us.
#include "mfma_act.h"

namespace nvq {

namespace {

typedef int int8v __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int8v fp4_operand(const uint4v &c) {
    return int8v{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}

// ---- tiles through LDS ----
typedef __attribute__((address_space(3))) void *lds_void_ptr;

// All of this wave's LDS accesses done and all but its last LOADS loads arrived, in every wave.  (The barrier of
// __syncthreads() waits for all loads.)
template <int LOADS>
__device__ __forceinline__ void stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LOADS & 15) | ((LOADS >> 4) << 14) | 0x0070);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// sum += a times b with byte K of the scales, the sums in accumulator registers.  (Given the builtin the compiler moves
// sums between the two halves of the register file, which they fill together with the operands.)
template <int K>
__device__ __forceinline__ void multiply_add(float4v &sum, const uint4v &a, const uint4v &b, uint32_t sa, uint32_t sb) {
    static_assert(K >= 0 && K < 4, "");
#define NVQ_MFMA(lo_, hi_)                                                                                   \
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[" #lo_ "," #lo_           \
                 ",0] op_sel_hi:[" #hi_ "," #hi_ ",0] cbsz:4 blgp:4"                                         \
                 : "+a"(sum)                                                                                 \
                 : "v"(a), "v"(b), "v"(sa), "v"(sb))
    if (K == 0) NVQ_MFMA(0, 0);
    if (K == 1) NVQ_MFMA(1, 0);
    if (K == 2) NVQ_MFMA(0, 1);
    if (K == 3) NVQ_MFMA(1, 1);
#undef NVQ_MFMA
}

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn; each XCD, with its own L2, works off a
// contiguous eighth of the tiles, in bands of four token tiles, row tile after row tile, so that the tiles its compute
// units hold at a time share their operands.
struct GemmTile {
    int n, m;
};
__device__ __forceinline__ GemmTile gemm_tile_of(int block, int tiles, int tiles_n) {
    const int xcd = block & 7, each = tiles >> 3, more = tiles & 7;
    const int t = xcd * each + (xcd < more ? xcd : more) + (block >> 3);
    const int tiles_m = tiles / tiles_n;
    const int band = t / (4 * tiles_n), first = 4 * band;
    const int high = tiles_m - first < 4 ? tiles_m - first : 4;
    const int in = t - first * tiles_n;
    return GemmTile{in / high, first + in % high};
}

// A wave's results: 16 A tokens at a time through LDS (`out`: 16 A rows of 16 P results and 16 bytes), so that
// they leave as whole runs of 16 P results, 16 bytes per lane at any alignment (4095 x 28669 x 4096: 281 us, by
// single results 390).  BYTES: of a result.
template <int P, int T, int A, int BYTES>
__device__ __forceinline__ void store_tile(unsigned char *out, float4v (&sum)[P][T], int n0, int N, int m0, int M, void *y) {
    constexpr int kRow = 16 * P * BYTES, kPitch = kRow + 16;
    const int lane = threadIdx.x & 63, i = lane & 15, kb = lane >> 4;
    typedef uint4v uint4v_any __attribute__((aligned(2)));  // (rows of y begin anywhere)
    const bool whole = n0 + 16 * P <= N;  // (uniform)
#pragma unroll
    for (int t0 = 0; t0 < T; t0 += A) {
        const int first = m0 + 16 * t0;
        if (first >= M) break;  // (uniform)
#pragma unroll
        for (int t = 0; t < A; ++t)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                unsigned char *const at = out + (16 * t + i) * kPitch + (16 * p + 4 * kb) * BYTES;
                const float4v v = sum[p][t0 + t];
                if (BYTES == 2)
                    *reinterpret_cast<uint2v *>(at) = uint2v{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                else
                    *reinterpret_cast<float4v *>(at) = v;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int tokens = M - first < 16 * A ? M - first : 16 * A;
        if (whole) {
            constexpr int kLanes = kRow / 16;  // of a row
#pragma unroll
            for (int c = 0; c < 16 * A * kLanes / 64; ++c) {
                const int r = (64 * c + lane) / kLanes, b = (64 * c + lane) % kLanes * 16;
                const uint4v v = *reinterpret_cast<const uint4v *>(out + r * kPitch + b);
                if (r < tokens)
                    *(__attribute__((address_space(1))) uint4v_any *)(static_cast<char *>(y) +
                                                                      ((int64_t)(first + r) * N + n0) * BYTES + b) = v;
            }
        } else {
            constexpr int kAtOnce = P == 8 ? 1 : 8;
            // (one by one, a read of LDS and its store took 2 us more; unrolled in the largest tile, which
            // fills the registers, they cost its whole rows 4 %)
#pragma unroll kAtOnce
            for (int c = lane; c < tokens * 16 * P; c += 64) {
                const int r = c / (16 * P), n = c % (16 * P);
                if (n0 + n >= N) continue;
                const int64_t to = (int64_t)(first + r) * N + n0 + n;
                if (BYTES == 2)
                    ((__attribute__((address_space(1))) uint16_t *)y)[to] =
                        *reinterpret_cast<const uint16_t *>(out + r * kPitch + n * 2);
                else
                    ((__attribute__((address_space(1))) float *)y)[to] =
                        *reinterpret_cast<const float *>(out + r * kPitch + n * 4);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// A wave of 64 x 64 results: weights are the first operand, so that a lane's four registers of a 16x16 tile are
// four neighbouring rows (columns of y) of one token.  For short K, where the results are the work: 658 x 9765
// x 448 took 20 us with a store from each lane for each result, 12 in whole runs; 4096 x 4096 x 256 40 and 17.
__global__ __launch_bounds__(64) void gemm_mxfp4_small_k_kernel(const uint4 *__restrict__ wq,
                                                               const uint8_t *__restrict__ ws, int N, int G,
                                                               const uint4 *__restrict__ xq,
                                                               const uint8_t *__restrict__ xs, int M,
                                                               void *__restrict__ y, int y_dtype, int tiles_n) {
    const int lane = threadIdx.x, i = lane & 15, kb = lane >> 4;
    __shared__ __attribute__((aligned(16))) unsigned char out[64 * (64 * 4 + 16)];
    const GemmTile tile = gemm_tile_of(blockIdx.x, gridDim.x, tiles_n);
    const int n0 = tile.n * 64, m0 = tile.m * 64;
    float4v sum[4][4] = {};
    int64_t wr[4], xr[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int n = n0 + 16 * t + i, m = m0 + 16 * t + i;
        wr[t] = (int64_t)(n < N ? n : N - 1) * G;
        xr[t] = (int64_t)(m < M ? m : M - 1) * G;
    }
    for (int g0 = 0; g0 < G; g0 += 4) {
        const int g = g0 + kb;
        const bool in = g < G;
        uint4v a[4], b[4];
        int sa[4], sb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t at = in ? g : G - 1;
            a[t] = load_stream(wq + wr[t] + at);
            b[t] = load_stream(xq + xr[t] + at);
            sa[t] = ws[wr[t] + at];
            sb[t] = xs[xr[t] + at];
            if (!in) {
                a[t] = b[t] = uint4v{0, 0, 0, 0};
                sa[t] = sb[t] = 127;
            }
        }
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                sum[p][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(a[p]), fp4_operand(b[t]), sum[p][t],
                                                                             4, 4, 0, sa[p], 0, sb[t]);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t) asm volatile("s_nop 7\n\ts_nop 7" : "+v"(sum[p][t]));
    if (y_dtype == NVQ_BF16)
        store_tile<4, 4, 4, 2>(out, sum, n0, N, m0, M, y);
    else
        store_tile<4, 4, 4, 4>(out, sum, n0, N, m0, M, y);
}

// 4 x 4 bytes transposed: word k of the result holds byte k of the four words.
__device__ __forceinline__ uint4v transpose_bytes(const uint4v &d) {
    const uint32_t lo01 = __builtin_amdgcn_perm(d.y, d.x, 0x05010400u), hi01 = __builtin_amdgcn_perm(d.y, d.x, 0x07030602u);
    const uint32_t lo23 = __builtin_amdgcn_perm(d.w, d.z, 0x05010400u), hi23 = __builtin_amdgcn_perm(d.w, d.z, 0x07030602u);
    return uint4v{__builtin_amdgcn_perm(lo23, lo01, 0x05040100u), __builtin_amdgcn_perm(lo23, lo01, 0x07060302u),
                  __builtin_amdgcn_perm(hi23, hi01, 0x05040100u), __builtin_amdgcn_perm(hi23, hi01, 0x07060302u)};
}

// S groups of 2 x 2 waves, each wave 16 P rows by 16 T tokens, W waves per SIMD.  A group takes a slice of K
// with LDS of its own; group 0 adds the slices' results in their order.
//
// A stage is 256 inputs, 128 bytes of codes, of all the workgroup's rows and tokens: whole lines (with 64 bytes
// per row the L2 gives half the rate, 69 against 131 bytes per ns and compute unit).  Two stages lie in LDS.  A
// stage is multiplied in two steps of four blocks.  The second step's operands are read in the first half of
// the first step; from there on the stage's place is free and the next but one is loaded into it, a few
// instructions between the products at a time, until the end of the second step, in whose second half the next
// stage's first operands are read.  Piece c (16 bytes) of row r is kept at position c ^ (r / 2 % 8): an LDS read
// of 16 bytes per lane takes lanes 0-3, 12-15 and 20-27 of a half wave together and then its other sixteen, and
// either sixteen touch all banks once.
template <int P, int T, int S, int W>
__global__ __launch_bounds__(256 * S) __attribute__((amdgpu_waves_per_eu(W, W))) void gemm_mxfp4_kernel(
    const unsigned char *__restrict__ wq, const unsigned char *__restrict__ ws, int N, int G,
    const unsigned char *__restrict__ xq, const unsigned char *__restrict__ xs, int M, void *__restrict__ y, int y_dtype,
    int tiles_n) {
    constexpr int kRows = 32 * P, kTokens = 32 * T, kBoth = kRows + kTokens;
    constexpr int kLoads = kBoth / 32;  // load instructions (of 8 rows or tokens) per wave and stage
    constexpr int kHalf = P / 2, kSlots = P + kHalf, kReads = kHalf > 1 ? kHalf - 1 : 1;
    static_assert(P % 2 == 0 && kBoth % 32 == 0, "");
    // (separate objects: the compiler then lets one be read while the other is filled)
    __shared__ __attribute__((aligned(1024))) unsigned char stage0[S * kBoth * 128], stage1[S * kBoth * 128];
    __shared__ __attribute__((aligned(16))) uint32_t scales[S * kBoth * 4];

    const int group = S == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8);
    const int tid = threadIdx.x & 255, lane = tid & 63, i = lane & 15, kb = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int own = group * kBoth;  // the group's first row in LDS
    const int wa = wave & 1, wb = wave >> 1;
    const GemmTile tile = gemm_tile_of(blockIdx.x, gridDim.x, tiles_n);
    const int n0 = tile.n * kRows, m0 = tile.m * kTokens;
    // windows of two stages, sixteen blocks: the group's begin and their number (some groups' last ones may lie
    // past the end)
    const int windows = S == 1 ? (G + 15) >> 4 : (((G + 15) >> 4) + S - 1) / S, window0 = group * windows;

    // Global memory -> LDS: instruction j of a wave takes 8 rows (then tokens), lane l position l % 8 of row
    // l / 8.  Rows past the end read the last one, blocks past the end the last one (their scale bytes are zero
    // on both sides: products of 2^-249 at most, which no fp32 sum holds).
    const unsigned char *const abase = wq + (int64_t)n0 * G * 16, *const bbase = xq + (int64_t)m0 * G * 16;
    uint32_t row_at[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int r = 8 * (kLoads * wave + j) + (lane >> 3);
        if (8 * (kLoads * wave + j) < kRows)  // (uniform)
            row_at[j] = (uint32_t)(n0 + r < N ? r : N - 1 - n0) * (uint32_t)(G * 16);
        else
            row_at[j] = (uint32_t)(m0 + r - kRows < M ? r - kRows : M - 1 - m0) * (uint32_t)(G * 16);
    }
    const int piece = (lane & 7) ^ (lane >> 4);  // of even instructions; of odd ones piece ^ 4
    auto piece_at = [&](int stage, int odd) -> uint32_t {
        const int b = stage * 8 + (piece ^ (4 * odd));
        return 16u * (uint32_t)(b < G ? b : G - 1);
    };
    auto load = [&](unsigned char *stage, int j, uint32_t even, uint32_t odd) {
        const int first = 8 * (kLoads * wave + j);
        const unsigned char *const base = first < kRows ? abase : bbase;  // (uniform)
        __builtin_amdgcn_global_load_lds((const void *)(base + (row_at[j] + ((kLoads * wave + j) & 1 ? odd : even))),
                                         (lds_void_ptr)(stage + (own + first) * 128), 16, 0, 0);
    };

    // Scales of a window: thread t takes rows t, t + 256 .. of both, 16 bytes each, transposed so that word kb
    // holds what lane-row kb needs in the four steps, zero past the end.
    constexpr int kSc = (kBoth + 255) / 256;
    const unsigned char *scale_row[kSc];
#pragma unroll
    for (int k = 0; k < kSc; ++k) {
        const int r = tid + 256 * k;
        if (r < kRows)
            scale_row[k] = ws + (int64_t)(n0 + r < N ? n0 + r : N - 1) * G;
        else
            scale_row[k] = xs + (int64_t)(m0 + r - kRows < M ? m0 + r - kRows : M - 1) * G;
    }
    typedef uint4v u32x4_any __attribute__((aligned(1)));
    // (16 bytes that all lie in the row: in the last window those that end it)
    auto ask_scales = [&](const unsigned char *row, int window) -> uint4v {
        const int begin = 16 * window < G - 16 ? 16 * window : G - 16;
        return *(const __attribute__((address_space(1))) u32x4_any *)(row + begin);
    };
    auto keep_scales = [&](uint4v v, int k, int window) {
        const int past = 16 * window - (G - 16);  // bytes of `v` before the window's
        if (S > 1 && past >= 16) v = uint4v{0, 0, 0, 0};
        if (past > 0) {  // (uniform)
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
        if (256 * (k + 1) <= kBoth || tid + 256 * k < kBoth)
            *reinterpret_cast<uint4v *>(&scales[4 * (own + tid + 256 * k)]) = transpose_bytes(v);
    };

    float4v sum[P][T];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int t = 0; t < T; ++t) sum[p][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    // LDS -> registers: piece 4 * step + kb of the lane's row
    const int pos0 = i * 128 + 16 * (kb ^ (i >> 1)), pos1 = i * 128 + 16 * ((4 + kb) ^ (i >> 1));
    const int arow = own * 128 + wa * (P * 2048), brow = (own + kRows) * 128 + wb * (T * 2048);
    const int sa_at = (own + wa * P * 16 + i) * 4 + kb, sb_at = (own + kRows + wb * T * 16 + i) * 4 + kb;
#define NVQ_OPERAND(stage_, row_, k_, pos_) *reinterpret_cast<const uint4v *>(&stage_[(row_) + (k_) * 2048 + (pos_)])

    uint4v sc[kSc];
#pragma unroll
    for (int k = 0; k < kSc; ++k) sc[k] = ask_scales(scale_row[k], window0);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load(stage0, j, piece_at(2 * window0, 0), piece_at(2 * window0, 1));
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load(stage1, j, piece_at(2 * window0 + 1, 0), piece_at(2 * window0 + 1, 1));
#pragma unroll
    for (int k = 0; k < kSc; ++k) keep_scales(sc[k], k, window0);
    stage_barrier<kLoads>();
    uint4v a0[P], a1[P], b0[T], b1[T];
    uint32_t sa[P], sb[T], na[P], nb[T];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        a0[p] = NVQ_OPERAND(stage0, arow, p, pos0);
        sa[p] = scales[sa_at + p * 64];
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        b0[t] = NVQ_OPERAND(stage0, brow, t, pos0);
        sb[t] = scales[sb_at + t * 64];
    }

#define NVQ_MULTIPLY(a_, b_, k_)                                                                                    \
    _Pragma("unroll") for (int t = 0; t < T; ++t) multiply_add<k_>(sum[p][t], a_[p], b_[t], sa[p], sb[t]);          \
    __builtin_amdgcn_sched_barrier(0);
#define NVQ_LOADS(stage_, slot_)                                                                                    \
    _Pragma("unroll") for (int j = kLoads * (slot_) / kSlots; j < kLoads * ((slot_) + 1) / kSlots; ++j)             \
        load(stage_, j, even_, odd_);
    // One stage: `cur_` is multiplied (its first operands in a0, b0) and then refilled with stage `ahead_`,
    // `next_` follows.
#define NVQ_STAGE(cur_, next_, k_, ahead_, scales_)                                                                 \
    {                                                                                                               \
        _Pragma("unroll") for (int p = 0; p < kHalf; ++p) {                                                         \
            NVQ_MULTIPLY(a0, b0, k_)                                                                                \
            if (p < kReads) {                                                                                       \
                _Pragma("unroll") for (int o = P * p / kReads; o < P * (p + 1) / kReads; ++o)                       \
                    a1[o] = NVQ_OPERAND(cur_, arow, o, pos1);                                                       \
                _Pragma("unroll") for (int t = T * p / kReads; t < T * (p + 1) / kReads; ++t)                       \
                    b1[t] = NVQ_OPERAND(cur_, brow, t, pos1);                                                       \
            }                                                                                                       \
        }                                                                                                           \
        stage_barrier<63>();                                                                                        \
        const uint32_t even_ = piece_at(ahead_, 0), odd_ = piece_at(ahead_, 1);                                     \
        _Pragma("unroll") for (int p = kHalf; p < P; ++p) {                                                         \
            NVQ_LOADS(cur_, p - kHalf)                                                                              \
            NVQ_MULTIPLY(a0, b0, k_)                                                                                \
        }                                                                                                           \
        _Pragma("unroll") for (int p = 0; p < kHalf; ++p) {                                                         \
            NVQ_LOADS(cur_, kHalf + p)                                                                              \
            NVQ_MULTIPLY(a1, b1, k_ + 1)                                                                            \
        }                                                                                                           \
        stage_barrier<kLoads * P / kSlots>();                                                                       \
        _Pragma("unroll") for (int p = kHalf; p < P; ++p) {                                                         \
            const int q = p - kHalf;                                                                                \
            if (q < kReads) {                                                                                       \
                _Pragma("unroll") for (int o = P * q / kReads; o < P * (q + 1) / kReads; ++o) {                     \
                    a0[o] = NVQ_OPERAND(next_, arow, o, pos0);                                                      \
                    if (scales_) na[o] = scales[sa_at + o * 64];                                                    \
                }                                                                                                   \
                _Pragma("unroll") for (int t = T * q / kReads; t < T * (q + 1) / kReads; ++t) {                     \
                    b0[t] = NVQ_OPERAND(next_, brow, t, pos0);                                                      \
                    if (scales_) nb[t] = scales[sb_at + t * 64];                                                    \
                }                                                                                                   \
            }                                                                                                       \
            NVQ_LOADS(cur_, kHalf + p)                                                                              \
            NVQ_MULTIPLY(a1, b1, k_ + 1)                                                                            \
        }                                                                                                           \
    }
    for (int w = 0; w < windows; ++w) {
        const int wn = w + 1 < windows ? window0 + w + 1 : 0;  // (the last one's loads are of the first: nothing reads them)
#pragma unroll
        for (int k = 0; k < kSc; ++k) sc[k] = ask_scales(scale_row[k], wn);
        NVQ_STAGE(stage0, stage1, 0, 2 * wn, false)
#pragma unroll
        for (int k = 0; k < kSc; ++k) keep_scales(sc[k], k, wn);
        NVQ_STAGE(stage1, stage0, 2, 2 * wn + 1, true)
#pragma unroll
        for (int p = 0; p < P; ++p) sa[p] = na[p];
#pragma unroll
        for (int t = 0; t < T; ++t) sb[t] = nb[t];
    }
#undef NVQ_STAGE
#undef NVQ_LOADS
#undef NVQ_MULTIPLY
#undef NVQ_OPERAND
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int t = 0; t < T; ++t) asm volatile("s_nop 0" : "+a"(sum[p][t]));  // (the last product was written long ago)
    if constexpr (S > 1) {
        // slices 1 .. of S hand over their results, a tile of 64 lanes after the other, half of them in either
        // stage's place
        constexpr int kTiles = P / 2 * T;
        static_assert(4 * kTiles * 1024 <= kBoth * 128, "a slice's results in its part of the stages");
        auto place = [&](int from, int p, int t) -> float4v & {
            unsigned char *const half = p < P / 2 ? stage0 : stage1;
            return reinterpret_cast<float4v *>(half + from * kBoth * 128)[(wave * kTiles + p % (P / 2) * T + t) * 64 + lane];
        };
        if (group) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int t = 0; t < T; ++t) place(group, p, t) = sum[p][t];
        }
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int from = 1; from < S; ++from)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int t = 0; t < T; ++t) sum[p][t] += place(from, p, t);
    }
    static_assert(2 * 16 * (16 * P * 4 + 16) <= kBoth * 128, "two waves' rows of results per stage");
    unsigned char *const out = (wave >> 1 ? stage1 : stage0) + (wave & 1) * (16 * (16 * P * 4 + 16));
    const int first_n = n0 + wa * (16 * P), first_m = m0 + wb * (16 * T);
    if (y_dtype == NVQ_BF16)
        store_tile<P, T, 1, 2>(out, sum, first_n, N, first_m, M, y);
    else
        store_tile<P, T, 1, 4>(out, sum, first_n, N, first_m, M, y);
}

struct GemmArgs {
    const uint8_t *wq, *ws, *xq, *xs;
    void *y;
    int N, M, G, y_dtype;
};

template <int P, int T, int S, int W>
int gemm_tiles(const GemmArgs &a, hipStream_t st) {
    const int64_t tn = ((int64_t)a.N + 32 * P - 1) / (32 * P), tm = ((int64_t)a.M + 32 * T - 1) / (32 * T);
    if (tn * tm * (256 * S) > 0xffffffffLL) return NVQ_ERR_SHAPE;  // (a launch's work items)
    hipLaunchKernelGGL((gemm_mxfp4_kernel<P, T, S, W>), dim3((unsigned)(tn * tm)), dim3(256 * S), 0, st, a.wq, a.ws, a.N,
                       a.G, a.xq, a.xs, a.M, a.y, a.y_dtype, (int)tn);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

int gemm_small_k(const GemmArgs &a, hipStream_t st) {
    const int64_t tn = ((int64_t)a.N + 63) / 64, tm = ((int64_t)a.M + 63) / 64;
    if (tn * tm * 64 > 0xffffffffLL) return NVQ_ERR_SHAPE;  // (a launch's work items)
    hipLaunchKernelGGL(gemm_mxfp4_small_k_kernel, dim3((unsigned)(tn * tm)), dim3(64), 0, st,
                       reinterpret_cast<const uint4 *>(a.wq), a.ws, a.N, a.G, reinterpret_cast<const uint4 *>(a.xq),
                       a.xs, a.M, a.y, a.y_dtype, (int)tn);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_gemm_mxfp4(const uint8_t *qweight, const uint8_t *scales, int64_t N, int64_t K, const uint8_t *xq,
                              const uint8_t *xscale, int64_t M, void *y, int y_dtype, void *stream) {
    using namespace nvq;
    if (!qweight || !scales || !xq || !xscale || !y || (y_dtype != NVQ_F32 && y_dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (N <= 0 || M <= 0 || K <= 0 || K % 32 || K > NVQ_MAX_K || N > (1 << 30) || M > (1 << 30)) return NVQ_ERR_SHAPE;
    if (!aligned(qweight, 16) || !aligned(xq, 16) || !aligned(y, y_dtype == NVQ_F32 ? 4 : 2)) return NVQ_ERR_ALIGN;
    const GemmArgs a = {qweight, scales, xq, xscale, y, (int)N, (int)M, (int)(K / 32), y_dtype};
    const hipStream_t st = (hipStream_t)stream;
    if (K < 512) return gemm_small_k(a, st);
    // The largest tile of which there are enough for the compute units (us; tile rows x tokens, in slices of K):
    //   M x N x K            256x256  128x128  128x64 in 2  64x64 in 2  64x32 in 2  in 4
    //   4096 x 4096 x 4096      42       49         70
    //   2048 x 4096 x 4096      35       26         45          63
    //   1024 x 6144 x 4096      34       23         34          49                   78
    //   2048 x 2048 x 4096      31       16         23          33         35        53
    //   768 x 4096 x 4096       30       16         22          24         27        40
    //   1500 x 3000 x 2048      36       16         22          25         25        41
    //   512 x 4096 x 14336      80       40         32          49                   66
    //   128 x 14336 x 4096      31       15         12          17                   27
    //   256 x 4096 x 4096       29       13        10.3         8.6                  13.5
    //   96 x 6144 x 4096                            9.9         8.0         9.4      12.8
    //   128 x 4096 x 4096                           9.7         7.8         7.2       7.3
    //   128 x 2048 x 14336                         21.7        17.0        15.3      13.6
    //   16 x 4096 x 14336                          24.5        19.7        17.7      14.8
    //   48 x 4096 x 4096                            9.4         7.5         6.7       6.9
    //   77 x 1003 x 2080                           10.5         7.7         6.4       7.3
    const int64_t cus = device_cu_count();
    const auto tiles = [&](int rows, int tokens) { return ((N + rows - 1) / rows) * ((M + tokens - 1) / tokens); };
    if (tiles(256, 256) >= cus * 7 / 8) return gemm_tiles<8, 8, 1, 1>(a, st);
    if (tiles(128, 64) > cus) return gemm_tiles<4, 4, 1, 2>(a, st);
    if (tiles(128, 64) >= cus * 3 / 4) return gemm_tiles<4, 2, 2, 2>(a, st);
    if (tiles(64, 32) > cus) return gemm_tiles<2, 2, 2, 2>(a, st);
    return K >= 8192 ? gemm_tiles<2, 1, 4, 4>(a, st) : gemm_tiles<2, 1, 2, 4>(a, st);
}
