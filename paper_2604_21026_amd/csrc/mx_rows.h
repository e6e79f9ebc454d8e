// Products of 16-row tiles of 4-bit weights with bf16 activations of 16-token tiles on the matrix cores, for
// both weight formats (nvq_gemv_mxfp4, nvq_moe_experts).
//
// A wave takes columns of 128 inputs: lane (n, kb) = (lane % 16, lane / 16) loads the 16 bytes of block 4c + kb
// of row n.  Microscaled: MFMA i (16x16x32) takes dword i of every lane's block, eight codes, which become bf16
// values, scale and all, in one instruction per two (exact: two bits of significand and a power of two); the
// four MFMAs add into the same sums.  Which inputs stand at which place of a product is free: the activations
// follow (lane (m, kb) supplies inputs 32 kb + 8 i .. + 7 of its column), and a lane needs its own block's
// scale alone. int4: each block's product is scaled on its way to the sum, so an MFMA is one block: a 4x4
// transpose across the lane-rows gives the lane dword kb of the blocks 4c .. 4c + 3 (mfma_act.h, as in the
// small-batch kernels of the int4 layers).
#pragma once

#include "mfma_act.h"

namespace nvq {

#if defined(__HIPCC__)

// Codes of C neighbouring columns of a row tile, a lane's 16 bytes of each, and its row's scales of 4 Q blocks,
// Q columns.
template <int C>
struct Codes {
    uint4v w[C];
};
template <int FMT, int Q>
struct Scales {
    uint32_t s[FMT == NVQ_FMT_MXFP4 ? Q : 2 * Q];  // four scale bytes, or fp16, per column
};

template <int FMT>
constexpr int scale_bytes() {
    return FMT == NVQ_FMT_MXFP4 ? 1 : 2;
}

// The codes q and scales s of a lane's row (s at any alignment of its type).
struct RowAt {
    const uint4 *q;
    const char *s;
};

template <int FMT>
__device__ __forceinline__ RowAt row_at(const uint8_t *q, const void *s, int64_t row, int G) {
    return RowAt{reinterpret_cast<const uint4 *>(q) + row * G,
                 reinterpret_cast<const char *>(s) + row * G * scale_bytes<FMT>()};
}

// Columns col .. of that many.  (A row's line of 128 bytes of codes is two columns: asked for together it is
// fetched once.)
template <int C>
__device__ __forceinline__ void load_codes(Codes<C> &c, const RowAt &at, int col, int kb) {
#pragma unroll
    for (int b = 0; b < C; ++b) c.w[b] = load_stream(at.q + 4 * (col + b) + kb);
}
// (A line of scales serves 32 columns of microscaled rows; asked for a column or two at a time it was fetched
// again every time, as many bytes as the codes are.)
template <int FMT, int Q>
__device__ __forceinline__ void load_scales(Scales<FMT, Q> &c, const RowAt &at, int col) {
    constexpr int kWords = FMT == NVQ_FMT_MXFP4 ? Q : 2 * Q, kWide = kWords < 4 ? kWords : 4;
    typedef uint32_t words __attribute__((ext_vector_type(kWide)));
    typedef words words_any __attribute__((aligned(1)));
    static_assert(kWords % kWide == 0, "");
#pragma unroll
    for (int k = 0; k < kWords / kWide; ++k) {
        const words v = *(const __attribute__((address_space(1))) words_any *)(at.s + 4 * scale_bytes<FMT>() * col + 4 * kWide * k);
#pragma unroll
        for (int b = 0; b < kWide; ++b) c.s[kWide * k + b] = v[b];
    }
}

// Scales of zero for the first `blocks` blocks (uniform), whose activations are zero: values beyond bf16 would
// make them NaN.
template <int FMT, int Q>
__device__ __forceinline__ void clear_scales(Scales<FMT, Q> &c, int blocks) {
    constexpr int kWords = FMT == NVQ_FMT_MXFP4 ? Q : 2 * Q;
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const int bytes = blocks * scale_bytes<FMT>() - 4 * k;
        c.s[k] &= bytes <= 0 ? ~0u : bytes >= 4 ? 0u : ~0u << (8 * bytes);
    }
}

// Column col, with `blocks` (1 to 4) of its four blocks in the row: the others are zero.
template <int FMT>
__device__ __forceinline__ void load_last(Codes<1> &c, Scales<FMT, 1> &sc, const RowAt &at, int col, int kb, int blocks) {
    c.w[0] = uint4v{0, 0, 0, 0};
    if (kb < blocks) c.w[0] = load_stream(at.q + 4 * col + kb);
    uint32_t s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < blocks)
            s[i] = FMT == NVQ_FMT_MXFP4 ? as_global<uint8_t>(at.s)[4 * col + i] : as_global<uint16_t>(at.s)[4 * col + i];
    if constexpr (FMT == NVQ_FMT_MXFP4) {
        sc.s[0] = s[0] | s[1] << 8 | s[2] << 16 | s[3] << 24;
    } else {
        sc.s[0] = s[0] | s[1] << 16;
        sc.s[1] = s[2] | s[3] << 16;
    }
}

// 2^(byte - 127) of byte kb of the word, as the conversions take it (they look at the exponent alone, 0
// standing for 2^-127).
__device__ __forceinline__ float mx_scale_of(uint32_t four, int kb) {
    return __uint_as_float(__builtin_amdgcn_ubfe(four, 8 * kb, 8) << 23);
}

// Where piece i of the lane's activations of a column begins (bytes from the token's first one of the column).
template <int FMT>
__device__ __forceinline__ int piece_at(int i, int kb) {
    return FMT == NVQ_FMT_MXFP4 ? 64 * kb + 16 * i : 64 * i + 16 * kb;
}

// Eight codes as bf16 values with their block's scale.
__device__ __forceinline__ bf16x8 mx_values(uint32_t codes, float s) {
    const uint4v v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
    return __builtin_bit_cast(bf16x8, v);
}

// The operands of a column from the lane's pieces of its token's 128 inputs.
template <int FMT>
__device__ __forceinline__ void to_operands(const uint4v (&raw)[4], bf16x8 (&a)[4]) {
    if constexpr (FMT == NVQ_FMT_MXFP4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_bit_cast(bf16x8, raw[i]);
    } else {
        Act<NVQ_W4A16>::operands(raw, a);
    }
}

// sum[r][t] += tile r times token tile t over column b of the codes loaded, qb of the scales.
template <int FMT, int R, int T, int C, int Q>
__device__ __forceinline__ void multiply_column(const Codes<C> (&col)[R], int b, const Scales<FMT, Q> (&sc)[R], int qb,
                                                const bf16x8 (&a)[T][4], float4v (&sum)[R][T]) {
    typedef Act<NVQ_W4A16> A;
    if constexpr (FMT == NVQ_FMT_MXFP4) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t q[4] = {col[r].w[b].x, col[r].w[b].y, col[r].w[b].z, col[r].w[b].w};
            const float s = mx_scale_of(sc[r].s[qb], (threadIdx.x & 63) >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 w = mx_values(q[i], s);
#pragma unroll
                for (int t = 0; t < T; ++t)
                    sum[r][t] = A::multiply(a[t][i], w, sum[r][t]);
            }
        }
    } else {
        uint32_t q[R][4];
        float s[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            q[r][0] = col[r].w[b].x;
            q[r][1] = col[r].w[b].y;
            q[r][2] = col[r].w[b].z;
            q[r][3] = col[r].w[b].w;
            transpose_rows(q[r]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s[r][i] = half_bits_to_float((uint16_t)(sc[r].s[2 * qb + (i >> 1)] >> (16 * (i & 1))));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4v off[T];
#pragma unroll
            for (int t = 0; t < T; ++t) off[t] = A::offset(a[t][i]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bf16x8 w = A::weights(q[r][i]);
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const float4v p = A::multiply(a[t][i], w, off[t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[r][t][j] = fmaf(s[r][i], p[j], sum[r][t][j]);
                }
            }
        }
    }
}

// ... over the columns from `column` on, one by one, the waves in turn (`turn`: whose it is at the first).
template <int FMT, int R, int T>
__device__ __forceinline__ void last_columns(const RowAt (&at)[R], const char *const (&x)[T], int G, int column, int turn,
                                             int first, int step, float4v (&sum)[R][T]) {
    const int kb = (threadIdx.x & 63) >> 4;
    const int columns = (G + 3) >> 2;
    for (int c = column; c < columns; ++c, ++turn) {
        if (turn % step != first) continue;  // (wave-uniform)
        const int blocks = G - 4 * c < 4 ? G - 4 * c : 4;
        Codes<1> col[R];
        Scales<FMT, 1> sc[R];
        uint4v raw[T][4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (blocks == 4) {  // (uniform)
                load_codes<1>(col[r], at[r], c, kb);
                load_scales<FMT, 1>(sc[r], at[r], c);
            } else {
                load_last<FMT>(col[r], sc[r], at[r], c, kb, blocks);
            }
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                raw[t][i] = uint4v{0, 0, 0, 0};
                if ((FMT == NVQ_FMT_MXFP4 ? kb : i) < blocks)
                    raw[t][i] = *as_global<uint4v>(x[t] + (size_t)c * 256 + piece_at<FMT>(i, kb));
            }
        bf16x8 a[T][4];
#pragma unroll
        for (int t = 0; t < T; ++t) to_operands<FMT>(raw[t], a[t]);
        multiply_column<FMT, R, T, 1, 1>(col, 0, sc, 0, a, sum);
    }
}

// A column that counts for nothing: codes of zero, or scales of zero, and activations of zero (an infinite one
// would make them NaN).
template <int FMT, int R, int T, int C, int Q>
__device__ __forceinline__ void clear_column(Codes<C> (&col)[R], uint4v (&raw)[C][T][4], int b,
                                             Scales<FMT, Q> (&sc)[R], int qb) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if constexpr (FMT == NVQ_FMT_MXFP4)
            col[r].w[b] = uint4v{0, 0, 0, 0};
        else
            sc[r].s[2 * qb] = sc[r].s[2 * qb + 1] = 0;
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[b][t][i] = uint4v{0, 0, 0, 0};
}

// sum[r][t] += R row tiles times T token tiles over K = 32 G inputs, shared out over `step` waves (this one:
// number `first`) in passes of Q columns: their scales at once, their codes and activations C columns at a
// time, requested while the C before are multiplied.  A last pass of fewer columns takes the last Q, and those
// that it shares with the one before count for nothing: they are left out (kSkip) or cleared.  (Left out in
// tiles of two steps or two token tiles, the branches cost up to a tenth, 8 tokens of 14336 x 4096 10.0 and
// 11.0 us; cleared in the others, up to 7 %.)  x[t]: the lane's token of tile t (bf16); a product keeps tokens
// apart, so a lane without one may take any.  (Loading nothing in such lanes was no faster.)  Every lane of the
// wave calls it.
template <int FMT, int R, int T, int C, int Q>
__device__ __forceinline__ void rows_times_tokens(const RowAt (&at)[R], const char *const (&x)[T], int G, int first,
                                                  int step, float4v (&sum)[R][T]) {
    static_assert(Q % C == 0, "");
    constexpr bool kSkip = Q == C && T == 1;
    const int kb = (threadIdx.x & 63) >> 4;
    const int full = G >> 2, passes = full >= Q ? (full + Q - 1) / Q : 0;
    auto load = [&](Codes<C> (&col)[R], uint4v (&raw)[C][T][4], int c) {
#pragma unroll
        for (int r = 0; r < R; ++r) load_codes<C>(col[r], at[r], c, kb);
#pragma unroll
        for (int b = 0; b < C; ++b)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    raw[b][t][i] = *as_global<uint4v>(x[t] + (size_t)(c + b) * 256 + piece_at<FMT>(i, kb));
    };
    for (int p = first; p < passes; p += step) {
        const int c0 = p * Q + Q <= full ? p * Q : full - Q, again = p * Q - c0;  // (uniform)
        Scales<FMT, Q> sc[R];
        Codes<C> col[2][R];
        uint4v raw[2][C][T][4];
#pragma unroll
        for (int r = 0; r < R; ++r) load_scales<FMT, Q>(sc[r], at[r], c0);
        load(col[0], raw[0], c0);
#pragma unroll
        for (int q = 0; q < Q / C; ++q) {
            if (q + 1 < Q / C) load(col[(q + 1) & 1], raw[(q + 1) & 1], c0 + (q + 1) * C);
            __builtin_amdgcn_sched_barrier(0);
            auto one = [&](int b) {
                bf16x8 a[T][4];
#pragma unroll
                for (int t = 0; t < T; ++t) to_operands<FMT>(raw[q & 1][b][t], a[t]);
                multiply_column<FMT, R, T, C, Q>(col[q & 1], b, sc, q * C + b, a, sum);
            };
            if (kSkip && again > 0) {  // (uniform)
#pragma unroll
                for (int b = 0; b < C; ++b)
                    if (b >= again) one(b);
            } else {
#pragma unroll
                for (int b = 0; b < C; ++b) {
                    if (!kSkip && q * C + b < Q - 1 && q * C + b < again)
                        clear_column<FMT, R, T, C, Q>(col[q & 1], raw[q & 1], b, sc, q * C + b);
                    one(b);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    last_columns<FMT, R, T>(at, x, G, passes ? full : 0, passes, first, step, sum);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) wait_written(sum[r][t]);
}

#endif  // __HIPCC__

}  // namespace nvq
