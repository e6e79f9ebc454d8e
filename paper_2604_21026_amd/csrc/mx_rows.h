// Products of 16-row tiles of 4-bit weights with bf16 activations of 16-token tiles on the matrix cores, for
// both weight formats (nvq_gemv_mxfp4, nvq_moe_experts).
//
// A wave takes columns of 128 inputs: lane (n, kb) = (lane % 16, lane / 16) loads the 16 bytes of block 4c + kb of
// row n and, after a 4x4 transpose across the lane-rows, has dword kb of the blocks 4c .. 4c + 3, eight inputs of
// each.  One 16x16x32 MFMA multiplies one block of 16 rows with 16 tokens.  Microscaled codes become bf16 values,
// scale and all, in one instruction per two (exact: two bits of significand and a power of two), and all blocks
// add up in the accumulators; int4 codes enter as in the small-batch kernels of the int4 layers (mfma_act.h), and each
// block's product is scaled on its way to the sum.
#pragma once

#include "mfma_act.h"

namespace nvq {

#if defined(__HIPCC__)

// One column of a row tile: a lane's 16 bytes of codes and its row's scales of the four blocks.
template <int FMT>
struct RowColumn;

template <>
struct RowColumn<NVQ_FMT_MXFP4> {
    uint4v w;
    uint32_t s;  // four scale bytes
};

template <>
struct RowColumn<NVQ_FMT_INT4> {
    uint4v w;
    uint2v s;  // four fp16
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

template <int FMT>
__device__ __forceinline__ void load_column(RowColumn<FMT> &c, const RowAt &at, int col, int kb) {
    typedef uint32_t u32_any __attribute__((aligned(1)));
    typedef uint2v u32x2_any __attribute__((aligned(2)));
    c.w = load_stream(at.q + 4 * col + kb);
    if constexpr (FMT == NVQ_FMT_MXFP4)
        c.s = *(const __attribute__((address_space(1))) u32_any *)(at.s + 4 * col);
    else
        c.s = *(const __attribute__((address_space(1))) u32x2_any *)(at.s + 8 * col);
}

// The last column, with `blocks` (1 to 3) of its four blocks: the others are zero.
template <int FMT>
__device__ __forceinline__ void load_last(RowColumn<FMT> &c, const RowAt &at, int col, int kb, int blocks) {
    c.w = uint4v{0, 0, 0, 0};
    if (kb < blocks) c.w = load_stream(at.q + 4 * col + kb);
    uint32_t s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < blocks)
            s[i] = FMT == NVQ_FMT_MXFP4 ? as_global<uint8_t>(at.s)[4 * col + i] : as_global<uint16_t>(at.s)[4 * col + i];
    if constexpr (FMT == NVQ_FMT_MXFP4)
        c.s = s[0] | s[1] << 8 | s[2] << 16;
    else
        c.s = uint2v{s[0] | s[1] << 16, s[2]};
}

__device__ __forceinline__ void clear_column(RowColumn<NVQ_FMT_MXFP4> &c) { c.w = uint4v{0, 0, 0, 0}; }
__device__ __forceinline__ void clear_column(RowColumn<NVQ_FMT_INT4> &c) { c.s = uint2v{0, 0}; }

// 2^(byte - 127) as the conversions take it (they look at the exponent alone, 0 standing for 2^-127).
template <int I>
__device__ __forceinline__ float mx_scale_of(uint32_t four) {
    return __uint_as_float(I == 0   ? (four & 0xffu) << 23
                           : I == 1 ? (four & 0xff00u) << 15
                           : I == 2 ? (four & 0xff0000u) << 7
                                    : four >> 24 << 23);
}

// Eight codes as bf16 values with their block's scale.
__device__ __forceinline__ bf16x8 mx_values(uint32_t codes, float s) {
    const uint4v v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
    return __builtin_bit_cast(bf16x8, v);
}

// sum[r][t] += tile r times token tile t over one column.  raw: the lane's pieces of its token's 128 inputs.
template <int FMT, int R, int T>
__device__ __forceinline__ void multiply_column(const RowColumn<FMT> (&col)[R], const uint4v (&raw)[T][4],
                                                float4v (&sum)[R][T]) {
    typedef Act<NVQ_W4A16> A;
    if constexpr (FMT == NVQ_FMT_MXFP4) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            uint32_t q[4] = {col[r].w.x, col[r].w.y, col[r].w.z, col[r].w.w};
            transpose_rows(q);
            const float s[4] = {mx_scale_of<0>(col[r].s), mx_scale_of<1>(col[r].s), mx_scale_of<2>(col[r].s),
                                mx_scale_of<3>(col[r].s)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 w = mx_values(q[i], s[i]);
#pragma unroll
                for (int t = 0; t < T; ++t)
                    sum[r][t] = A::multiply(__builtin_bit_cast(bf16x8, raw[t][i]), w, sum[r][t]);
            }
        }
    } else {
        bf16x8 a[T][4];
#pragma unroll
        for (int t = 0; t < T; ++t) A::operands(raw[t], a[t]);
        uint32_t q[R][4];
        float s[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            q[r][0] = col[r].w.x;
            q[r][1] = col[r].w.y;
            q[r][2] = col[r].w.z;
            q[r][3] = col[r].w.w;
            transpose_rows(q[r]);
            s[r][0] = half_bits_to_float((uint16_t)(col[r].s.x & 0xffffu));
            s[r][1] = half_bits_to_float((uint16_t)(col[r].s.x >> 16));
            s[r][2] = half_bits_to_float((uint16_t)(col[r].s.y & 0xffffu));
            s[r][3] = half_bits_to_float((uint16_t)(col[r].s.y >> 16));
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

// sum[r][t] += R row tiles times T token tiles over the columns first, first + step, ... of K = 32 G inputs, B
// columns requested at a time.  x[t]: the lane's token of tile t (bf16, at input 8 * kb).  Every lane of the
// wave calls it.
template <int FMT, int R, int T, int B>
__device__ __forceinline__ void rows_times_tokens(const RowAt (&at)[R], const char *const (&x)[T], int G, int first,
                                                  int step, float4v (&sum)[R][T]) {
    typedef Act<NVQ_W4A16> A;
    const int kb = (threadIdx.x & 63) >> 4;
    const int full = G >> 2;
    for (int c0 = first; c0 < full; c0 += step * B) {
        RowColumn<FMT> col[B][R];
        uint4v raw[B][T][4];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int c = c0 + b * step;
            const int cc = c < full ? c : full - 1;  // (wave-uniform)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                load_column<FMT>(col[b][r], at[r], cc, kb);
                if (c >= full) clear_column(col[b][r]);
            }
#pragma unroll
            for (int t = 0; t < T; ++t) A::load(x[t] + (size_t)cc * 256, raw[b][t]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < B; ++b) multiply_column<FMT, R, T>(col[b], raw[b], sum);
    }
    const int blocks = G & 3;
    if (blocks && full % step == first) {  // (wave-uniform)
        RowColumn<FMT> col[R];
        uint4v raw[T][4];
#pragma unroll
        for (int r = 0; r < R; ++r) load_last<FMT>(col[r], at[r], full, kb, blocks);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                raw[t][i] = uint4v{0, 0, 0, 0};
                if (i < blocks) raw[t][i] = *as_global<uint4v>(x[t] + (size_t)full * 256 + 64 * i);
            }
        multiply_column<FMT, R, T>(col, raw, sum);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) wait_written(sum[r][t]);
}

#endif  // __HIPCC__

}  // namespace nvq
