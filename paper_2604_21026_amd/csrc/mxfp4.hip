// nvq_quant_mxfp4 / nvq_dequant_mxfp4: microscaled 4-bit floating point.  A block of 32 values shares the
// power of two s = 2^(floor(log2(absmax)) - 2), kept as its biased exponent in a byte; a value is held as
// e2m1(x / s), rounded to nearest even, what lies beyond 6 at 6 (absmax / s is in [4, 8)).
//
// The block's exponent is that of its largest magnitude's bits, and gfx950 divides by a power of two, rounds
// and packs two values in one instruction, so that memory bounds both directions.  A lane takes 16 bytes of
// input: eight lanes of four fp32 values or four lanes of eight bf16 values make a block and find its
// maximum with two or three data-parallel moves; the codes leave as whole words, the scales of four blocks
// as one.
//
// Measured at 14336 x 4096: fp32 to codes 42.7 us (6.2 TB/s; 49.8 with one load in flight per lane, 43.8 with
// two or eight), codes to bf16 22.4 (6.6 TB/s); 8 x 2048 2.4 us each, an empty launch.
#include "mfma_act.h"

namespace nvq {

namespace {

struct OrOp {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a | b; }
};
struct MaxBitsOp {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

constexpr uint32_t kMxNan = 0xffu;  // the scale byte that stands for no number

// The scale byte of a block from the bits of its largest magnitude: an infinity or NaN gives kMxNan.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e == 0xffu ? kMxNan : e > 2 ? e - 2 : 0u;
}

// 2^(byte - 127) as fp32: byte 0 is 2^-127, a subnormal number.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __uint_as_float(byte ? byte << 23 : 0x400000u);
}

// Four scale bytes, one of each block of four in its lanes' low byte, as a word in all of their lanes.
// LPB: lanes per block (4 or 8).
template <int LPB>
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte, int lane) {
    uint32_t v = byte << (8 * (lane / LPB & 3));
    if (LPB == 8) v = with_lane_xor<16>(v, OrOp());
    v = with_lane_xor<8>(v, OrOp());
    if (LPB == 4) v = with_lane_xor<4>(v, OrOp());
    return v;
}

// T = float: four values per lane, eight lanes per block; bf16 bits: eight values, four lanes.
template <bool BF16, int U>
__global__ __launch_bounds__(256) void quant_mxfp4_kernel(const uint4 *__restrict__ x, int64_t blocks,
                                                          uint32_t *__restrict__ q, uint8_t *__restrict__ scales) {
    constexpr int kLanes = BF16 ? 4 : 8, kPerLoad = 256 / kLanes;  // blocks of a workgroup's load
    const int lane = threadIdx.x & 63, sub = threadIdx.x % kLanes;
    const int64_t first = (int64_t)blockIdx.x * (U * kPerLoad) + threadIdx.x / kLanes;
    uint4v v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        int64_t b = first + i * kPerLoad;
        if (b >= blocks) b = blocks - 1;  // (the lanes stay in the exchanges below)
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const uint4v *>(x) + b * kLanes + sub);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t b = first + i * kPerLoad;
        uint32_t top;
        if (BF16) {
            // magnitudes order as their bits do; the upper halves keep theirs, with the lower halves behind
            uint32_t hi = 0, lo = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                hi = MaxBitsOp()(hi, v[i][k] & 0x7fffffffu);
                lo = MaxBitsOp()(lo, v[i][k] << 16 & 0x7fffffffu);
            }
            top = MaxBitsOp()(hi, lo);
        } else {
            top = MaxBitsOp()(MaxBitsOp()(v[i].x & 0x7fffffffu, v[i].y & 0x7fffffffu),
                              MaxBitsOp()(v[i].z & 0x7fffffffu, v[i].w & 0x7fffffffu));
        }
        if (!BF16) top = with_lane_xor<1>(top, MaxBitsOp());
        top = BF16 ? with_lane_xor<1>(top, MaxBitsOp()) : with_lane_xor<2>(top, MaxBitsOp());
        if (BF16)
            top = with_lane_xor<2>(top, MaxBitsOp());
        else  // (the mirror of eight lanes: the other four)
            top = MaxBitsOp()(top, (uint32_t)__builtin_amdgcn_update_dpp((int)top, (int)top, 0x141, 0xf, 0xf, false));
        const uint32_t byte = mx_scale_byte(top);
        const float s = mx_scale(byte);
        uint32_t codes = 0;
        if (BF16) {
            // (a bit cast of an element in place takes element 0)
            const uint32_t p0 = v[i].x, p1 = v[i].y, p2 = v[i].z, p3 = v[i].w;
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(nvq_bf16x2, p0), s, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(nvq_bf16x2, p1), s, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(nvq_bf16x2, p2), s, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(nvq_bf16x2, p3), s, 3);
        } else {
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[i].x), __uint_as_float(v[i].y), s, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[i].z), __uint_as_float(v[i].w), s, 1);
            // the neighbour's four codes behind the own ones (for even lanes)
            const uint32_t next = (uint32_t)__builtin_amdgcn_update_dpp((int)codes, (int)codes, 0xb1, 0xf, 0xf, false);
            codes = (codes & 0xffffu) | next << 16;
        }
        if (byte == kMxNan) codes = 0;
        const uint32_t four = gather_scales<kLanes>(byte, lane);
        if (b < blocks) {
            if (BF16)
                q[b * 4 + sub] = codes;
            else if ((sub & 1) == 0)
                q[b * 4 + sub / 2] = codes;
            // blocks b .. b + 3 begin at a multiple of four
            if ((b | 3) < blocks) {
                if (sub == 0 && (b & 3) == 0) *reinterpret_cast<uint32_t *>(scales + b) = four;
            } else if (sub == 0) {
                scales[b] = (uint8_t)byte;
            }
        }
    }
}

// A lane unpacks four bytes of codes, eight values, a quarter of a block.
template <int U>
__global__ __launch_bounds__(256) void dequant_mxfp4_kernel(const uint32_t *__restrict__ q,
                                                            const uint8_t *__restrict__ scales, int64_t words,
                                                            uint4 *__restrict__ out) {
    const int64_t first = (int64_t)blockIdx.x * (256 * U) + threadIdx.x;
    uint32_t c[U], byte[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        int64_t w = first + i * 256;
        if (w >= words) w = words - 1;
        c[i] = q[w];
        byte[i] = scales[w >> 2];
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t w = first + i * 256;
        if (w >= words) return;
        const float s = mx_scale(byte[i]);
        uint4v o = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 3))};
        if (byte[i] == kMxNan) o = uint4v{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
        *reinterpret_cast<uint4v *>(out + w) = o;
    }
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_quant_mxfp4(const void *x, int x_dtype, int64_t M, int64_t K, uint8_t *q, uint8_t *scales,
                               void *stream) {
    if (!x || !q || !scales || (x_dtype != NVQ_F32 && x_dtype != NVQ_BF16)) return NVQ_ERR_INVALID_ARG;
    if (M <= 0 || K <= 0 || K % 32 || K > NVQ_MAX_K || M > (INT64_C(1) << 34) / K) return NVQ_ERR_SHAPE;
    if (!nvq::aligned(x, 16) || !nvq::aligned(q, 16) || !nvq::aligned(scales, 4)) return NVQ_ERR_ALIGN;
    const int64_t blocks = M * (K / 32);
    constexpr int U = 4;
    const int64_t per = x_dtype == NVQ_BF16 ? U * 64 : U * 32, grid = (blocks + per - 1) / per;
    if (x_dtype == NVQ_BF16)
        hipLaunchKernelGGL((nvq::quant_mxfp4_kernel<true, U>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream,
                           reinterpret_cast<const uint4 *>(x), blocks, reinterpret_cast<uint32_t *>(q), scales);
    else
        hipLaunchKernelGGL((nvq::quant_mxfp4_kernel<false, U>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream,
                           reinterpret_cast<const uint4 *>(x), blocks, reinterpret_cast<uint32_t *>(q), scales);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

extern "C" int nvq_dequant_mxfp4(const uint8_t *q, const uint8_t *scales, int64_t M, int64_t K, uint16_t *out_bf16,
                                 void *stream) {
    if (!q || !scales || !out_bf16) return NVQ_ERR_INVALID_ARG;
    if (M <= 0 || K <= 0 || K % 32 || K > NVQ_MAX_K || M > (INT64_C(1) << 34) / K) return NVQ_ERR_SHAPE;
    if (!nvq::aligned(q, 16) || !nvq::aligned(out_bf16, 16)) return NVQ_ERR_ALIGN;
    constexpr int U = 4;
    const int64_t words = M * (K / 8), grid = (words + 256 * U - 1) / (256 * U);
    hipLaunchKernelGGL((nvq::dequant_mxfp4_kernel<U>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream,
                       reinterpret_cast<const uint32_t *>(q), scales, words, reinterpret_cast<uint4 *>(out_bf16));
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
