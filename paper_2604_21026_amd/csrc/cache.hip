// nvq_cache_append, nvq_cache_read: keys and values of new tokens into the paged cache, and out of it again.
#include "cache.h"

namespace nvq {

int check_cache(const nvq_cache *c) {
    if (!c || !c->k || !c->v || (c->dtype != NVQ_BF16 && c->dtype != NVQ_E4M3) || (c->dtype == NVQ_E4M3 && !c->scales))
        return NVQ_ERR_INVALID_ARG;
    if (c->pages < 1 || c->heads < 1 || c->heads > NVQ_MAX_HEADS || c->page_size < 8 || c->page_size > NVQ_MAX_PAGE ||
        (c->page_size & (c->page_size - 1)) || c->head_dim < 32 || c->head_dim > NVQ_MAX_HEAD_DIM || c->head_dim % 32)
        return NVQ_ERR_SHAPE;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || (c->dtype == NVQ_E4M3 && !aligned(c->scales, 8))) return NVQ_ERR_ALIGN;
    return NVQ_OK;
}

int check_places(const Places &p) {
    if (!p.table || !p.positions) return NVQ_ERR_INVALID_ARG;
    if (p.B < 1 || p.width < 1 || p.T < 1 || p.T > 1 << 24) return NVQ_ERR_SHAPE;
    if (!aligned(p.table, 4) || !aligned(p.positions, 4) || !aligned(p.sequences, 4)) return NVQ_ERR_ALIGN;
    return NVQ_OK;
}

CacheView view_of(const nvq_cache &c) {
    CacheView v;
    v.k = c.k;
    v.v = c.v;
    v.scales = c.scales;
    v.pages = c.pages;
    v.heads = c.heads;
    v.page_size = c.page_size;
    v.page_shift = __builtin_ctz((unsigned)c.page_size);
    v.D = c.head_dim;
    v.e4m3 = c.dtype == NVQ_E4M3;
    return v;
}

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxRows = 1 << 26;  // of a call: at most 32 threads each, fewer than 2^32 in all

struct Place {
    int page, slot, position;
    bool used;
};

__device__ __forceinline__ Place place_of(const CacheView &c, const Places &p, int t, int angles) {
    Place r;
    const int b = p.sequences ? p.sequences[t] : t;
    r.position = p.positions[t];
    r.used = (unsigned)b < (unsigned)p.B && r.position >= 0 && r.position >> c.page_shift < p.width &&
             (angles == 0 || r.position < angles);
    r.page = r.used ? p.table[(int64_t)b * p.width + (r.position >> c.page_shift)] : -1;
    r.used = (unsigned)r.page < (unsigned)c.pages;
    r.slot = r.position & (c.page_size - 1);
    return r;
}

struct AppendArgs {
    CacheView c;
    Places p;
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    uint16_t *q_out;
    const float *cos_sin;
    int H, angles, rot, interleaved;
};

struct MaxBits {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// The largest of L neighbouring lanes (a power of two up to 16).
template <int L>
__device__ __forceinline__ uint32_t most_of(uint32_t v) {
    if (L >= 16) v = with_lane_xor<8>(v, MaxBits());
    // (with_lane_xor<4> rotates by four among sixteen: right where lanes eight apart agree or lie in other groups
    // that do not matter, so groups of eight take the plain exchange)
    if (L >= 16) v = with_lane_xor<4>(v, MaxBits());
    if (L == 8) v = MaxBits()(v, (uint32_t)__shfl_xor((int)v, 4));
    if (L >= 4) v = with_lane_xor<2>(v, MaxBits());
    if (L >= 2) v = with_lane_xor<1>(v, MaxBits());
    return v;
}

// The scale byte of a row whose largest magnitude has these bf16 bits: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f80u) return 255;
    const int b = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u);
    return b < 1 ? 1 : (uint32_t)b;
}

// Eight values -> codes under that scale byte (255: zeros).
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], uint32_t byte) {
    if (byte == 255) return make_uint2(0, 0);
    const float up = __uint_as_float((254u - byte) << 23);  // (byte 1 to 246: a normal number)
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * up, x[4 * i + 1] * up, 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * up, x[4 * i + 3] * up, r, true);
    }
    return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void unpack(const uint4 &w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ uint32_t top_bits(const uint4 &w) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = v[i] & 0x7fffu, hi = v[i] >> 16 & 0x7fffu;
        m = m > lo ? m : lo;
        m = m > hi ? m : hi;
    }
    return m;
}

// A row (one head of one token) by L lanes, sixteen of its channels each: two pieces of eight, which are each other's
// partners of the rotation, or hold whole pairs.
template <int L>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendArgs a) {
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
    const int i = threadIdx.x % L, D = a.c.D;
    const int rows = a.H + 2 * a.c.heads;
    const int64_t t64 = unit / rows;
    const bool lane = t64 < a.p.T && i < D / 16;
    const int t = t64 < a.p.T ? (int)t64 : 0;
    int h = (int)(unit - t64 * rows);
    const Place at = place_of(a.c, a.p, t, a.angles);
    const int kind = h < a.H ? 0 : h < a.H + a.c.heads ? 1 : 2;  // query, key, value
    h -= kind == 0 ? 0 : kind == 1 ? a.H : a.H + a.c.heads;
    const bool on = lane && at.used;
    const uint16_t *const row = (kind == 0   ? a.q + t * a.q_stride
                                 : kind == 1 ? a.k + t * a.k_stride
                                             : a.v + t * a.v_stride) + h * D;
    const bool halves = kind < 2 && !a.interleaved && i < a.rot / 16;
    const int o0 = halves ? 8 * i : kind < 2 && !a.interleaved ? a.rot + 16 * (i - a.rot / 16) : 16 * i;
    const int o1 = halves ? o0 + a.rot / 2 : o0 + 8;
    uint4 w0 = {}, w1 = {};
    if (on) {
        w0 = *reinterpret_cast<const uint4 *>(row + o0);
        w1 = *reinterpret_cast<const uint4 *>(row + o1);
    }
    if (on && kind < 2 && i < a.rot / 16) {
        const float *const cs = a.cos_sin + (int64_t)at.position * a.rot + 8 * i;
        float x0[8], x1[8], c[8], s[8];
        unpack(w0, x0);
        unpack(w1, x1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = cs[j];
            s[j] = cs[a.rot / 2 + j];
        }
        if (a.interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = x0[2 * j], q = x0[2 * j + 1], u = x1[2 * j], v = x1[2 * j + 1];
                x0[2 * j] = p * c[j] - q * s[j];
                x0[2 * j + 1] = q * c[j] + p * s[j];
                x1[2 * j] = u * c[4 + j] - v * s[4 + j];
                x1[2 * j + 1] = v * c[4 + j] + u * s[4 + j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = x0[j], q = x1[j];
                x0[j] = p * c[j] - q * s[j];
                x1[j] = q * c[j] + p * s[j];
            }
        }
        w0 = pack(x0);
        w1 = pack(x1);
    }
    if (kind == 0) {
        if (on) {
            uint16_t *const out = a.q_out + ((int64_t)t * a.H + h) * D;
            *reinterpret_cast<uint4 *>(out + o0) = w0;
            *reinterpret_cast<uint4 *>(out + o1) = w1;
        }
    }
    uint32_t byte = 0;
    uint2 c0 = {}, c1 = {};
    if (a.c.e4m3) {
        const uint32_t m0 = top_bits(w0), m1 = top_bits(w1);
        byte = scale_byte(most_of<L>(m0 > m1 ? m0 : m1));
        float x0[8], x1[8];
        unpack(w0, x0);
        unpack(w1, x1);
        c0 = codes_of(x0, byte);
        c1 = codes_of(x1, byte);
    }
    if (!on || kind == 0) return;
    if (a.c.e4m3 && i == 0) a.c.scales[scale_at(a.c, at.page, h, kind - 1, at.slot)] = (uint8_t)byte;
    if (kind == 1) {
        const int64_t to = key_at(a.c, at.page, h, at.slot);
        if (a.c.e4m3) {
            uint8_t *const out = static_cast<uint8_t *>(a.c.k) + to;
            *reinterpret_cast<uint2 *>(out + o0) = c0;
            *reinterpret_cast<uint2 *>(out + o1) = c1;
        } else {
            uint16_t *const out = static_cast<uint16_t *>(a.c.k) + to;
            *reinterpret_cast<uint4 *>(out + o0) = w0;
            *reinterpret_cast<uint4 *>(out + o1) = w1;
        }
        return;
    }
    const int64_t to = value_at(a.c, at.page, h, at.slot) + 8 * (int64_t)o0;  // (o1 = o0 + 8)
    if (a.c.e4m3) {
        uint8_t *const out = static_cast<uint8_t *>(a.c.v) + to;
        const uint32_t v[4] = {c0.x, c0.y, c1.x, c1.y};
#pragma unroll
        for (int j = 0; j < 16; ++j) out[8 * j] = (uint8_t)(v[j >> 2] >> 8 * (j & 3));
    } else {
        uint16_t *const out = static_cast<uint16_t *>(a.c.v) + to;
        const uint32_t v[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int j = 0; j < 16; ++j) out[8 * j] = (uint16_t)(v[j >> 1] >> 16 * (j & 1));
    }
}

struct ReadArgs {
    CacheView c;
    Places p;
    uint16_t *k, *v;
};

typedef float float2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint4 values_of(uint2 codes, float scale) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? codes.x : codes.y;
        const float2v f = i % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        r[i] = pack_bf16x2(f.x * scale, f.y * scale);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// Eight channels of one head of one token, of its keys or its values, per thread.
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadArgs a) {
    const int pieces = a.c.D / 8, per_token = 2 * a.c.heads * pieces;
    const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = u / per_token;
    if (t >= a.p.T) return;
    int i = (int)(u - t * per_token);
    const int which = i / (a.c.heads * pieces);
    i -= which * a.c.heads * pieces;
    const int h = i / pieces, d = i % pieces * 8;
    const Place at = place_of(a.c, a.p, (int)t, 0);
    uint4 w = {};
    if (at.used) {
        if (which == 0) {
            const int64_t from = key_at(a.c, at.page, h, at.slot) + d;
            if (a.c.e4m3)
                w = values_of(*reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.c.k) + from),
                              scale_value(a.c.scales[scale_at(a.c, at.page, h, 0, at.slot)]));
            else
                w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.c.k) + from);
        } else {
            const int64_t from = value_at(a.c, at.page, h, at.slot) + 8 * d;
            if (a.c.e4m3) {
                const uint8_t *const v = static_cast<const uint8_t *>(a.c.v) + from;
                uint2 c = {};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c.x |= (uint32_t)v[8 * j] << 8 * j;
                    c.y |= (uint32_t)v[8 * j + 32] << 8 * j;
                }
                w = values_of(c, scale_value(a.c.scales[scale_at(a.c, at.page, h, 1, at.slot)]));
            } else {
                const uint16_t *const v = static_cast<const uint16_t *>(a.c.v) + from;
                w = make_uint4(v[0] | (uint32_t)v[8] << 16, v[16] | (uint32_t)v[24] << 16, v[32] | (uint32_t)v[40] << 16,
                               v[48] | (uint32_t)v[56] << 16);
            }
        }
    }
    *reinterpret_cast<uint4 *>((which ? a.v : a.k) + (t * a.c.heads + h) * a.c.D + d) = w;
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_cache_append(const nvq_cache *cache, const int32_t *table, int B, int table_width,
                                const int32_t *sequences, const int32_t *positions, int T, const uint16_t *q,
                                int64_t q_stride, int H, uint16_t *q_out, const uint16_t *k, int64_t k_stride,
                                const uint16_t *v, int64_t v_stride, const float *cos_sin, int angles, int rot,
                                int interleaved, void *stream) {
    using namespace nvq;
    AppendArgs a;
    a.p = Places{table, sequences, positions, B, table_width, T};
    if (const int bad = check_cache(cache)) return bad;
    if (const int bad = check_places(a.p)) return bad;
    if (T * ((int64_t)H + 2 * cache->heads) > kMaxRows) return NVQ_ERR_SHAPE;
    if (!k || !v || (q != nullptr) != (H > 0) || (q != nullptr) != (q_out != nullptr) || (interleaved != 0 && interleaved != 1))
        return NVQ_ERR_INVALID_ARG;
    const int64_t D = cache->head_dim;
    if (H < 0 || H > NVQ_MAX_HEADS || (cos_sin && (angles < 1 || rot < 16 || rot % 16 || rot > D))) return NVQ_ERR_SHAPE;
    if (k_stride < cache->heads * D || v_stride < cache->heads * D || (q && q_stride < H * D)) return NVQ_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(cos_sin, 16) ||
        (q && q_stride % 8) || k_stride % 8 || v_stride % 8)
        return NVQ_ERR_ALIGN;
    if (q == q_out && q && q_stride != H * D) return NVQ_ERR_INVALID_ARG;
    a.c = view_of(*cache);
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out = q_out;
    a.cos_sin = cos_sin;
    a.H = H;
    a.angles = cos_sin ? angles : 0;
    a.rot = cos_sin ? rot : 0;
    a.interleaved = interleaved;
    const int lanes = (int)D / 16;
    const int L = lanes <= 2 ? 2 : lanes <= 4 ? 4 : lanes <= 8 ? 8 : 16;
    const int64_t rows = (int64_t)T * (H + 2 * cache->heads);
    const int64_t blocks = (rows * L + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)blocks), block(kThreads);
    const hipStream_t st = (hipStream_t)stream;
    if (L == 2)
        hipLaunchKernelGGL(cache_append_kernel<2>, grid, block, 0, st, a);
    else if (L == 4)
        hipLaunchKernelGGL(cache_append_kernel<4>, grid, block, 0, st, a);
    else if (L == 8)
        hipLaunchKernelGGL(cache_append_kernel<8>, grid, block, 0, st, a);
    else
        hipLaunchKernelGGL(cache_append_kernel<16>, grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

extern "C" int nvq_cache_read(const nvq_cache *cache, const int32_t *table, int B, int table_width,
                              const int32_t *sequences, const int32_t *positions, int T, uint16_t *k, uint16_t *v,
                              void *stream) {
    using namespace nvq;
    ReadArgs a;
    a.p = Places{table, sequences, positions, B, table_width, T};
    if (const int bad = check_cache(cache)) return bad;
    if (const int bad = check_places(a.p)) return bad;
    if (T * ((int64_t)2 * cache->heads) > kMaxRows) return NVQ_ERR_SHAPE;
    if (!k || !v) return NVQ_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16)) return NVQ_ERR_ALIGN;
    a.c = view_of(*cache);
    a.k = k;
    a.v = v;
    const int64_t threads = (int64_t)T * 2 * cache->heads * (cache->head_dim / 8);
    const int64_t blocks = (threads + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(cache_read_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
