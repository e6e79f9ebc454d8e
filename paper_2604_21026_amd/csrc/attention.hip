// nvq_attention: one new token per sequence over the paged cache.
//
// A wave takes steps of 32 tokens of one sequence and key head, for up to sixteen query heads at once, with one pass
// over keys and values: the running maximum m and sum l of a softmax, and the weighted sum of the values rescaled when
// m grows.  Both products run on the matrix cores, transposed, so that a query head is a lane's column throughout and
// nothing moves between lanes but the maxima:
//   S^T = K Q^T   two tiles of 16 tokens; row r of tile t is token 8 (r / 4) + 4 t + r % 4 of the step, so that the
//                 lane row kb = lane / 16 gets the scores of tokens 8 kb .. 8 kb + 7
//   O^T = V^T P^T the weights P as they come out of S^T: lane row kb multiplies tokens 8 kb .. 8 kb + 7, which is what
//                 one 16-byte piece of the value layout holds for a channel
// P enters as two bf16 values (p - bf16(p) is the second), 16 bits of it: the products are a twentieth of the time that
// the bytes take, so twice as many of them cost nothing, and results keep the precision of fp32 outputs.  The two
// products are summed apart and added at the end: what an infinite value makes of the second (zero times infinity,
// or the other sign) is left out there.
#include "cache.h"
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kStep = 32, kHeadTile = 16;

struct AttentionArgs {
    CacheView c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *table, *lengths;
    int B, H, width, group, tiles;  // query heads per key head; head tiles of them
    int window;
    float scale, softcap;
    void *out;
    int out_dtype;
    float *lse;
};

struct MaxOp {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// The tokens of a sequence that count, and its steps.
struct Span {
    int start, end, first, steps;  // tokens [start, end), steps first .. first + steps - 1
};
__device__ __forceinline__ Span span_of(const AttentionArgs &a, int b) {
    Span s;
    const int n = a.lengths[b], most = a.width << a.c.page_shift;
    s.end = n < 0 ? 0 : n > most ? most : n;
    s.start = a.window && s.end > a.window ? s.end - a.window : 0;
    s.first = s.start / kStep;
    s.steps = s.end > s.start ? (s.end + kStep - 1) / kStep - s.first : 0;
    return s;
}

// What a wave holds of one sequence and head tile: m and l per lane (l of the lane's own tokens), O^T in tiles of 16
// channels.
template <int D>
struct State {
    float m, l;
    float4v o[D / 16], rest[D / 16];  // of the weights' first and second values
    __device__ void clear() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = rest[i] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ float sum(int tile, int r) const {
        return __builtin_isfinite(o[tile][r]) ? o[tile][r] + rest[tile][r] : o[tile][r];
    }
};

// Pieces of eight values as they lie in the cache, and as an operand.
template <bool E4M3>
struct Piece;
template <>
struct Piece<false> {
    typedef uint4v raw;
    __device__ static raw load(const void *base, int64_t at) {
        return *as_global<uint4v>(static_cast<const uint16_t *>(base) + at);
    }
    __device__ static bf16x8 operand(raw r) { return __builtin_bit_cast(bf16x8, r); }
    // Zeros where the token of a value does not count (bit j: token j does).
    __device__ static raw only(raw r, uint32_t valid) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] &= (valid >> 2 * i & 1 ? 0xffffu : 0u) | (valid >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
        return r;
    }
};
template <>
struct Piece<true> {
    typedef uint2v raw;
    __device__ static raw load(const void *base, int64_t at) {
        return *as_global<uint2v>(static_cast<const uint8_t *>(base) + at);
    }
    __device__ static bf16x8 operand(raw r) {
        const uint32_t lo = r.x, hi = r.y;
        const uint4 w = make_uint4(
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true)));
        return __builtin_bit_cast(bf16x8, w);
    }
    __device__ static raw only(raw r, uint32_t valid) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t mask = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) mask |= valid >> (4 * i + j) & 1 ? 0xffu << 8 * j : 0u;
            r[i] &= mask;
        }
        return r;
    }
};

// Steps `step` .. `step + count - 1` (of the sequence's tokens from 0) into st.
template <int D, bool E4M3>
__device__ void attend(const AttentionArgs &a, int b, int head, int tile, const Span &sp, int step, int count, State<D> &st) {
    typedef Piece<E4M3> P;
    constexpr int C = D / 32, T = D / 16;
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int heads = a.group - kHeadTile * tile < kHeadTile ? a.group - kHeadTile * tile : kHeadTile;
    bf16x8 q[C];
    {
        const uint16_t *const at = a.q + b * a.q_stride + (int64_t)(head * a.group + kHeadTile * tile + (n < heads ? n : 0)) * D;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            uint4v w = *as_global<uint4v>(at + 32 * c + 8 * kb);
            if (n >= heads) w = uint4v{0, 0, 0, 0};
            q[c] = __builtin_bit_cast(bf16x8, w);
        }
    }
    const int32_t *const table = a.table + (int64_t)b * a.width;
    // A lane reads keys of the step's block n / 4 of eight tokens (its tile rows' own) and values of block kb.
    auto page_of = [&](int s, int block) {
        const int t = kStep * s + 8 * block;
        return t < sp.end ? table[t >> a.c.page_shift] : -1;
    };
    int key_page = page_of(step, n >> 2), value_page = page_of(step, kb);
    for (int i = 0; i < count; ++i) {
        const int s = step + i, t0 = kStep * s;
        const bool value_ok = (unsigned)value_page < (unsigned)a.c.pages;
        const int kp = (unsigned)key_page < (unsigned)a.c.pages ? key_page : 0, vp = value_ok ? value_page : 0;
        const int key_slot = (t0 + 8 * (n >> 2) + (n & 3)) & (a.c.page_size - 1);
        const int value_slot = (t0 + 8 * kb) & (a.c.page_size - 1);
        const int64_t ka = key_at(a.c, kp, head, key_slot) + 8 * kb, va = value_at(a.c, vp, head, value_slot) + 8 * n;
        typename P::raw k[2][C], v[T];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c) k[t][c] = P::load(a.c.k, ka + 4 * t * D + 32 * c);
#pragma unroll
        for (int d = 0; d < T; ++d) v[d] = P::load(a.c.v, va + 128 * d);
        uint2v key_scales = {}, value_scales = {};
        if (E4M3) {
            key_scales = *as_global<uint2v>(a.c.scales + scale_at(a.c, vp, head, 0, value_slot));
            value_scales = *as_global<uint2v>(a.c.scales + scale_at(a.c, vp, head, 1, value_slot));
        }
        key_page = page_of(s + 1, n >> 2);
        value_page = page_of(s + 1, kb);

        float4v raw[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            raw[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c)
                raw[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P::operand(k[t][c]), q[c], raw[t], 0, 0, 0);
        }
        wait_written(raw[0], raw[1]);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = raw[j >> 2][j & 3] * a.scale;
            if (E4M3) x[j] *= scale_value(key_scales[j >> 2] >> 8 * (j & 3) & 255);
        }
        if (a.softcap > 0.0f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = a.softcap * tanhf(x[j] / a.softcap);
        }
        // Which of the lane's tokens count; of steps in the middle of a sequence all do.
        uint32_t valid = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = t0 + 8 * kb + j;
            valid |= value_ok && t >= sp.start && t < sp.end ? 1u << j : 0u;
        }
        if (!__all(valid == 255u)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = valid >> j & 1 ? x[j] : -INFINITY;
#pragma unroll
            for (int d = 0; d < T; ++d) v[d] = P::only(v[d], valid);
        }
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        top = with_lane_xor<16>(top, MaxOp());
        top = with_lane_xor<32>(top, MaxOp());
        if (__any(top > st.m)) {
            const float m = fmaxf(st.m, top), f = st.m == m ? 1.0f : exp2f((st.m - m) * kLog2e);
            st.m = m;
            st.l *= f;
#pragma unroll
            for (int d = 0; d < T; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    st.o[d][r] *= f;
                    st.rest[d][r] *= f;
                }
        }
        const float ref = st.m == -INFINITY ? 0.0f : st.m;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float p[2], rest[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                p[e] = exp2f((x[j + e] - ref) * kLog2e);
                st.l += p[e];
                if (E4M3) {
                    const float f = scale_value(value_scales[(j + e) >> 2] >> 8 * ((j + e) & 3) & 255);
                    p[e] = valid >> (j + e) & 1 ? p[e] * f : 0.0f;
                }
            }
            hi[j / 2] = pack_bf16x2(p[0], p[1]);
            rest[0] = p[0] - __uint_as_float(hi[j / 2] << 16);
            rest[1] = p[1] - __uint_as_float(hi[j / 2] & 0xffff0000u);
            lo[j / 2] = pack_bf16x2(rest[0], rest[1]);
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
        for (int d = 0; d < T; ++d) {
            const bf16x8 w = P::operand(v[d]);
            st.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, ph, st.o[d], 0, 0, 0);
            st.rest[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, pl, st.rest[d], 0, 0, 0);
        }
#pragma unroll
        for (int d = 0; d < T; ++d) wait_written(st.o[d], st.rest[d]);
    }
}

// One wave per sequence and head tile.
template <int D, bool E4M3>
__global__ __launch_bounds__(64) void attention_kernel(AttentionArgs a) {
    const int per = a.c.heads * a.tiles;
    const int b = blockIdx.x / per, head = blockIdx.x % per / a.tiles, tile = blockIdx.x % a.tiles;
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int heads = a.group - kHeadTile * tile < kHeadTile ? a.group - kHeadTile * tile : kHeadTile;
    const Span sp = span_of(a, b);
    State<D> st;
    st.clear();
    attend<D, E4M3>(a, b, head, tile, sp, sp.first, sp.steps, st);
    float l = with_lane_xor<16>(st.l, AddOp());
    l = with_lane_xor<32>(l, AddOp());
    if (n >= heads) return;
    const int64_t row = (int64_t)b * a.H + head * a.group + kHeadTile * tile + n;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) store_global(a.out, a.out_dtype, row * D + 16 * d + 4 * kb + r, l == 0.0f ? 0.0f : st.sum(d, r) * f);
    if (a.lse && kb == 0) a.lse[row] = l == 0.0f ? -INFINITY : st.m + logf(l);
}

template <int D>
int launch_attention(const AttentionArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.B * a.c.heads * a.tiles)), block(64);
    if (a.c.e4m3)
        hipLaunchKernelGGL((attention_kernel<D, true>), grid, block, 0, st, a);
    else
        hipLaunchKernelGGL((attention_kernel<D, false>), grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}

// What the sizes alone say; H / heads query heads read each key head.
bool attention_shape(const nvq_cache *c, int B, int H) {
    return c && c->heads >= 1 && c->heads <= NVQ_MAX_HEADS && c->head_dim >= 32 && c->head_dim <= NVQ_MAX_HEAD_DIM &&
           c->head_dim % 32 == 0 && B >= 1 && B <= NVQ_ATTENTION_MAX_B && H >= 1 && H <= NVQ_MAX_HEADS && H % c->heads == 0;
}

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_attention_workspace_bytes(const nvq_cache *cache, int B, int H) {
    using namespace nvq;
    if (!attention_shape(cache, B, H)) return 0;
    return NVQ_ATTENTION_CLEAR_BYTES;
}

extern "C" int nvq_attention(const nvq_cache *cache, const uint16_t *q, int64_t q_stride, int H, const int32_t *table, int B,
                             int table_width, const int32_t *lengths, float scale, int window, float softcap, void *out,
                             int out_dtype, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace nvq;
    if (const int bad = check_cache(cache)) return bad;
    if (!q || !table || !lengths || !out || (out_dtype != NVQ_F32 && out_dtype != NVQ_BF16) || !(scale - scale == 0.0f) ||
        !(softcap >= 0.0f && softcap - softcap == 0.0f))
        return NVQ_ERR_INVALID_ARG;
    if (!attention_shape(cache, B, H) || table_width < 1 || (int64_t)table_width * cache->page_size > 1 << 30 || window < 0 ||
        q_stride < (int64_t)H * cache->head_dim)
        return NVQ_ERR_SHAPE;
    if (!aligned(q, 16) || q_stride % 8 || !aligned(table, 4) || !aligned(lengths, 4) ||
        !aligned(out, 16) || !aligned(lse, 4))
        return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_attention_workspace_bytes(cache, B, H))
        return NVQ_ERR_WORKSPACE;
    AttentionArgs a;
    a.c = view_of(*cache);
    a.q = q;
    a.q_stride = q_stride;
    a.table = table;
    a.lengths = lengths;
    a.B = B;
    a.H = H;
    a.width = table_width;
    a.group = H / cache->heads;
    a.tiles = (a.group + kHeadTile - 1) / kHeadTile;
    a.window = window;
    a.scale = scale;
    a.softcap = softcap;
    a.out = out;
    a.out_dtype = out_dtype;
    a.lse = lse;
    const hipStream_t st = (hipStream_t)stream;
    switch (cache->head_dim / 32) {
        case 1: return launch_attention<32>(a, st);
        case 2: return launch_attention<64>(a, st);
        case 3: return launch_attention<96>(a, st);
        case 4: return launch_attention<128>(a, st);
        case 5: return launch_attention<160>(a, st);
        case 6: return launch_attention<192>(a, st);
        case 7: return launch_attention<224>(a, st);
        default: return launch_attention<256>(a, st);
    }
}
