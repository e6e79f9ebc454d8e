// nvq_cache_append, nvq_cache_read: keys and values of new tokens into the paged cache, and out of it again.
//
// Bytes bound both, with prompts: every row is read and written once, 16 bytes at a time.  Keys (and queries) lie in the
// cache as they come.  Values lie eight tokens of a channel side by side, so eight tokens that follow each other in one
// such block are taken together, turned over in registers (8 channels by 8 tokens a thread) and stored as whole pieces;
// a token whose neighbours are elsewhere, as each one of a decode step, goes element by element.
//
// 4096 tokens of 32 + 8 heads of 128 into an 8-bit cache: 94 MB in 21 us, 4.5 TB/s (a copy of that size 4.8); read back 25 MB in
// 9.1.  One token: 3.7 and 2.2 us, a launch and two trips to memory (places, then rows).
#include <type_traits>

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
// Rows of a call (queries, keys, values).  A launch has fewer than 2^32 threads: a key and a value row read together take up to 32
// and 64 of them, written 16 (of four rows) and 64.
constexpr int64_t kMaxRows = 1 << 26;
static_assert(kMaxRows / 2 * (32 + 64) < 1ll << 32, "threads of a launch");

struct Place {
    int page, slot, position;
    bool used;
};

__device__ __forceinline__ Place place_at(const CacheView &c, const Places &p, int b, int position, int angles) {
    Place r;
    r.position = position;
    r.used = (unsigned)b < (unsigned)p.B && r.position >= 0 && r.position >> c.page_shift < p.width &&
             (angles == 0 || r.position < angles);
    r.page = r.used ? p.table[(int64_t)b * p.width + (r.position >> c.page_shift)] : -1;
    r.used = (unsigned)r.page < (unsigned)c.pages;
    r.slot = r.position & (c.page_size - 1);
    return r;
}
__device__ __forceinline__ Place place_of(const CacheView &c, const Places &p, int t, int angles) {
    return place_at(c, p, p.sequences ? p.sequences[t] : t, p.positions[t], angles);
}

struct AppendArgs {
    CacheView c;
    Places p;
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    uint16_t *q_out;
    const float *cos_sin;
    int H, angles, rot, interleaved;
    int row_blocks;  // workgroups of queries and keys
    int step;        // tokens of a workgroup's threads, one after the other: 8, or 1 of a few tokens
    bool once;       // queries and keys past the caches
};

struct MaxBits {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// The largest of L neighbouring lanes (a power of two).
template <int L>
__device__ __forceinline__ uint32_t most_of(uint32_t v) {
    if (L >= 64) v = with_lane_xor<32>(v, MaxBits());
    if (L >= 32) v = with_lane_xor<16>(v, MaxBits());
    if (L >= 16) v = with_lane_xor<8>(v, MaxBits());
    // (with_lane_xor<4> rotates by four among sixteen: right where lanes eight apart agree)
    if (L >= 16) v = with_lane_xor<4>(v, MaxBits());
    if (L == 8) v = MaxBits()(v, (uint32_t)__shfl_xor((int)v, 4));
    if (L >= 4) v = with_lane_xor<2>(v, MaxBits());
    if (L >= 2) v = with_lane_xor<1>(v, MaxBits());
    return v;
}

// Which of eight tokens from t0 on lie side by side in the cache's blocks of eight slots, by at least sixteen lanes for one
// t0: `position` and `sequence` of token t0 - 1 + (lane % 16), and bit j of `follows`: token t0 - 1 + j takes the slot behind
// its predecessor's, in the same block.  (All asked for at once: one after the other 4096 tokens took 36 us instead of 33.)
struct Neighbours {
    int position, sequence;
    uint32_t follows;
    __device__ Neighbours(const Places &p, int t0, int angles) {
        const int lane = threadIdx.x & 63, j = lane & 15, u = t0 - 1 + j;
        const bool in = u >= 0 && u < p.T;
        sequence = in ? (p.sequences ? p.sequences[u] : u) : -1;
        position = in ? p.positions[u] : -1;
        const int s = __shfl_up(sequence, 1), q = __shfl_up(position, 1);
        const bool f = j > 0 && in && sequence == s && position == q + 1 && (position & 7) && (angles == 0 || position < angles);
        follows = (uint32_t)(__ballot(f) >> (lane & 48)) & 0xffffu;
    }
    // Of token t0 - 1 + j, by every lane.
    __device__ int of(int v, int j) const { return __shfl(v, (int)(threadIdx.x & 48) | j); }
    // How many lie side by side from token t0 - 1 + j on; 0 if it is not the first of them.
    __device__ int run(int j) const { return follows >> j & 1 ? 0 : __builtin_ctz(~(follows >> (j + 1))) + 1; }
};

// The scale byte of a row whose largest magnitude has these bf16 bits: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f80u) return 255;
    const int b = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u);
    return b < 1 ? 1 : (uint32_t)b;
}

// Eight values -> codes under that scale byte (255: zeros).
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], uint32_t byte) {
    if (byte == 255) return make_uint2(0, 0);
    const float up = __uint_as_float((254u - byte) << 23);  // (byte 1 to 247: a normal number)
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

// A thread's channels of the values, E of them side by side (in 2 E bytes of bf16).
template <int E>
struct Channels;
template <>
struct Channels<2> {
    typedef uint32_t word;
    __device__ static uint32_t pair(const word &w, int p) { return w; }
    __device__ static word from(const uint32_t (&p)[1]) { return p[0]; }
};
template <>
struct Channels<4> {
    typedef uint2 word;
    __device__ static uint32_t pair(const word &w, int p) { return p ? w.y : w.x; }
    __device__ static word from(const uint32_t (&p)[2]) { return make_uint2(p[0], p[1]); }
};
// 16-bit value i (0: the low one) of a pair of each of two words, side by side.
__device__ __forceinline__ uint32_t both(uint32_t a, uint32_t b, int i) {
    return __builtin_amdgcn_perm(b, a, i ? 0x07060302u : 0x05040100u);
}

constexpr int kRowsEach = 4;

// 16 bytes of a row; ONCE: past the caches, for calls whose rows are more than these keep anyway (once_of).
template <bool ONCE>
__device__ __forceinline__ uint4 load_row(const uint16_t *p) {
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
    if constexpr (!ONCE) return *reinterpret_cast<const uint4 *>(p);
    const vec v = __builtin_nontemporal_load(reinterpret_cast<const vec *>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
}
template <typename T>
__device__ __forceinline__ void store_row(uint16_t *p, const T &w, bool once) {
    typedef uint32_t vec __attribute__((ext_vector_type(sizeof(T) / 4)));
    if (once) {
        asm volatile("" ::: "memory");  // (around it, or the two stores become one plain one)
        __builtin_nontemporal_store(__builtin_bit_cast(vec, w), reinterpret_cast<vec *>(p));
        asm volatile("" ::: "memory");
    } else {
        *reinterpret_cast<T *>(p) = w;
    }
}

// The values of `a.step` tokens from t0 on, E channels of head h per thread, L threads to a head: what lies side by side
// is read row by row, turned over and stored as whole pieces of eight tokens.
template <int E, int L>
__device__ void append_values(const AppendArgs &a, int unit_block) {
    typedef typename Channels<E>::word word;
    const int64_t unit = ((int64_t)unit_block * kThreads + threadIdx.x) / L;
    const int i = threadIdx.x % L, D = a.c.D;
    const int64_t g = unit / a.c.heads;
    const int h = (int)(unit - g * a.c.heads);
    const int t0 = g * a.step < a.p.T ? (int)g * a.step : a.p.T;
    const Neighbours near(a.p, t0, a.angles);
    for (int j = 1; j <= a.step; ++j) {
        const int t = t0 - 1 + j, n = near.run(j);
        const int sequence = near.of(near.sequence, j), position = near.of(near.position, j);
        const bool mine = t < a.p.T && n > 0 && i * E < D;
        if (!__any(mine)) continue;
        const uint16_t *const from = a.v + (int64_t)t * a.v_stride + h * D + E * i;
        word row[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            row[k] = word{};
            if (mine && k < n) row[k] = *reinterpret_cast<const word *>(from + k * a.v_stride);
        }
        const Place at = place_at(a.c, a.p, sequence, position, a.angles);
        const bool on = mine && at.used;
        const int64_t to = value_at(a.c, at.page, h, at.slot) + 8 * E * i;
        if (a.c.e4m3) {
            uint32_t code[8];  // E bytes each
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                uint32_t top = 0;
#pragma unroll
                for (int p = 0; p < E / 2; ++p) {
                    const uint32_t w = Channels<E>::pair(row[k], p), lo = w & 0x7fffu, hi = w >> 16 & 0x7fffu;
                    top = top > lo ? top : lo;
                    top = top > hi ? top : hi;
                }
                const uint32_t byte = scale_byte(most_of<L>(top));
                const float up = __uint_as_float((byte == 255 ? 0u : 254u - byte) << 23);
                int c = 0;
                if (byte != 255) {
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const uint32_t w = Channels<E>::pair(row[k], p);
                        const float x = __uint_as_float(w << 16) * up, y = __uint_as_float(w & 0xffff0000u) * up;
                        c = p ? __builtin_amdgcn_cvt_pk_fp8_f32(x, y, c, true) : __builtin_amdgcn_cvt_pk_fp8_f32(x, y, c, false);
                    }
                }
                code[k] = (uint32_t)c;
                if (on && i == 0 && k < n) a.c.scales[scale_at(a.c, at.page, h, 1, at.slot + k)] = (uint8_t)byte;
            }
            if (!on) continue;
            uint8_t *const out = static_cast<uint8_t *>(a.c.v) + to;
            if (n == 8) {
                uint32_t w[2 * E];  // channel by channel
#pragma unroll
                for (int c = 0; c < E; ++c)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t pick = 0x0c0c0000u | (uint32_t)(4 + c) << 8 | (uint32_t)c;  // byte c of both
                        w[2 * c + q] = __builtin_amdgcn_perm(code[4 * q + 1], code[4 * q], pick) |
                                       __builtin_amdgcn_perm(code[4 * q + 3], code[4 * q + 2], pick) << 16;
                    }
#pragma unroll
                for (int q = 0; q < 2 * E; q += 4) *reinterpret_cast<uint4 *>(out + 4 * q) = make_uint4(w[q], w[q + 1], w[q + 2], w[q + 3]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int c = 0; c < E; ++c)
                        if (k < n) out[8 * c + k] = (uint8_t)(code[k] >> 8 * c);
            }
        } else if (on) {
            uint16_t *const out = static_cast<uint16_t *>(a.c.v) + to;
            if (n == 8) {
#pragma unroll
                for (int c = 0; c < E; ++c) {
                    uint32_t w[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = both(Channels<E>::pair(row[2 * q], c / 2), Channels<E>::pair(row[2 * q + 1], c / 2), c & 1);
                    *reinterpret_cast<uint4 *>(out + 8 * c) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int c = 0; c < E; ++c)
                        if (k < n) out[8 * c + k] = (uint16_t)(Channels<E>::pair(row[k], c / 2) >> 16 * (c & 1));
            }
        }
    }
}

// The first blocks: queries and keys, sixteen channels of kRowsEach heads of one token per thread, that it turns by the
// same angles, L threads to a head: two pieces of eight channels, which are each other's partners of the rotation, or hold
// whole pairs.  The others: values.
template <int L>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(AppendArgs a) {
    const int D = a.c.D;
    if ((int)blockIdx.x >= a.row_blocks) {
        append_values<L == 16 ? 4 : 2, L == 16 ? 64 : 8 * L>(a, (int)blockIdx.x - a.row_blocks);
        return;
    }
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / L;
    const int i = threadIdx.x % L, all = a.H + a.c.heads, groups = (all + kRowsEach - 1) / kRowsEach;
    const int64_t t64 = unit / groups;
    const int t = t64 < a.p.T ? (int)t64 : 0, h0 = (int)(unit - t64 * groups) * kRowsEach;
    const Place at = place_of(a.c, a.p, t, a.angles);
    const bool in = t64 < a.p.T && i < D / 16, on = in && at.used;
    const bool turn = i < a.rot / 16, halves = turn && !a.interleaved;
    const int o0 = halves ? 8 * i : !a.interleaved ? a.rot + 16 * (i - a.rot / 16) : 16 * i;
    const int o1 = halves ? o0 + a.rot / 2 : o0 + 8;
    uint4 w[kRowsEach][2];
    float c[8], s[8];
    auto read_rows = [&](auto once) {
#pragma unroll
        for (int r = 0; r < kRowsEach; ++r) {
            w[r][0] = w[r][1] = make_uint4(0, 0, 0, 0);
            const int h = h0 + r;
            if (!in || h >= all) continue;  // (rows are read before it is known whether they have a place)
            const uint16_t *const row = h < a.H ? a.q + t * a.q_stride + h * D : a.k + t * a.k_stride + (h - a.H) * D;
            w[r][0] = load_row<decltype(once)::value>(row + o0);
            w[r][1] = load_row<decltype(once)::value>(row + o1);
        }
    };
    if (a.once)
        read_rows(std::true_type());
    else
        read_rows(std::false_type());
    if (on && turn) {
        const float *const cs = a.cos_sin + (int64_t)at.position * a.rot + 8 * i;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = cs[j];
            s[j] = cs[a.rot / 2 + j];
        }
    }
#pragma unroll
    for (int r = 0; r < kRowsEach; ++r) {
        const int h = h0 + r;
        if (on && turn) {
            float x0[8], x1[8];
            unpack(w[r][0], x0);
            unpack(w[r][1], x1);
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
            w[r][0] = pack(x0);
            w[r][1] = pack(x1);
        }
        if (on && h < a.H) {
            uint16_t *const out = a.q_out + ((int64_t)t * a.H + h) * D;
            store_row(out + o0, w[r][0], a.once);
            store_row(out + o1, w[r][1], a.once);
        }
        const bool key = on && h >= a.H && h < all;
        if (!__any(key)) continue;
        const int64_t to = key_at(a.c, at.page, h - a.H, at.slot);
        if (a.c.e4m3) {
            const uint32_t m0 = top_bits(w[r][0]), m1 = top_bits(w[r][1]);
            const uint32_t byte = scale_byte(most_of<L>(m0 > m1 ? m0 : m1));
            float x0[8], x1[8];
            unpack(w[r][0], x0);
            unpack(w[r][1], x1);
            const uint2 c0 = codes_of(x0, byte), c1 = codes_of(x1, byte);
            if (!key) continue;
            if (i == 0) a.c.scales[scale_at(a.c, at.page, h - a.H, 0, at.slot)] = (uint8_t)byte;
            uint8_t *const out = static_cast<uint8_t *>(a.c.k) + to;
            *reinterpret_cast<uint2 *>(out + o0) = c0;
            *reinterpret_cast<uint2 *>(out + o1) = c1;
        } else if (key) {
            uint16_t *const out = static_cast<uint16_t *>(a.c.k) + to;
            *reinterpret_cast<uint4 *>(out + o0) = w[r][0];
            *reinterpret_cast<uint4 *>(out + o1) = w[r][1];
        }
    }
}

struct ReadArgs {
    CacheView c;
    Places p;
    uint16_t *k, *v;
    int row_blocks;  // workgroups of keys
    int step;        // as in AppendArgs
    bool once;       // results past the caches
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

// The values of `a.step` tokens, as append_values has them.
template <int E, int L>
__device__ void read_values(const ReadArgs &a, int unit_block) {
    typedef typename Channels<E>::word word;
    const int64_t unit = ((int64_t)unit_block * kThreads + threadIdx.x) / L;
    const int i = threadIdx.x % L, D = a.c.D;
    const int64_t g = unit / a.c.heads;
    const int h = (int)(unit - g * a.c.heads);
    const int t0 = g * a.step < a.p.T ? (int)g * a.step : a.p.T;
    const Neighbours near(a.p, t0, 0);
    for (int j = 1; j <= a.step; ++j) {
        const int t = t0 - 1 + j, n = near.run(j);
        const Place at = place_at(a.c, a.p, near.of(near.sequence, j), near.of(near.position, j), 0);
        if (t >= a.p.T || n == 0 || i * E >= D) continue;
        uint16_t *const out = a.v + ((int64_t)t * a.c.heads + h) * D + E * i;
        const int first = at.slot & 7;
        word row[8];
        if (!at.used) {
#pragma unroll
            for (int k = 0; k < 8; ++k) row[k] = word{};
        } else {
            const int64_t from = value_at(a.c, at.page, h, at.slot - first) + 8 * E * i;
            if (a.c.e4m3) {
                uint2 piece[E];
                const uint8_t *const v = static_cast<const uint8_t *>(a.c.v) + from;
#pragma unroll
                for (int c = 0; c < E; ++c) piece[c] = *reinterpret_cast<const uint2 *>(v + 8 * c);
                const uint2 scales = *reinterpret_cast<const uint2 *>(a.c.scales + scale_at(a.c, at.page, h, 1, at.slot - first));
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float scale = scale_value((k < 4 ? scales.x : scales.y) >> 8 * (k & 3) & 255);
                    uint32_t pairs[E / 2];
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const uint2 &l = piece[2 * p], &r = piece[2 * p + 1];
                        const uint32_t two = __builtin_amdgcn_perm(k < 4 ? r.x : r.y, k < 4 ? l.x : l.y,
                                                                   0x0c0c0000u | (uint32_t)(4 + (k & 3)) << 8 | (uint32_t)(k & 3));
                        const float2v f = __builtin_amdgcn_cvt_pk_f32_fp8((int)two, false);
                        pairs[p] = pack_bf16x2(f.x * scale, f.y * scale);
                    }
                    row[k] = Channels<E>::from(pairs);
                }
            } else {
                uint4 piece[E];
                const uint16_t *const v = static_cast<const uint16_t *>(a.c.v) + from;
#pragma unroll
                for (int c = 0; c < E; ++c) piece[c] = *reinterpret_cast<const uint4 *>(v + 8 * c);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t pairs[E / 2];
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const uint32_t l[4] = {piece[2 * p].x, piece[2 * p].y, piece[2 * p].z, piece[2 * p].w};
                        const uint32_t r[4] = {piece[2 * p + 1].x, piece[2 * p + 1].y, piece[2 * p + 1].z, piece[2 * p + 1].w};
                        pairs[p] = both(l[k / 2], r[k / 2], k & 1);
                    }
                    row[k] = Channels<E>::from(pairs);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k >= first && k < first + n) store_row(out + (int64_t)(k - first) * a.c.heads * D, row[k], a.once);
    }
}

// The first blocks: eight channels of one token's and head's keys per thread, 2 L threads to a head.  The others: values.
template <int L>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadArgs a) {
    if ((int)blockIdx.x >= a.row_blocks) {
        read_values<L == 16 ? 4 : 2, L == 16 ? 64 : 8 * L>(a, (int)blockIdx.x - a.row_blocks);
        return;
    }
    const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / (2 * L);
    const int64_t t = unit / a.c.heads;
    const int i = threadIdx.x % (2 * L), h = (int)(unit - t * a.c.heads), D = a.c.D;
    if (t >= a.p.T || i >= D / 8) return;
    const Place at = place_of(a.c, a.p, (int)t, 0);
    uint4 w = {};
    if (at.used) {
        const int64_t from = key_at(a.c, at.page, h, at.slot) + 8 * i;
        if (a.c.e4m3)
            w = values_of(*reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.c.k) + from),
                          scale_value(a.c.scales[scale_at(a.c, at.page, h, 0, at.slot)]));
        else
            w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.c.k) + from);
    }
    store_row(a.k + (t * a.c.heads + h) * D + 8 * i, w, a.once);
}

// Threads to a head: L of sixteen channels of keys; and of the values 8 L of two, or 64 of four.
int key_lanes(int D) { return D <= 32 ? 2 : D <= 64 ? 4 : D <= 128 ? 8 : 16; }
int value_lanes(int D) { return D <= 128 ? 8 * key_lanes(D) : 64; }
// Tokens that the threads of a head of values take in turn: eight in prompts, of which few do not follow each other; one
// where each may be elsewhere or few are there.  (Eight heads of 128 appended and read back, one and eight: a prompt of 256
// tokens 4.0 + 3.0 and 3.7 + 3.7 us, of 512 5.1 + 3.7 and 4.4 + 3.9, of 1024 8.3 + 5.4 and 6.3 + 4.3, in 8 bits 11.4 + 6.3 and 7.3 +
// 4.5; 512 tokens of as many sequences 6.8 + 3.3 and 9.5 + 7.2.)
int step_of(const Places &p) { return p.sequences && p.T >= 512 ? 8 : 1; }
// Rows past the caches from 8 MiB on, twice a cache's size.  Queries and keys of 40 heads of 128, past the caches and through them: 1024
// tokens 8.6 and 9.6 us, 2048 13.7 and 14.0, 4096 21.4 and 22.8, 8192 37.9 and 44.5; read back, 2048 5.4 and 6.0, 4096 8.5 and 9.9, 8192 13.9
// and 15.0.  With a kernel behind that reads all results: 13.4 and 13.5, 21.1 and 19.7, 33.3 and 36.6, 65.7 and 66.3; 12.4 and 12.6, 17.7
// and 17.7, 28.4 and 27.1.
bool once_of(int64_t values) { return 2 * values >= 8 << 20; }
int64_t value_blocks(const Places &p, int heads, int D) {
    const int step = step_of(p);
    return ((int64_t)((p.T + step - 1) / step) * heads * value_lanes(D) + kThreads - 1) / kThreads;
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
    const int L = key_lanes((int)D);
    const int64_t rows = (int64_t)T * ((H + cache->heads + kRowsEach - 1) / kRowsEach);
    a.row_blocks = (int)((rows * L + kThreads - 1) / kThreads);
    a.step = step_of(a.p);
    a.once = once_of(T * ((int64_t)H + cache->heads) * D);
    const dim3 grid((unsigned)(a.row_blocks + value_blocks(a.p, cache->heads, (int)D))), block(kThreads);
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
    const int L = key_lanes(cache->head_dim);
    a.row_blocks = (int)(((int64_t)T * cache->heads * 2 * L + kThreads - 1) / kThreads);
    a.step = step_of(a.p);
    a.once = once_of((int64_t)T * 2 * cache->heads * cache->head_dim);
    const dim3 grid((unsigned)(a.row_blocks + value_blocks(a.p, cache->heads, cache->head_dim))), block(kThreads);
    const hipStream_t st = (hipStream_t)stream;
    if (L == 2)
        hipLaunchKernelGGL(cache_read_kernel<2>, grid, block, 0, st, a);
    else if (L == 4)
        hipLaunchKernelGGL(cache_read_kernel<4>, grid, block, 0, st, a);
    else if (L == 8)
        hipLaunchKernelGGL(cache_read_kernel<8>, grid, block, 0, st, a);
    else
        hipLaunchKernelGGL(cache_read_kernel<16>, grid, block, 0, st, a);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
