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
// P enters as three bf16 values whose sum it is, all 24 bits.  (With two, 2^-18 of a weight left out, large values that cancel show
// it, also in results of bf16; 32 ragged sequences in 8 bits 59.6 us instead of 60.3, 131072 tokens the same.)  The products with
// the first and with the rest are summed apart and added at the end: what an infinite value makes of the rest (zero times
// infinity, or the other sign) is left out there.
//
// The bytes of keys and values bound it: one sequence of 131072 tokens, 8 key heads of 128 in bf16, 537 MB, takes 90 us,
// 6.0 TB/s, where a plain reading of as much takes 83; 32 ragged ones of up to 16384 tokens in 8 bits, 261 MB, 60.3 us,
// 47 of them reading.  Short ones are bound by the memory's latency, four times over (lengths, pages, keys and values,
// joins): 500 tokens 8.9 us, 7 sequences of up to 3000 behind a window of 1000 11.4 us.
#include <type_traits>

#include "cache.h"
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kStep = 32, kHeadTile = 16;
constexpr int kMaxGroups = 256;
// Steps that a sequence and head tile counts for beyond its own: its numbers, first loads and last sums take a wave about
// as long, and workgroups of many short ones would end last.  (0, 1, 2, 3: 68, 64.5, 63, 62 us for 32 ragged sequences of
// up to 16384 tokens in 8 bits, 24, 22.4, 21.7, 21.5 for 40 of 150 to 300.)
constexpr int kPieceCost = 2;

struct AttentionArgs {
    CacheView c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *table, *lengths;
    int B, H, width, group, tiles;  // query heads per key head; head tiles of them
    int window;
    int most_each;  // workgroups that there are for each sequence and head tile
    float scale, softcap;
    void *out;
    int out_dtype;
    float *lse;
    uint32_t *arrived;  // workspace, per workgroup
    float *partial;     // [workgroup][2][16][D + 2]
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
template <int D, bool E4M3>
struct State {
    static constexpr bool kApart = !E4M3;  // (the 8-bit format has no infinities)
    float m, l;
    float4v o[D / 16], rest[kApart ? D / 16 : 1];  // of the weights' first values and of the rest
    __device__ void clear() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            o[i] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            if (kApart) rest[i] = o[i];
        }
    }
    // Where the products with the rest of the weights are summed.
    __device__ float4v &small(int i) { return kApart ? rest[kApart ? i : 0] : o[i]; }
    __device__ float sum(int tile, int r) const {
        return kApart && __builtin_isfinite(o[tile][r]) ? o[tile][r] + rest[kApart ? tile : 0][r] : o[tile][r];
    }
};

// Pieces of eight values as they lie in the cache, and as an operand.  load_once: for what one load takes whole lines of (the
// values: 131072 tokens 98.1 -> 90.9 us, 30 sequences of 2000 47.8 -> 45.1; keys, of whose lines a load takes a half or a quarter,
// would come twice, 61 -> 72 us in 8 bits).  It costs where a cache may hold the values, 16000 tokens 20.0 -> 21.1, and where groups
// of more than sixteen query heads read them once for each tile: of 32, 16000 tokens of 4 key heads 25.0 -> 26.1, 131072 of 8 115.7 -> 123.3,
// 8 sequences of 8000 49.1 -> 50.2, but 40 of 4000 58.7 -> 57.7.
template <bool E4M3>
struct Piece;
template <>
struct Piece<false> {
    typedef uint4v raw;
    __device__ static raw load(const void *base, int64_t at) {
        return *as_global<uint4v>(static_cast<const uint16_t *>(base) + at);
    }
    __device__ static raw load_once(const void *base, int64_t at) {
        return __builtin_nontemporal_load(as_global<uint4v>(static_cast<const uint16_t *>(base) + at));
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
    __device__ static raw load_once(const void *base, int64_t at) {
        return __builtin_nontemporal_load(as_global<uint2v>(static_cast<const uint8_t *>(base) + at));
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

// Loads stay on their side of this.  (The compiler moved the values' up to the keys', into registers of their own that it
// waited for and copied at the loop's end.)
__device__ __forceinline__ void keep_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Keys and values of a step on their way to a wave.
template <int D, bool E4M3>
struct Fetch {
    typename Piece<E4M3>::raw k[2][D / 32], v[D / 16];
    uint2v key_scales, value_scales;
    bool value_ok;  // the lane's block of eight tokens has a page
};

// Steps `step` .. `step + count - 1` (of the sequence's tokens from 0; at least one) into st.  Keys of the next step are
// asked for as soon as the products have taken this step's, values likewise, and pages a step before that.
template <int D, bool E4M3>
__device__ __forceinline__ void attend(const AttentionArgs &a, int b, int head, int tile, const Span &sp, int step, int count,
                                       State<D, E4M3> &st) {
    typedef Piece<E4M3> P;
    constexpr int C = D / 32, T = D / 16;
    const int lane = threadIdx.x & 63, n = lane & 15, kb = lane >> 4;
    const int heads = a.group - kHeadTile * tile < kHeadTile ? a.group - kHeadTile * tile : kHeadTile;
    const int32_t *const table = a.table + (int64_t)b * a.width;
    // A lane reads keys of the step's block n / 4 of eight tokens (its tile rows' own) and values of block kb.  No load
    // stands behind a branch: where one does, the compiler waits for all of them at the loop's end, and a step takes the
    // memory's latency (103 instead of 101 us at 131072 tokens).  So a number is looked up for every block, past the last one the
    // last one's, and what it is worth is decided where it is used; past the last step the last one is read again.
    auto page_of = [&](int s, int block) {
        const int t = kStep * s + 8 * block;
        return *as_global<int32_t>(table + ((t < sp.end ? t : sp.end - 1) >> a.c.page_shift));
    };
    auto there = [&](int s, int block, int page) { return kStep * s + 8 * block < sp.end && (unsigned)page < (unsigned)a.c.pages; };
    auto load_keys = [&](Fetch<D, E4M3> &f, int s, int page, int page_kb) {
        const int slot = (kStep * s + 8 * (n >> 2) + (n & 3)) & (a.c.page_size - 1);
        const int64_t at = key_at(a.c, there(s, n >> 2, page) ? page : 0, head, slot) + 8 * kb;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < C; ++c) f.k[t][c] = P::load(a.c.k, at + 4 * t * D + 32 * c);
        if (E4M3)
            f.key_scales = *as_global<uint2v>(
                a.c.scales + scale_at(a.c, there(s, kb, page_kb) ? page_kb : 0, head, 0, (kStep * s + 8 * kb) & (a.c.page_size - 1)));
    };
    auto load_values = [&](Fetch<D, E4M3> &f, int s, int page) {
        const int slot = (kStep * s + 8 * kb) & (a.c.page_size - 1);
        f.value_ok = there(s, kb, page);
        const int64_t at = value_at(a.c, f.value_ok ? page : 0, head, slot) + 8 * n;
#pragma unroll
        for (int d = 0; d < T; ++d) f.v[d] = P::load_once(a.c.v, at + 128 * d);
        if (E4M3) f.value_scales = *as_global<uint2v>(a.c.scales + scale_at(a.c, f.value_ok ? page : 0, head, 1, slot));
    };
    const int key_page = page_of(step, n >> 2), first_value_page = page_of(step, kb);
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
    // (in the order of the loop, whose waits count what is under way)
    Fetch<D, E4M3> fetch;
    keep_order();
    load_keys(fetch, step, key_page, first_value_page);
    keep_order();
    int next_key_page = page_of(count > 1 ? step + 1 : step, n >> 2), next_value_page = page_of(count > 1 ? step + 1 : step, kb);
    keep_order();
    load_values(fetch, step, first_value_page);
    keep_order();
    for (int i = 0; i < count; ++i) {
        Fetch<D, E4M3> &f = fetch;
        const int s = step + i, t0 = kStep * s, next = i + 1 < count ? s + 1 : s;
        const bool value_ok = f.value_ok;
        float4v raw[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            raw[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c)
                raw[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P::operand(f.k[t][c]), q[c], raw[t], 0, 0, 0);
        }
        wait_written(raw[0], raw[1]);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = raw[j >> 2][j & 3] * a.scale;
            if (E4M3) x[j] *= scale_value(f.key_scales[j >> 2] >> 8 * (j & 3) & 255);
        }
        keep_order();
        load_keys(f, next, next_key_page, next_value_page);
        const int value_page = next_value_page;
        next_key_page = page_of(i + 2 < count ? s + 2 : step + count - 1, n >> 2);
        next_value_page = page_of(i + 2 < count ? s + 2 : step + count - 1, kb);
        keep_order();
        if (a.softcap > 0.0f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = a.softcap * tanhf(x[j] / a.softcap);
        }
        // Which of the lane's tokens count; of steps in the middle of a sequence all do.
        uint32_t valid = 255u;
        if (t0 < sp.start || t0 + kStep > sp.end || !__all(value_ok)) {
            valid = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = t0 + 8 * kb + j;
                valid |= value_ok && t >= sp.start && t < sp.end ? 1u << j : 0u;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = valid >> j & 1 ? x[j] : -INFINITY;
#pragma unroll
            for (int d = 0; d < T; ++d) f.v[d] = P::only(f.v[d], valid);
        }
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        top = with_lane_xor<16>(top, MaxOp());
        top = with_lane_xor<32>(top, MaxOp());
        if (__any(top > st.m)) {
            const float m = fmaxf(st.m, top), c = st.m == m ? 1.0f : __builtin_amdgcn_exp2f((st.m - m) * kLog2e);
            st.m = m;
            st.l *= c;
#pragma unroll
            for (int d = 0; d < T; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    st.o[d][r] *= c;
                    if (State<D, E4M3>::kApart) st.small(d)[r] *= c;
                }
        }
        const float ref = st.m == -INFINITY ? 0.0f : st.m;
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = __builtin_amdgcn_exp2f((x[j] - ref) * kLog2e);
            st.l += p[j];
            if (E4M3) {
                const float c = scale_value(f.value_scales[j >> 2] >> 8 * (j & 3) & 255);
                p[j] = valid >> j & 1 ? p[j] * c : 0.0f;
            }
        }
        auto part = [&]() {  // the next eight bits of the weights
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
                p[2 * j] -= __uint_as_float(w[j] << 16);
                p[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
            }
            return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        };
        const bf16x8 w0 = part(), w1 = part(), w2 = part();
#pragma unroll
        for (int d = 0; d < T; ++d) {
            const bf16x8 y = P::operand(f.v[d]);
            st.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, w0, st.o[d], 0, 0, 0);
            st.small(d) = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, w1, st.small(d), 0, 0, 0);
            st.small(d) = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, w2, st.small(d), 0, 0, 0);
        }
#pragma unroll
        for (int d = 0; d < T; ++d) wait_written(st.o[d], st.small(d));
        keep_order();
        load_values(f, next, value_page);
        keep_order();
    }
}

// A piece: steps [begin, end) of the n steps of one sequence and head tile (ht: key head times tiles, tile).
struct PieceOf {
    int b, ht, begin, end, n;
};

// The grid is one flat line of all steps of all sequences and head tiles, cut into as many equal ranges as there are
// workgroups (or, of few short ones, dealt out by sequence and head tile), and a range into one per wave: however ragged
// the lengths, every compute unit reads as much.  What a
// wave has of a sequence and head tile that others share goes to LDS and is joined there, what a workgroup has of one
// to the workspace, where the workgroup that arrives last joins it.
template <int D>
constexpr int waves_of() { return D <= 128 ? 8 : 4; }

// a / b for 0 <= a < 2^49, 0 < b < 2^41 and quotients whose product with b is below 2^49: in fp64 (a quotient that is no
// whole number is further from one than its rounding), which takes a tenth of an integer division of 64 bits.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) { return (int64_t)((double)a / (double)b); }

__device__ __forceinline__ float factor(float m, float most) {
    return m == most ? 1.0f : __builtin_amdgcn_exp2f((m - most) * kLog2e);
}
__device__ __forceinline__ float wave_max(float v) {
    v = with_lane_xor<32>(v, MaxOp());
    v = with_lane_xor<16>(v, MaxOp());
    v = with_lane_xor<8>(v, MaxOp());
    v = with_lane_xor<4>(v, MaxOp());
    v = with_lane_xor<2>(v, MaxOp());
    return with_lane_xor<1>(v, MaxOp());
}

struct MostOp {
    __device__ int operator()(int a, int b) const { return a > b ? a : b; }
};
__device__ __forceinline__ int wave_most(int v) {
    v = with_lane_xor<32>(v, MostOp());
    v = with_lane_xor<16>(v, MostOp());
    v = with_lane_xor<8>(v, MostOp());
    v = with_lane_xor<4>(v, MostOp());
    v = with_lane_xor<2>(v, MostOp());
    return with_lane_xor<1>(v, MostOp());
}

__device__ __forceinline__ void put(float *p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <int D, bool E4M3>
__global__ __launch_bounds__(64 * waves_of<D>()) void attention_kernel(AttentionArgs a) {
    constexpr int kWaves = waves_of<D>(), kThreads = 64 * kWaves, kRow = D + 2;  // (a head's sum, m, l)
    extern __shared__ __align__(16) char lds[];
    __shared__ int scan[kWaves], longest_of[kWaves];
    __shared__ PieceOf held[kWaves][2];
    __shared__ int last[2];
    int *const upto = reinterpret_cast<int *>(lds);  // [B + 1]: steps before a sequence, of one head tile, kPieceCost included
    float *const parts = reinterpret_cast<float *>(lds + (((int64_t)a.B + 1) * 4 + 15) / 16 * 16);  // [waves][2][heads][kRow]
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    const int per = a.c.heads * a.tiles;                                   // head tiles
    const int heads_most = a.group < kHeadTile ? a.group : kHeadTile;
    auto key_head_of = [&](int ht) { return a.tiles == 1 ? ht : ht / a.tiles; };  // (mostly without a division)
    auto tile_of = [&](int ht) { return a.tiles == 1 ? 0 : ht % a.tiles; };
    auto heads_of = [&](int ht) {
        const int h = a.group - kHeadTile * tile_of(ht);
        return h < kHeadTile ? h : kHeadTile;
    };
    auto row_of = [&](int b, int ht) { return (int64_t)b * a.H + key_head_of(ht) * a.group + kHeadTile * tile_of(ht); };

    int total = 0, longest = 0;
    if (a.B <= 64) {  // every wave all of them, without waiting for the others
        const int steps = lane < a.B ? span_of(a, lane).steps : 0, sum = scan_wave(steps > 0 ? steps + kPieceCost : 0);
        longest = wave_most(steps);
        total = of_lane(sum, 63);
        if (lane < a.B) upto[lane + 1] = sum;  // (the same by all)
    }
    for (int b0 = 0; a.B > 64 && b0 < a.B; b0 += kThreads) {
        const int b = b0 + (int)threadIdx.x;
        const int steps = b < a.B ? span_of(a, b).steps : 0;
        const int sum = scan_wave(steps > 0 ? steps + kPieceCost : 0);
        longest = steps > longest ? steps : longest;
        __syncthreads();
        if (lane == 63) scan[w] = sum;
        const int most = wave_most(longest);
        if (lane == 0) longest_of[w] = most;
        __syncthreads();
        int before = total, all = total;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            before += i < w ? scan[i] : 0;
            all += scan[i];
            longest = longest_of[i] > longest ? longest_of[i] : longest;
        }
        if (b < a.B) upto[b + 1] = before + sum;
        total = all;
    }
    if (lane == 0) upto[0] = 0;
    if (lane < 2) held[w][lane].b = -1;
    if (a.B > 64) __syncthreads();
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
        if (upto[b + 1] == upto[b]) {  // nothing to attend to
            for (int i = threadIdx.x; i < a.H * D; i += kThreads) store_global(a.out, a.out_dtype, (int64_t)b * a.H * D + i, 0.0f);
            if (a.lse)
                for (int i = threadIdx.x; i < a.H; i += kThreads) a.lse[(int64_t)b * a.H + i] = -INFINITY;
        }
    const int64_t T = (int64_t)total * per;
    if (T == 0) return;
    // Two steps to a wave at least, in ranges.  Where there are workgroups for each sequence and head tile to have its own, as many
    // as its steps take, they are dealt out so, unless the longest part takes longer than the line's equal ranges and the joins
    // that these need: a range is read at the memory's rate (its bytes count), a part of one's own at the memory's latency,
    // about twice that rate at most.  (Two steps a wave throughout, 7 sequences of 1000 tokens, 8 key heads of 128: 17 us dealt out,
    // 20.6 in ranges; 30 of 1000: 28 and 33.5; 16 of 100 to 4000: 31 and 25.5; 30 of 100 to 2000: 29.6 and 26.5.)
    constexpr int kPart = 2 * kWaves;
    // One workgroup takes up to two steps a wave, which cost what a join through memory does; of more, every step a wave of its
    // own, where there are as many.  (Two steps to a wave, and one: a sequence of 1000 tokens, 8 key heads of 128, 14.9 and 12.6 us, of
    // 4000 16.9 and 14.4, 7 of 1000 17.2 and 14.9; 500 tokens of heads of 64 8.7 and, in two workgroups, 10.1.)
    auto parts_for = [&](int n) { return n <= kPart ? 1 : (n + kWaves - 1) / kWaves; };
    const int each = a.most_each < parts_for(longest) ? a.most_each : parts_for(longest);
    const bool dealt = each > 0 && (int64_t)longest * gridDim.x <= each * (kPart * (int64_t)gridDim.x + (E4M3 ? 1 : 2) * T * D * kWaves / 1024);
    const int cost = dealt ? kPieceCost : 0;  // (that a part of one's own has no use for)
    const int64_t want = (T + kPart - 1) / kPart;
    const int groups = want < (int64_t)gridDim.x ? (int)want : (int)gridDim.x;
    const int g = blockIdx.x;
    int64_t f0, f1;
    PieceOf own;      // the sequence and head tile of one's own, if dealt out; `begin`: none
    int64_t own_at;   // its place on the line
    // Of a sequence and head tile's n steps: workgroups that have some of them.
    auto members_of = [&](int n) { return parts_for(n) < each ? parts_for(n) : each; };
    if (dealt) {
        const int piece = each == 1 ? g : g / each, j = g - piece * each;
        own.b = piece / per;
        own.ht = piece - own.b * per;
        own.n = own.b < a.B ? upto[own.b + 1] - upto[own.b] - cost : 0;
        const int members = members_of(own.n);
        if (own.n <= 0 || j >= members) return;
        f0 = own_at = (int64_t)per * upto[own.b] + (int64_t)own.ht * own.n;
        f1 = f0 + own.n;
        if (members > 1) {
            f1 = f0 + quotient((int64_t)own.n * (j + 1), members);
            f0 += quotient((int64_t)own.n * j, members);
        }
    } else {
        if (g >= groups) return;
        f0 = quotient(T * g, groups);
        f1 = quotient(T * (g + 1), groups);
    }
    const int64_t R = f1 - f0;
    const int64_t w0 = f0 + R * w / kWaves, w1 = f0 + R * (w + 1) / kWaves;

    auto write = [&](int64_t row, int i, float v) { store_global(a.out, a.out_dtype, row * D + i, v); };
    for (int64_t f = w0; f < w1;) {
        PieceOf p;
        if (dealt) {
            p = own;
            p.begin = __builtin_amdgcn_readfirstlane((int)(f - own_at));
        } else {
            const int x = (int)quotient(f, per);
            int lo = 0, hi = a.B;  // upto[lo] <= x < upto[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (upto[mid] <= x)
                    lo = mid;
                else
                    hi = mid;
            }
            p.b = __builtin_amdgcn_readfirstlane(lo);
            p.n = upto[lo + 1] - upto[lo];
            const int64_t r = f - (int64_t)per * upto[lo];
            p.ht = __builtin_amdgcn_readfirstlane((int)quotient(r, p.n));
            p.begin = __builtin_amdgcn_readfirstlane((int)(r - (int64_t)p.ht * p.n));
        }
        p.n = __builtin_amdgcn_readfirstlane(p.n);
        p.end = (int64_t)(p.n - p.begin) < w1 - f ? p.n : p.begin + (int)(w1 - f);
        p.end = __builtin_amdgcn_readfirstlane(p.end);
        f += p.end - p.begin;
        Span sp = span_of(a, p.b);
        State<D, E4M3> st;
        st.clear();
        const int count = (p.end < sp.steps ? p.end : sp.steps) - p.begin;
        if (count > 0) attend<D, E4M3>(a, p.b, key_head_of(p.ht), tile_of(p.ht), sp, sp.first + p.begin, count, st);
        float l = with_lane_xor<16>(st.l, AddOp());
        l = with_lane_xor<32>(l, AddOp());
        const int heads = heads_of(p.ht);
        if (p.begin == 0 && p.end == p.n) {
            if (n < heads) {
                const int64_t row = row_of(p.b, p.ht) + n;
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) write(row, 16 * d + 4 * kb + i, l == 0.0f ? 0.0f : st.sum(d, i) * inv);
                if (a.lse && kb == 0) a.lse[row] = l == 0.0f ? -INFINITY : st.m + logf(l);
            }
        } else {
            const int slot = p.begin > 0 ? 0 : 1;
            if (n < heads) {
                float *const to = parts + ((w * 2 + slot) * heads_most + n) * kRow;
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[16 * d + 4 * kb + i] = st.sum(d, i);
                if (kb == 0) {
                    to[D] = st.m;
                    to[D + 1] = l;
                }
            }
            if (lane == 0) held[w][slot] = p;
        }
    }
    __syncthreads();

    // The waves' parts: a piece that starts in one wave goes on in the next ones' first slots.  (What all have is looked at
    // at once; with loops over the waves, one value after the other, this took 4 us.)
    PieceOf shared_piece[2];  // what is left for others to join: begun before this workgroup, going on after it
    shared_piece[0].b = shared_piece[1].b = -1;
    // Of the first slots, by a lane each: where their pieces end, which there are, and which end in them; which second ones there are.
    const PieceOf first_slot = held[lane & (kWaves - 1)][0];
    const int end_of = first_slot.end;
    const uint32_t goes = (uint32_t)__ballot(lane < kWaves && first_slot.b >= 0);
    const uint32_t ended = goes & (uint32_t)__ballot(first_slot.end == first_slot.n);
    const uint32_t starts = (uint32_t)__ballot(lane < kWaves && held[lane & (kWaves - 1)][1].b >= 0);
    // (start -1: what begins before this workgroup, in the first slot of the first wave that has any steps)
    int front = 0;
    while (R * (front + 1) / kWaves == 0) ++front;
    // (of short sequences many begin and end in a workgroup, a wave to each then)
    const bool many = __builtin_popcount(starts) > 2;
    for (int start = -1, turn = 0; start < kWaves; ++start) {
        if (start >= 0 && !(starts >> start & 1)) continue;
        const int slot = start < 0 ? 0 : 1, first = start < 0 ? front : start;
        const PieceOf in_lds = held[first][slot];
        PieceOf p;
        p.b = __builtin_amdgcn_readfirstlane(in_lds.b);
        if (p.b < 0) continue;
        p.ht = __builtin_amdgcn_readfirstlane(in_lds.ht);
        p.begin = __builtin_amdgcn_readfirstlane(in_lds.begin);
        p.end = __builtin_amdgcn_readfirstlane(in_lds.end);
        p.n = __builtin_amdgcn_readfirstlane(in_lds.n);
        uint32_t members = 1u << first;
        int until = p.end;
        if (until < p.n) {
            const uint32_t after = ~((2u << first) - 1), stop = ended & after;
            members |= goes & after & (stop ? stop ^ (stop - 1) : ~0u);
            const int top = 31 - __builtin_clz(members);
            if (top > first) until = __builtin_amdgcn_readlane(end_of, top);
        }
        const int heads = heads_of(p.ht);
        const bool whole = p.begin == 0 && until == p.n;
        const int to_slot = p.begin > 0 ? 0 : 1;
        if (!whole) {
            p.end = until;
            if (to_slot)
                shared_piece[1] = p;
            else
                shared_piece[0] = p;
        }
        auto finish = [&](int h, int d, float most, float sum, float out) {
            if (whole) {
                const int64_t row = row_of(p.b, p.ht) + h;
                write(row, d, sum == 0.0f ? 0.0f : out / sum);
                if (a.lse && d == 0) a.lse[row] = sum == 0.0f ? -INFINITY : most + logf(sum);
            } else {
                float *const to = a.partial + ((int64_t)(g * 2 + to_slot) * kHeadTile + h) * kRow;
                put(to + d, out);
                if (d == 0) {
                    put(to + D, most);
                    put(to + D + 1, sum);
                }
            }
        };
        if (many) {
            if (turn++ % kWaves != w) continue;
            for (int h = 0; h < heads; ++h) {  // (of few waves each)
                float most = -INFINITY, sum = 0.0f, out[(D + 63) / 64] = {};
                for (uint32_t left = members; left; left &= left - 1) {
                    const int i = __builtin_ctz(left);
                    const float *const part = parts + ((i * 2 + (i == first ? slot : 0)) * heads_most + h) * kRow;
                    const float m = part[D], next = fmaxf(most, m), old = factor(most, next), c = factor(m, next);
                    sum = sum * old + c * part[D + 1];
#pragma unroll
                    for (int k = 0; k < (D + 63) / 64; ++k) out[k] = out[k] * old + c * part[64 * k + lane < D ? 64 * k + lane : 0];
                    most = next;
                }
#pragma unroll
                for (int k = 0; k < (D + 63) / 64; ++k)
                    if (64 * k + lane < D) finish(h, 64 * k + lane, most, sum, out[k]);
            }
            continue;
        }
        for (int e = threadIdx.x; e < heads * D; e += kThreads) {
            const int h = e / D, d = e % D;
            float m[kWaves], l[kWaves], o[kWaves], most = -INFINITY;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float *const part = parts + ((i * 2 + (i == first ? slot : 0)) * heads_most + h) * kRow;
                const bool there = members >> i & 1;
                m[i] = part[D];  // (without a branch; what is not there may be anything)
                l[i] = part[D + 1];
                o[i] = part[d];
                m[i] = there ? m[i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < kWaves; ++i) most = fmaxf(most, m[i]);
            float sum = 0.0f, out = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const bool there = members >> i & 1;
                const float c = factor(m[i], most);
                sum += there ? c * l[i] : 0.0f;
                out += there ? c * o[i] : 0.0f;
            }
            finish(h, d, most, sum, out);
        }
    }
    // Parts in the workspace are written through to where all XCDs see them, and waited for, before this workgroup
    // arrives; the last one's loads pass its caches by.
    if (shared_piece[0].b < 0 && shared_piece[1].b < 0) return;  // (the same for the whole workgroup)
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
    // The workgroups that have some of a sequence and head tile, which only one can be the first of.
    auto group_of = [&](int64_t f) { return (int)quotient((f + 1) * groups - 1, T); };
    auto groups_with = [&](const PieceOf &p, int *from, int *to) {
        if (dealt) {
            *from = (p.b * per + p.ht) * each;
            *to = *from + members_of(p.n) - 1;
        } else {
            const int64_t at = (int64_t)per * upto[p.b] + (int64_t)p.ht * p.n;
            *from = group_of(at);
            *to = group_of(at + p.n - 1);
        }
    };
    if (w < 2) {  // (a wave each, side by side)
        const PieceOf p = w ? shared_piece[1] : shared_piece[0];
        bool done = false;
        if (p.b >= 0 && lane == 0) {
            int from, to;
            groups_with(p, &from, &to);
            const uint32_t before = __hip_atomic_fetch_add(a.arrived + from, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            done = before == (uint32_t)(to - from);
            if (done) __hip_atomic_store(a.arrived + from, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (lane == 0) last[w] = done;
    }
    __syncthreads();
    for (int i = 0; i < 2; ++i) {
        if (!last[i]) continue;  // (the same for the whole workgroup)
        const PieceOf p = i ? shared_piece[1] : shared_piece[0];
        int from, to;
        groups_with(p, &from, &to);
        from = __builtin_amdgcn_readfirstlane(from);
        const int count = __builtin_amdgcn_readfirstlane(to) - from + 1, heads = heads_of(p.ht);
        // What workgroup from + j has of it: behind the beginning in the first slot.
        auto part = [&](int j) { return a.partial + (int64_t)((from + j) * 2 + (j == 0 ? 1 : 0)) * kHeadTile * kRow; };
        // The factors of the parts, [count][heads], where the waves' parts were; m and l of a head behind them.  The first
        // parts' sums are asked for together with what the factors are made of, as many as there are likely to be and
        // without branches between the loads.
        float *const scale = parts, *const sums = parts + count * heads;
        auto join = [&](auto at_once) {
            constexpr int kAtOnce = decltype(at_once)::value;
            float v[kAtOnce];
            auto ask = [&](int off, int j0) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) v[j] = get(part(j0 + j < count ? j0 + j : count - 1) + off);
            };
            const int e0 = (int)threadIdx.x < heads * D ? (int)threadIdx.x : 0;
            ask(e0 / D * kRow + e0 % D, 0);
            for (int h = w; h < heads; h += kWaves) {
                float most = -INFINITY, l = 0.0f;
                for (int j0 = 0; j0 < count; j0 += 64) {
                    const int j = j0 + lane < count ? j0 + lane : count - 1;
                    const float m = get(part(j) + h * kRow + D), s = get(part(j) + h * kRow + D + 1);
                    if (j0 + lane < count) scale[j * heads + h] = m;
                    const float top = fmaxf(most, wave_max(m));
                    l = l * factor(most, top) + (j0 + lane < count ? s * factor(m, top) : 0.0f);  // (of a lane)
                    most = top;
                }
                l = group_sum<64>(l);
                for (int j = lane; j < count; j += 64) scale[j * heads + h] = factor(scale[j * heads + h], most);
                if (lane == 0) {
                    sums[2 * h] = most;
                    sums[2 * h + 1] = l;
                }
            }
            __syncthreads();
            for (int e = threadIdx.x; e < heads * D; e += kThreads) {
                const int h = e / D, d = e % D;
                float o = 0.0f;
                for (int j0 = 0; j0 < count; j0 += kAtOnce) {
                    if (j0 > 0 || e >= kThreads) ask(h * kRow + d, j0);
                    float c[kAtOnce];
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) c[j] = scale[(j0 + j < count ? j0 + j : count - 1) * heads + h];
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) o += j0 + j < count ? c[j] * v[j] : 0.0f;
                }
                const float most = sums[2 * h], l = sums[2 * h + 1];
                const int64_t row = row_of(p.b, p.ht) + h;
                write(row, d, l == 0.0f ? 0.0f : o / l);
                if (a.lse && d == 0) a.lse[row] = l == 0.0f ? -INFINITY : most + logf(l);
            }
        };
        if (count <= 4)
            join(std::integral_constant<int, 4>());
        else
            join(std::integral_constant<int, 16>());
        __syncthreads();  // (the room may be needed for the other piece)
    }
}

constexpr int64_t kMostSteps = 1ll << 30;  // of all sequences, per head tile

template <int D>
int launch_attention(AttentionArgs a, hipStream_t st) {
    constexpr int kWaves = waves_of<D>();
    const int cu = device_cu_count(), heads = a.group < kHeadTile ? a.group : kHeadTile;
    const int64_t steps = (int64_t)a.B * (((int64_t)a.width << a.c.page_shift) / kStep + 1 + kPieceCost) * a.c.heads * a.tiles;
    const int64_t pieces = (int64_t)a.B * a.c.heads * a.tiles, ranges = (steps + kWaves - 1) / kWaves,
                  want = ranges > pieces ? ranges : pieces, most = cu < kMaxGroups ? cu : kMaxGroups;
    const dim3 grid((unsigned)(want < most ? want : most)), block(64 * kWaves);
    a.most_each = (int)(grid.x / pieces);
    // (the parts' room also holds the factors and sums of a join: kMaxGroups + 2 per head)
    static_assert(2 * kWaves * (D + 2) >= kMaxGroups + 2, "room for a join");
    const size_t lds = (((size_t)a.B + 1) * 4 + 15) / 16 * 16 + sizeof(float) * 2 * kWaves * heads * (D + 2);
    if (a.c.e4m3)
        hipLaunchKernelGGL((attention_kernel<D, true>), grid, block, lds, st, a);
    else
        hipLaunchKernelGGL((attention_kernel<D, false>), grid, block, lds, st, a);
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
    return NVQ_ATTENTION_CLEAR_BYTES + sizeof(float) * kMaxGroups * 2 * kHeadTile * (size_t)(cache->head_dim + 2);
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
        B * ((int64_t)table_width * cache->page_size / kStep + 1) > kMostSteps ||
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
    a.arrived = static_cast<uint32_t *>(workspace);
    a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + NVQ_ATTENTION_CLEAR_BYTES);
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
