// The paged cache of keys and values as its kernels see it.
#pragma once

#include "nvq_internal.h"

namespace nvq {

struct CacheView {
    void *k, *v;
    uint8_t *scales;
    int pages, heads, page_size, page_shift, D;
    bool e4m3;
};

// Where token t of a call is to be found.
struct Places {
    const int32_t *table, *sequences, *positions;
    int B, width, T;
};

int check_cache(const nvq_cache *c);     // NVQ_OK or what is wrong with it
int check_places(const Places &p);       // likewise
CacheView view_of(const nvq_cache &c);   // of a checked one

#if defined(__HIPCC__)

// The first value of a token's key row, and of channel 0 in a token's value row (channel d: 8 d further).
__device__ __forceinline__ int64_t key_at(const CacheView &c, int page, int head, int slot) {
    return (((int64_t)page * c.heads + head) * c.page_size + slot) * c.D;
}
__device__ __forceinline__ int64_t value_at(const CacheView &c, int page, int head, int slot) {
    return (((int64_t)page * c.heads + head) * (c.page_size >> 3) + (slot >> 3)) * c.D * 8 + (slot & 7);
}
// The scale byte of a token's keys (which = 0) or values (1).
__device__ __forceinline__ int64_t scale_at(const CacheView &c, int page, int head, int which, int slot) {
    return (((int64_t)page * c.heads + head) * 2 + which) * c.page_size + slot;
}
// 2^(byte - 127); byte 0 has no normal number, 255 stands for NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte << 23 | (byte == 0 || byte == 255 ? 0x400000u : 0u));
}

#endif  // __HIPCC__

}  // namespace nvq
