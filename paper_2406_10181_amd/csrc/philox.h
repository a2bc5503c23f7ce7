// Dropout masks from a counter-based generator: Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), the fewest rounds that the authors found to pass all of their tests.
//
// A round multiplies words 0 and 2 of the counter by two constants and takes both halves of the products; the halves, the
// other two words and a key that grows by a constant every round make the next counter.  Four words come out; here they are
// taken as eight of 16 bits, one an element: the integer multiplies are what a mask costs (four passes of the vector unit each), and a
// probability in steps of 1 / 65536 is as fine as a dropout rate needs.
#pragma once

#include "lsp_internal.h"

namespace lsp {

// What a kernel needs of a dropout: 16-bit words below `limit` are dropped, the others scaled.
struct Dropout {
    uint32_t key0, key1, offset;
    uint32_t limit;              // 0: nothing is dropped
    float    scale;              // 65536 / (65536 - limit)
};

static inline Dropout make_dropout(float p, uint64_t seed, uint32_t offset) {
    Dropout d;
    d.key0 = (uint32_t)seed; d.key1 = (uint32_t)(seed >> 32); d.offset = offset;
    const double t = (double)p * 65536.0 + 0.5;
    d.limit = t >= 65535.0 ? 65535u : (uint32_t)t;               // (p < 1: the one that is left at the very end is never dropped)
    d.scale = 65536.0f / (float)(65536u - d.limit);
    return d;
}

#if defined(__HIPCC__)
__device__ __forceinline__ u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 7; ++round) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0; c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1; c3 = (uint32_t)a;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}
// Word e of the eight
__device__ __forceinline__ uint32_t philox_word(const u32x4& w, int e) { return e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu; }
#endif

}  // namespace lsp
