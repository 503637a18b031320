// Which elements dropout keeps: the counter-based decisions shared by qmm_dropout.hip and qmm_layernorm.hip.  Element p of a dense tensor has number
// n = p + offset; its 16 random bits are half (n % 2), the low one first, of word (n % 8) / 2 of Philox4x32-10 with counter (n / 8 as two 32-bit
// words, 1, 0) and key = seed, and it is dropped iff they are below `least` = round(65536 p).  16 bits, not 24 as in stochastic rounding: one block of the
// generator, what bounds that, serves eight elements instead of four; the third counter word keeps the two streams apart.
#pragma once
#include "qmm_encode.h"

namespace qmm {
namespace {

struct Drop {
    uint64_t seed, offset;
    uint32_t least;            // 0: nothing is dropped
    float scale;               // 65536 / (65536 - least): what is kept is multiplied by it, so the mean stays what it was exactly
};

// The random bits of V (4 or 8) elements from number n on, and whether element n + e is kept: its sixteen bits, as the high half of a word, are above the last word
// of those that are dropped.
struct Kept {
    u32x4 words;
    uint32_t last;             // (least << 16) - 1: nothing is above it where everything is dropped; least 0 is the caller's
    QMM_DEV bool operator[](int e) const { return ((e & 1) ? words[e >> 1] : words[e >> 1] << 16) > last; }
};
template <int V> QMM_DEV Kept kept(const Drop& d, uint64_t n)
{
    const uint64_t c = n >> 3;
    const uint32_t j = (uint32_t)n & 7u, k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
    // (words of 64 bits, not an array of eight of 32: the compiler kept that in LDS, 16 us where 4 M bytes take 3)
    auto words = [&](uint64_t n, uint64_t& low, uint64_t& high) {
        const Philox4 p = philox4x32_10((uint32_t)n, (uint32_t)(n >> 32), 1u, 0u, k0, k1);
        low = p.v[0] | (uint64_t)p.v[1] << 32;
        high = p.v[2] | (uint64_t)p.v[3] << 32;
    };
    uint64_t q0, q1;
    words(c, q0, q1);
    if (__any(j != 0u)) {
        uint64_t q2 = 0, q3 = 0;
        if (__any(j + V > 8u)) {
            asm volatile("; parts of blocks");           // (keeps the compiler from computing this for every call and selecting)
            words((n + 8) >> 3, q2, q3);         // (behind the last number comes number 0: element counts are modulo 2^64)
        }
        if (j & 4u) { q0 = q1; q1 = q2; q2 = q3; }
        const uint32_t away = (j & 3u) * 16u;
        q0 = q0 >> away | (q1 << 1) << (63u - away);
        q1 = q1 >> away | (q2 << 1) << (63u - away);
    }
    return Kept{u32x4{(uint32_t)q0, (uint32_t)(q0 >> 32), (uint32_t)q1, (uint32_t)(q1 >> 32)}, (d.least << 16) - 1u};
}
// V values times the factor where they are kept, 0 where not.
template <int V> QMM_DEV void drop_values(const Drop& d, uint64_t n, const float* v, float* out)
{
    if (d.least == 0u) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = v[e];
        return;
    }
    const Kept keep = kept<V>(d, n);
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = keep[e] ? v[e] * d.scale : 0.0f;
}

// host: p in [0, 1]
inline bool drop_of(float p, uint64_t seed, uint64_t offset, Drop* d)
{
    if (!(p >= 0.0f && p <= 1.0f)) return false;
    d->seed = seed; d->offset = offset;
    d->least = (uint32_t)((double)p * 65536.0 + 0.5);
    d->scale = d->least < 65536u ? (float)(65536.0 / (65536.0 - d->least)) : 0.0f;
    return true;
}

}  // namespace
}  // namespace qmm
