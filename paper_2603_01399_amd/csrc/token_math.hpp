// The arithmetic of drawing tokens from filtered logits (tokens.hpp): weights, the order that the filters go by, buckets.  Plain C++ for both sides: the
// kernels run it on the GPU, the tests run the same functions on the CPU.
//
// Weights are exp((z - largest) / temperature) in 64 bits, taken as whole multiples of 2^-bits of a reference: sums are exact in any order, so
// that atomics change no result, and what is drawn inside a part of the vocabulary is drawn from exactly the mass that was counted there.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>

#include "draw.hpp"

namespace quasar {

typedef unsigned long long u64;

constexpr int kBuckets = 512, kBucketsPerUnit = 16;          // of (largest - z) / temperature: the first 32 units; what lies behind weighs less than 2^-46
constexpr int kPartBits = 48;                                // a part of the vocabulary has at most 2^13 tokens
constexpr int kListBits = 42;                                // a whole vocabulary has at most 2^20
constexpr int kIndexBits = 20;
constexpr float kLargest = 3.4028234663852886e38f;

// A logit as it counts: none for what is not a number, the largest finite value for infinity ...
QUASAR_BOTH float logit_weighed(float z) { return __builtin_fminf(__builtin_fmaxf(z, -__builtin_inff()), kLargest); }
// ... and, where it is ordered, one zero.
QUASAR_BOTH float logit_value(float z) { return logit_weighed(z) + 0.0f; }

QUASAR_BOTH u64 bits_of(double x) {
    u64 u;
    memcpy(&u, &x, 8);
    return u;
}
QUASAR_BOTH double double_of(u64 u) {
    double x;
    memcpy(&x, &u, 8);
    return x;
}
// A constant, SCALAR: in a scalar register pair on the GPU, which a multiply-add takes as it is.  Else the compiler copies each into vector registers where it is
// used, two instructions beside every multiply-add.  That costs where many tokens' weights bound a kernel (64 rows of 151936 logits without filters 26.1 us, and 25.2
// so), not where a few wait for one another (one row 12.3, and 12.8 so).
template <bool SCALAR> QUASAR_BOTH double constant(double c) {
#ifdef __HIP_DEVICE_COMPILE__
    if (SCALAR) asm("" : "+s"(c));
#endif
    return c;
}
// 2^(y + extra) for -1000 < y < 1000: y's nearest whole number, by the sum with 1.5 2^52 (and extra), goes to the exponent; 2^f of the rest, |f| <= 1/2, by the
// polynomial of degree ten that meets it at the Chebyshev points of the interval: off by at most 2^-51.5 of it.
template <bool SCALAR = false> QUASAR_BOTH double exp2_by(double y, int extra) {
    const double whole = 0x1.8p52 + (double)extra, t = y + whole, f = y - (t - whole);
    double r = 0x1.e6063f7217bc6p-28;
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.b675bca4eeebbp-24));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.62bfd47773353p-20));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.ffcb54062e698p-17));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.430913096fd9fp-13));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.5d87fe9d7a584p-10));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.3b2ab6fba1ddap-7));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.c6b08d703ce49p-5));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.ebfbdff82c598p-3));
    r = __builtin_fma(r, f, constant<SCALAR>(0x1.62e42fefa3a19p-1));
    r = __builtin_fma(r, f, 1.0);
    const u64 at = bits_of(r);
    return double_of((u64)((uint32_t)(at >> 32) + ((uint32_t)bits_of(t) << 20)) << 32 | (uint32_t)at);
}
// exp((z - ref) / temperature) for z <= ref, 0 below 2^-60 (and of -inf, also times a rate of 0); rate: log2(e) / temperature.
QUASAR_BOTH double weight_of(float z, float ref, double rate) {
    const double y = ((double)z - (double)ref) * rate;
    return y > -60.0 ? exp2_by(y, 0) : 0.0;
}
// The same in whole multiples of 2^-bits, to nearest (bits <= 51).
template <bool SCALAR = false> QUASAR_BOTH u64 weight_units(float z, float ref, double rate, int bits) {
    const double y = __builtin_fmax(((double)z - (double)ref) * rate, -110.0);   // (which rounds to none)
    return bits_of(exp2_by<SCALAR>(y, bits) + 0x1p52) & ((1ull << 52) - 1);
}

// The order of the filters: larger logits first, equal ones by their place.  A logit's rank is its bits in falling order: 32 of an fp32 one, 16 of a bf16 one
// (DT 1), so that keys are dense: 52 or 36 bits with the place.
QUASAR_BOTH uint32_t ordered_bits(float z) {                 // grows with z
    uint32_t u;
    memcpy(&u, &z, 4);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
QUASAR_BOTH float value_of_ordered(uint32_t u) {
    u = u & 0x80000000u ? u & 0x7FFFFFFFu : ~u;
    float z;
    memcpy(&z, &u, 4);
    return z;
}
constexpr int kLastPlace = (1 << kIndexBits) - 1;
template <int DT> QUASAR_BOTH u64 rank_key(float z, int v) {
    return (u64)(~ordered_bits(z) >> (DT == 1 ? 16 : 0)) << kIndexBits | (u64)(uint32_t)v;
}
template <int DT> QUASAR_BOTH float key_value(u64 key) {
    const uint32_t rank = (uint32_t)(key >> kIndexBits);
    // (a bf16's lower bits are 0: those of the ordered form where it is not negative, of its complement where it is)
    return value_of_ordered(DT == 1 ? (rank < 0x8000u ? ~rank << 16 : ~(rank << 16)) : ~rank);
}
QUASAR_BOTH int key_token(u64 key) { return (int)(key & (u64)kLastPlace); }
// The last key of logits whose ordered bits are at least these: of the smallest bf16 that is not below them.
template <int DT> QUASAR_BOTH u64 last_key(uint32_t least) {
    if (DT == 1) least = least & 0x80000000u ? (least + 0xFFFFu) & 0xFFFF0000u : least | 0xFFFFu;
    return (u64)(~least >> (DT == 1 ? 16 : 0)) << kIndexBits | (u64)kLastPlace;
}

// The first key of logits whose ordered bits are at most these: of the largest bf16 that is not above them.
template <int DT> QUASAR_BOTH u64 first_key(uint32_t most) {
    if (DT == 1 && !(most & 0x80000000u)) most = ((most + 1) & 0xFFFF0000u) - 1;
    return (u64)(~most >> (DT == 1 ? 16 : 0)) << kIndexBits;
}

// A logit's place on the line of buckets: whole, falls with z never, and the same for every part of a vocabulary.  (fmax takes what is not a number,
// -inf times a scale of 0, for the smallest.)
QUASAR_BOTH float bucket_line(float z, float scale) { return __builtin_floorf(__builtin_fminf(__builtin_fmaxf(z * scale, -kLargest), kLargest)); }
// Bucket of a logit, 0 for those nearest the largest one (line_top: its place, of a finite logit); kBuckets: beyond them all, as -inf is.
QUASAR_BOTH int bucket_of(float z, float scale, float line_top) {
    const float d = line_top - bucket_line(z, scale);
    return z == -__builtin_inff() ? kBuckets : (int)__builtin_fminf(d, (float)kBuckets);
}

// What a row's filters come to.
struct Filters {
    double rate;              // log2(e) / temperature
    float scale;              // kBucketsPerUnit / temperature
    int k;                    // 0: no limit
    float p;                  // 1: no limit
    float min_p;              // 0: no limit
};
QUASAR_BOTH Filters filters_of(float temperature, int top_k, float top_p, float min_p, int V) {
    Filters f;
    f.k = top_k > 0 && top_k < V ? top_k : 0;
    f.p = top_p < 1.0f ? top_p : 1.0f;                       // (not a number: no limit)
    f.min_p = min_p > 0x1p-50f ? (min_p < 1.0f ? min_p : 1.0f) : 0.0f;   // (what weighs less is beyond the buckets)
    if (!(temperature > 0.0f)) temperature = 1.0f, f.k = 1;
    if (f.p <= 0.0f) f.p = 1.0f, f.k = 1;                    // (the first is always left)
    f.rate = 1.4426950408889634 / (double)temperature;
    const float scale = (float)kBucketsPerUnit / temperature;
    f.scale = scale < kLargest ? scale : kLargest;
    return f;
}
// The smallest logit whose weight is at least min_p (> 0); most: the largest logit.
QUASAR_BOTH float least_logit(float most, double rate, float min_p) {
    const double at = (double)most + log2((double)min_p) / rate;
    float z = at > -(double)kLargest ? (float)at : -kLargest;
    for (int i = 0; i < 4 && z < most && weight_of(z, most, rate) < (double)min_p; ++i) z = value_of_ordered(ordered_bits(z) + 1);
    for (int i = 0; i < 4 && z > -kLargest; ++i) {
        const float below = value_of_ordered(ordered_bits(z) - 1);
        if (weight_of(below, most, rate) < (double)min_p) break;
        z = below;
    }
    return z < most ? z : most;
}

}  // namespace quasar
