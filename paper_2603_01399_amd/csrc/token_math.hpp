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
constexpr int kListBits = 43;                                // a whole vocabulary has at most 2^20
constexpr int kFewBits = 51;                                 // of at most 2^11 tokens
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

// A logit's place on the line of buckets, plus 1.5 2^52: to the nearest whole number, falls with z never, and the same for every part of a vocabulary.  In 64 bits:
// a logit may be 2^24 buckets and more away from 0 (2^20 temperatures), and the few between it and another one have to be exact all the same.  (Beyond 2^51, where
// places are no longer every whole number, different logits are 2^26 buckets apart.)
QUASAR_BOTH double bucket_line(float z, double scale) { return __builtin_fma((double)z, scale, 0x1.8p52); }
// Bucket of a logit, 0 for those nearest the largest one (line_top: its place, of a finite logit); kBuckets: beyond them all, as -inf is (whose place is no
// number at a scale of 0: fmin takes the other one).
QUASAR_BOTH int bucket_of(float z, double scale, double line_top) { return (int)__builtin_fmin(line_top - bucket_line(z, scale), (double)kBuckets); }
// The last bucket that a logit can lie in whose weight is at least this: D = 16 ln(1 / min_p) buckets below the largest, two roundings of at most half a bucket each.
QUASAR_BOTH int last_bucket(float log2_min_p) {
    const int last = (int)(-0.6931472f * kBucketsPerUnit * log2_min_p) + 2;
    return last < kBuckets - 1 ? last : kBuckets - 1;
}
// What a row's filters come to.
struct Filters {
    double rate;              // log2(e) / temperature
    double scale;             // kBucketsPerUnit / temperature
    float temperature;        // above 0
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
    f.temperature = temperature;
    if (f.p <= 0.0f) f.p = 1.0f, f.k = 1;                    // (the first is always left)
    const double scale = (double)kBucketsPerUnit / (double)temperature;
    f.rate = scale * (1.4426950408889634 / kBucketsPerUnit);
    f.scale = scale < (double)kLargest ? scale : (double)kLargest;
    return f;
}
// The smallest logit of buckets 0 .. j, as ordered bits, found by 64 at a time: around where the line says, else anywhere.  `ballot` asks whether a number holds
// for lanes 0 .. 63, `most` is the largest logit.  What a bucket holds is asked of bucket_of, so that an interval of logits is the bucket's exactly.  (Zero in the
// form that orders ahead of the other.)
template <class Ballot>
QUASAR_BOTH uint32_t least_of_buckets(int j, const Filters &f, double line_top, float most, Ballot ballot) {
    const uint32_t least = ordered_bits(-kLargest), largest = ordered_bits(most);
    auto holds = [&](uint32_t at) { return bucket_of(value_of_ordered(at), f.scale, line_top) <= j; };
    const double place = (line_top - 0x1.8p52 - (double)j - 0.5) * (1.0 / kBucketsPerUnit * (double)f.temperature);
    const float guess = (float)__builtin_fmin(__builtin_fmax(place, -(double)kLargest), (double)most);
    const long long first = (long long)ordered_bits(guess) - 32;
    auto around = [&](int i) { return (uint32_t)(first + i < (long long)least ? least : first + i > (long long)largest ? largest : first + i); };
    u64 held = ballot([&](int i) { return holds(around(i)); });
    uint32_t found;
    if (held && (!(held & 1) || around(0) == least)) {
        found = around(__builtin_ctzll(held));
    } else {
        uint32_t lo = least, hi = largest;                       // (it holds for the largest)
        while (lo < hi) {
            const uint32_t step = (hi - lo) / 64 + 1;
            auto here = [&](int i) { return (uint32_t)((u64)lo + (u64)step * (u64)i < hi ? (u64)lo + (u64)step * (u64)i : hi); };
            held = ballot([&](int i) { return holds(here(i)); });
            const int l = held ? __builtin_ctzll(held) : 64;     // (none: it is behind the last one asked)
            const uint32_t behind = l ? here(l - 1) + 1 : lo;
            if (held) hi = here(l);
            lo = behind;
        }
        found = hi;
    }
    return found == ordered_bits(0.0f) ? found - 1 : found;
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
