// Paged key/value cache of a batch of sequences (gfx950): where a position lies, which rows a sequence has, and the
// append of new tokens.  Head dimension 128.
//
// A page holds `page_len` positions (a power of two, 32 .. 1024) of every kv head: [kv head][block of 32 positions][keys | values],
// each block in the matrix-core operand order of the contiguous cache (attention.hpp), so that a wave's 128-bit loads are
// 1 KB of contiguous memory and already operands:
//   bf16  as there;
//   e4m3  half as long, a lane's 16 bytes being two neighbouring operands:
//         keys [sub 2][kstep pair 4/2][g4 4][p 16][kstep 2][8 d], values [dt pair 8/2][g4 4][dd 16][dt 2][slot 8].
// A sequence's pages are a row of the page table; -1 = none.  Everything that says what to touch (table, lengths, row starts) is device memory
// that the host never sees: every kernel bounds what it reads from there before it uses it as an address, so that wrong books give
// wrong values but touch nothing outside the buffers.
#pragma once

#include "books.hpp"
#include "kv_layout.hpp"

namespace quasar {

constexpr float kE4m3Max = 448.f;            // largest finite e4m3 value: beyond it the append saturates

constexpr int kBlockShift = 5;               // a block of 32 positions
static_assert(kKvBlock == 1 << kBlockShift, "positions of a block");

enum { KV_BF16 = 0, KV_E4M3 = 1 };
template <int KV> constexpr int kv_block_bytes = KV == KV_E4M3 ? kKvBlockBytes / 2 : kKvBlockBytes;   // keys or values of 32 positions of a head

struct PagedParams {
    unsigned char *pages;     // [n_pages][Hkv][page_blocks][2][kv_block_bytes], one layer
    const int32_t *table;     // [n_seqs][table_ld] page ids
    const int32_t *lengths;   // [n_seqs] positions cached ahead of the new rows
    const int32_t *row_start; // [n_seqs + 1] rows of the packed tensors
    const float *k_scale, *v_scale;   // [Hkv] of e4m3 pages (NULL: 1)
    long long table_ld;
    int T, n_seqs, n_pages, columns, Hkv, Hq, G;
    int block_shift;          // log2 of the blocks of a page
    int max_new;              // rows of a sequence that the call takes
};

__device__ __forceinline__ SeqSpan seq_span(const PagedParams &p, int s) {
    SeqSpan a = span_of(p.row_start[s], p.row_start[s + 1], p.lengths[s], p.T);
    a.n = a.n < p.max_new ? a.n : p.max_new;
    return a;
}
__device__ __forceinline__ int blocks_of(const PagedParams &p, int total) { return blocks_reached(total, p.columns, p.block_shift); }

// Sequence of packed row t (-1 behind the last one): how many sequences end at or before it.
__device__ __forceinline__ int seq_of_row(const PagedParams &p, int t, int lane) {
    int s = 0;
    for (int i = 0; i < p.n_seqs; i += 64) {
        const bool before = i + lane < p.n_seqs && p.row_start[i + lane + 1] <= t;
        s += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    return s < p.n_seqs ? s : -1;
}

// Exclusive prefix sums of v(0 .. n - 1) into out[0 .. n - 1]; the sum for all threads of the workgroup.
template <int NW, class V>
__device__ __forceinline__ int prefix_sums(int n, int *out, int *wave_sums, V v) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int carry = 0;
    for (int i0 = 0; i0 < n; i0 += 64 * NW) {
        const int i = i0 + tid, mine = i < n ? v(i) : 0;
        int sum = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(sum, off, 64);
            if (lane >= off) sum += up;
        }
        if (lane == 63) wave_sums[w] = sum;
        __syncthreads();
        int before = carry;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            before += k < w ? wave_sums[k] : 0;
            carry += wave_sums[k];
        }
        if (i < n) out[i] = before + sum - mine;
        __syncthreads();
    }
    return carry;
}

// Sum of v over the lanes up to each one (all 64 active).
__device__ __forceinline__ int lane_sums(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);               // from 1, 2, 4 and 8 lanes before, within 16 lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);              // lane 15 to the 16 lanes behind it, lane 47 likewise
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);              // lane 31 to the 32 lanes behind it
    return v;
}

template <int KV> __device__ __forceinline__ int k_page_index(int pib, int d) {
    if constexpr (KV == KV_BF16) return (int)k_cache_index(pib, d);
    return (((((pib >> 4) * 2 + (d >> 6)) * 4 + ((d & 31) >> 3)) * 16 + (pib & 15)) * 2 + ((d >> 5) & 1)) * 8 + (d & 7);
}
template <int KV> __device__ __forceinline__ int v_page_index(int pib, int d) {
    if constexpr (KV == KV_BF16) return (int)v_cache_index(pib, d);
    const int o = pib & 15;
    return ((((d >> 5) * 4 + (o >> 2)) * 16 + (d & 15)) * 2 + ((d >> 4) & 1)) * 8 + (o & 3) + ((pib >> 4) << 2);
}

// four fp32 -> four e4m3 codes (round to nearest even, saturating; not a number stays none), value i in byte i
__device__ __forceinline__ unsigned int floats_to_e4m3x4(float a, float b, float c, float d) {
    auto sat = [](float x) { return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -kE4m3Max), kE4m3Max); };
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
    return (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), r, true);
}

// eight e4m3 codes -> eight bf16, exactly (four significant bits; the smallest is 2^-9)
__device__ __forceinline__ u32x4 e4m3x8_to_bf16(unsigned int lo, unsigned int hi) {
    u32x4 r;
    r.x = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r.y = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r.z = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r.w = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return r;
}

// ---- softmax in the 32 x 32 x 16 products' layout: a lane owns a query column, lanes l and l ^ 32 share it
typedef float f32x16 __attribute__((ext_vector_type(16)));
// Scores may pass the running maximum by this much (in powers of two) before sums and outputs are scaled down: p up to 2^8 costs neither
// product nor sum any precision.
constexpr float kLazyMax = 8.f;

// The maximum that hands a NaN on: one instruction, also of three operands (fmaxf has every operand made quiet first).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// the larger of lanes l and l ^ 32
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Weights and values meet in the second product in 16 bits.  bf16 pages: bf16, the weights rounded to 8 significant bits.  e4m3 pages: fp16, which
// holds their values exactly and the weights to 11 bits; weights are scaled by 2^7 there, so that with kLazyMax they end at 2^15 and what
// is lost below the smallest fp16, 2^-24, is 2^-31 of the largest.  (Sums carry the same factor: it cancels.)
template <int KV> constexpr float kWeightShift = KV == KV_E4M3 ? 7.f : 0.f;
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int KV> __device__ __forceinline__ unsigned int weight_pair(float lo, float hi) {
    if constexpr (KV == KV_BF16) return float2_to_bf16_pair(lo, hi);
    else return __builtin_bit_cast(unsigned int, __builtin_convertvector(f32x2{lo, hi}, f16x2));
}
// sum + both weights of a pair, in fp32: sums are taken of the rounded weights, so that the weights that are applied sum to one
template <int KV> __device__ __forceinline__ float add_pair(unsigned int pair, float sum) {
    if constexpr (KV == KV_BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
    else return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), f16x2{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
}
// eight e4m3 codes -> eight fp16, exactly
__device__ __forceinline__ u32x4 e4m3x8_to_f16(unsigned int lo, unsigned int hi) {
    u32x4 r;
    r.x = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
    r.y = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
    r.z = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
    r.w = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    return r;
}
// A value that is not finite, at a position that some rows of a product see and others do not, would reach those others as 0 x inf: it is
// taken out of the product, and the rows that see it get a NaN for their sum.
template <int KV> __device__ __forceinline__ unsigned int nonfinite_halves(unsigned int x) {      // bits 15 and 31
    return KV == KV_BF16 ? ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u : ((x & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
}
template <int KV> __device__ __forceinline__ bool any_nonfinite(const u32x4 v) {                  // of the wave
    const unsigned int bad = nonfinite_halves<KV>(v.x) | nonfinite_halves<KV>(v.y) | nonfinite_halves<KV>(v.z) | nonfinite_halves<KV>(v.w);
    return __builtin_amdgcn_ballot_w64(bad != 0) != 0ull;
}
// Clears them; the first position that had one, of the wave.  `first`: of the lane's slot 0; slots 4 .. 7 are 16 further on.
template <int KV> __device__ __forceinline__ int drop_nonfinite(u32x4 &v, int first) {
    int at = kMaxPositions * 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned int bad = nonfinite_halves<KV>(v[j]);
        const int pos = first + 16 * (j >> 1) + 2 * (j & 1);
        if (bad & 0x80000000u) { v[j] &= 0x0000FFFFu; at = min(at, pos + 1); }
        if (bad & 0x00008000u) { v[j] &= 0xFFFF0000u; at = min(at, pos); }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) at = min(at, __shfl_xor(at, off, 64));
    return at;
}

// The same where a row may see a later position and not an earlier one: clears them, and says which positions of the block of 32 had one, of the wave.
// `first`: the lane's slot 0 in the block.
template <int KV> __device__ __forceinline__ unsigned int drop_nonfinite_of_block(u32x4 &v, int first) {
    unsigned int at = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned int bad = nonfinite_halves<KV>(v[j]);
        const int pos = first + 16 * (j >> 1) + 2 * (j & 1);
        if (bad & 0x80000000u) { v[j] &= 0x0000FFFFu; at |= 2u << pos; }
        if (bad & 0x00008000u) { v[j] &= 0xFFFF0000u; at |= 1u << pos; }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) at |= __shfl_xor(at, off, 64);
    return at;
}

template <int KV> __device__ __forceinline__ f32x16 values_times_weights(const u32x4 v, const u32x4 w, const f32x16 acc) {
    if constexpr (KV == KV_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, w), acc, 0, 0, 0);
}
template <int KV> __device__ __forceinline__ f32x4 values_times_weights(const u32x4 v, const u32x4 w, const f32x4 acc) {
    if constexpr (KV == KV_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, w), acc, 0, 0, 0);
}

// ---------------------------------------------------------------------------------------------
// Append: per head of a new row RMSNorm and rotary embedding (queries and keys), queries to q_out, keys and values to the
// page of the row's position.
// ---------------------------------------------------------------------------------------------
struct PrepareParams {
    PagedParams c;
    const uint16_t *qkv, *q_gamma, *k_gamma;
    uint16_t *q_out;
    long long ld, ldq;
    float eps;
    double log2_theta;
    int parts;                // waves that share a row's heads; heads of a workgroup in the block form
    // forms other than ROPE_THETA
    const double *inv_freq;   // [dims / 2] radians a position
    float magnitude;          // of cosines and sines
    int dims;                 // of a head, from its first on, that are rotated: a multiple of 16
};

// How a head is rotated.  ROPE_THETA: all of it, pairs d and d + 64, angles from theta, behind the norm.  The others: pairs d and d + dims / 2
// (ROPE_HALF) or 2 d and 2 d + 1 (ROPE_PAIRS) of the first `dims`, angles from a table, behind the norm or without one (gammas NULL).
enum { ROPE_THETA = 0, ROPE_HALF = 1, ROPE_PAIRS = 2 };

// What a lane does with its eight elements of a head, d = 8 j .. 8 j + 7, of lanes 16 h + j: the norm, with its two roundings to bf16 ...
__device__ __forceinline__ u32x4 normed(const u32x4 raw, const u32x4 graw, float eps) {
    float x[8];
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(raw[e] << 16);
        x[2 * e + 1] = __uint_as_float(raw[e] & 0xFFFF0000u);
    }
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, (float)kHeadDim) + eps));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned int n = float2_to_bf16_pair(x[2 * e] * r, x[2 * e + 1] * r);
        out[e] = float2_to_bf16_pair(__uint_as_float(n << 16) * __uint_as_float(graw[e] << 16),
                                     __uint_as_float(n & 0xFFFF0000u) * __uint_as_float(graw[e] & 0xFFFF0000u));
    }
    return out;
}

// ... then the rotation of the first `turned` = dims / 8 lanes' elements, others as they are.  ROPE_HALF: the partner (d +- dims / 2) is turned / 2 lanes
// away and sinv negative in the first half (x1 cos - x2 sin); ROPE_PAIRS: both are in one word, whose angle is cosv[e], sinv[e] of word e.
template <int ROPE>
__device__ __forceinline__ u32x4 rotated(const u32x4 x, int turned, const float (&cosv)[8], const float (&sinv)[8]) {
    const int lane = threadIdx.x & 63, j = lane & 15;
    u32x4 out;
    if constexpr (ROPE == ROPE_HALF) {
        const int partner = (lane & 48) + (j < turned / 2 ? j + turned / 2 : j < turned ? j - turned / 2 : j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned int other = __shfl(x[e], partner, 64);
            out[e] = float2_to_bf16_pair(__uint_as_float(x[e] << 16) * cosv[2 * e] + __uint_as_float(other << 16) * sinv[2 * e],
                                         __uint_as_float(x[e] & 0xFFFF0000u) * cosv[2 * e + 1] + __uint_as_float(other & 0xFFFF0000u) * sinv[2 * e + 1]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = __uint_as_float(x[e] << 16), b = __uint_as_float(x[e] & 0xFFFF0000u);
            out[e] = float2_to_bf16_pair(a * cosv[e] - b * sinv[e], b * cosv[e] + a * sinv[e]);
        }
    }
    return j < turned ? out : x;
}
// Which angle of the table a lane's element e takes (word e in ROPE_PAIRS); lanes that are not turned take any.
template <int ROPE> __device__ __forceinline__ int angle_of(int j, int e, int turned) {
    return ROPE == ROPE_HALF ? (8 * (j < turned / 2 ? j : j - turned / 2) + e) & 63 : (4 * j + e) & 63;
}

// The norm and the rotation in one: the rotary partner (d +- 64) is lane j ^ 8.  sinv is negative in the first half (x1 cos - x2 sin).
__device__ __forceinline__ u32x4 norm_and_rotate(const u32x4 raw, const u32x4 graw, float eps, const float (&cosv)[8], const float (&sinv)[8]) {
    float x[8], o[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(raw[e] << 16);
        x[2 * e + 1] = __uint_as_float(raw[e] & 0xFFFF0000u);
    }
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, (float)kHeadDim) + eps));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned int n = float2_to_bf16_pair(x[2 * e] * r, x[2 * e + 1] * r);
        const unsigned int g = float2_to_bf16_pair(__uint_as_float(n << 16) * __uint_as_float(graw[e] << 16),
                                                   __uint_as_float(n & 0xFFFF0000u) * __uint_as_float(graw[e] & 0xFFFF0000u));
        const unsigned int other = __shfl_xor(g, 8, 64);
        o[2 * e] = __uint_as_float(g << 16) * cosv[2 * e] + __uint_as_float(other << 16) * sinv[2 * e];
        o[2 * e + 1] = __uint_as_float(g & 0xFFFF0000u) * cosv[2 * e + 1] + __uint_as_float(other & 0xFFFF0000u) * sinv[2 * e + 1];
    }
    return u32x4{float2_to_bf16_pair(o[0], o[1]), float2_to_bf16_pair(o[2], o[3]), float2_to_bf16_pair(o[4], o[5]), float2_to_bf16_pair(o[6], o[7])};
}

// x / scale to nearest, where that makes a difference to the code; inv: 1 / scale, to nearest.  Two steps of q + (x - q scale) inv: after the first q is
// one of the two neighbours of the quotient, x - q scale is then exact, and with a correctly rounded inverse the second gives the nearest
// (Markstein's theorem).  Not for scales or quotients whose remainder could leave the normal range: below 2^-11 the code is a zero of x's sign,
// beyond 2^20 the largest, by the first product already.  Fewer instructions than a division: 11 prompts of up to 1531 rows 57.7 us, and 61.3 on the same card.
__device__ __forceinline__ float quotient_of_code(float x, float scale, float inv) {
    const float q0 = x * inv, q1 = __builtin_fmaf(__builtin_fmaf(-q0, scale, x), inv, q0);
    const float q2 = __builtin_fmaf(__builtin_fmaf(-q1, scale, x), inv, q1);
    return fabsf(q0) > 0x1p-11f && fabsf(q0) < 0x1p20f ? q2 : q0;
}
// eight bf16 -> eight codes of value / scale
__device__ __forceinline__ u32x2 e4m3_codes(const u32x4 v, float scale) {
    float f[8];
    if (scale > 0x1p-60f && scale < 0x1p60f) {
        const float inv = __fdiv_rn(1.0f, scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = quotient_of_code(__uint_as_float(v[e] << 16), scale, inv);
            f[2 * e + 1] = quotient_of_code(__uint_as_float(v[e] & 0xFFFF0000u), scale, inv);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = __fdiv_rn(__uint_as_float(v[e] << 16), scale);
            f[2 * e + 1] = __fdiv_rn(__uint_as_float(v[e] & 0xFFFF0000u), scale);
        }
    }
    return u32x2{floats_to_e4m3x4(f[0], f[1], f[2], f[3]), floats_to_e4m3x4(f[4], f[5], f[6], f[7])};
}

// theta^(-2 i / 128) / 2 pi: an angle in turns, reduced in double by rotation(): positions reach tens of thousands of radians
__device__ __forceinline__ double turns_per_position(double log2_theta, int i) { return exp2(-(2.0 * i / kHeadDim) * log2_theta) * 0.15915494309189535; }
__device__ __forceinline__ void rotation(int pos, double per_position, float &sn, float &cs) {
    const double turns = (double)pos * per_position;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
}

// Turns a position of the angle that a lane has in hand, 0 where there are fewer.
template <int ROPE> __device__ __forceinline__ double turns_of_lane(const PrepareParams &p, int lane) {
    if constexpr (ROPE == ROPE_THETA) return turns_per_position(p.log2_theta, lane);
    return lane < p.dims / 2 ? p.inv_freq[lane] * 0.15915494309189535 : 0.0;
}

// For few rows a sequence: a wave takes four heads of a row at a time, 16 lanes of 16 bytes each.  Bound by the launch and one trip to memory: one row of
// one sequence 5 us a call, 3.6 in the kernel; of another rotation the same.
template <int KV, int ROPE>
__global__ __launch_bounds__(256) void paged_prepare_kernel(const PrepareParams p) {
    const PagedParams &c = p.c;
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(unit / p.parts), part = (int)(unit % p.parts);
    if (t >= c.T) return;
    const int s = seq_of_row(c, t, lane);
    if (s < 0) return;
    const SeqSpan sp = seq_span(c, s);
    if (t < sp.row0 || t >= sp.row0 + sp.n) return;
    const int pos = sp.len + t - sp.row0;
    const int j = lane & 15;
    float sn, cs;
    rotation(pos, turns_of_lane<ROPE>(p, lane), sn, cs);
    float cosv[8], sinv[8];
    const int turned = ROPE == ROPE_THETA ? 16 : p.dims / 8;
    if constexpr (ROPE == ROPE_THETA) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cosv[e] = __shfl(cs, 8 * (j & 7) + e, 64);
            sinv[e] = __shfl(sn, 8 * (j & 7) + e, 64);
            if (j < 8) sinv[e] = -sinv[e];
        }
    } else {
        cs *= p.magnitude;
        sn *= p.magnitude;
#pragma unroll
        for (int e = 0; e < (ROPE == ROPE_HALF ? 8 : 4); ++e) {
            cosv[e] = __shfl(cs, angle_of<ROPE>(j, e, turned), 64);
            sinv[e] = __shfl(sn, angle_of<ROPE>(j, e, turned), 64);
            if (ROPE == ROPE_HALF && j < turned / 2) sinv[e] = -sinv[e];
        }
    }
    const int blk = pos / kKvBlock, pib = pos % kKvBlock, col = blk >> c.block_shift;
    const int page = col < c.columns ? c.table[s * c.table_ld + col] : -1;
    const bool stored = page_exists(page, c.n_pages);
    constexpr int BB = kv_block_bytes<KV>;
    const long long base = stored ? ((((long long)page * c.Hkv) << c.block_shift) + (blk & ((1 << c.block_shift) - 1))) * (2 * BB) : 0;
    const long long head_step = (long long)(2 * BB) << c.block_shift;
    const int heads = c.Hq + 2 * c.Hkv;
    for (int h = 4 * part + (lane >> 4); h < ((heads + 3) & ~3); h += 4 * p.parts) {
        const bool live = h < heads;
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (live) raw = *reinterpret_cast<const u32x4 *>(p.qkv + t * p.ld + (long long)h * kHeadDim + 8 * j);
        u32x4 done;                                                              // (all lanes: they exchange)
        if constexpr (ROPE == ROPE_THETA) {
            const u32x4 graw = *reinterpret_cast<const u32x4 *>((h < c.Hq ? p.q_gamma : p.k_gamma) + 8 * j);
            done = norm_and_rotate(raw, graw, p.eps, cosv, sinv);
        } else {
            done = raw;
            if (p.q_gamma) done = normed(raw, *reinterpret_cast<const u32x4 *>((h < c.Hq ? p.q_gamma : p.k_gamma) + 8 * j), p.eps);
            done = rotated<ROPE>(done, turned, cosv, sinv);
        }
        if (!live) continue;
        const bool value = h >= c.Hq + c.Hkv;
        const u32x4 rounded = value ? raw : done;                                // (values are stored as they are)
        if (h < c.Hq) {
            *reinterpret_cast<u32x4 *>(p.q_out + t * p.ldq + (long long)h * kHeadDim + 8 * j) = rounded;
            continue;
        }
        if (!stored) continue;
        const int hk = value ? h - c.Hq - c.Hkv : h - c.Hq;
        unsigned char *dst = c.pages + base + hk * head_step + (value ? BB : 0);
        if constexpr (KV == KV_BF16) {
            if (!value) {
                *reinterpret_cast<u32x4 *>(dst + 2 * k_page_index<KV>(pib, 8 * j)) = rounded;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    *reinterpret_cast<uint16_t *>(dst + 2 * v_page_index<KV>(pib, 8 * j + e)) = (uint16_t)(rounded[e >> 1] >> (16 * (e & 1)));
            }
        } else {
            const float *scale = value ? c.v_scale : c.k_scale;
            const u32x2 codes = e4m3_codes(rounded, scale ? scale[hk] : 1.0f);
            if (!value) {
                *reinterpret_cast<u32x2 *>(dst + k_page_index<KV>(pib, 8 * j)) = codes;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[v_page_index<KV>(pib, 8 * j + e)] = (unsigned char)(codes[e >> 2] >> (8 * (e & 3)));
            }
        }
    }
}

// For many rows a sequence: a workgroup takes the new rows of one block of 32 positions and p.parts heads.  The rotations of
// the block are computed once, in LDS; a value head goes through LDS too, since its 16-byte units hold eight positions of one d: written
// one by one they cost 2 bytes of every 16 a store.  11 prompts of up to 1531 rows into 8-bit pages (229 MB moved): 57 to 60 us, 4 TB/s where a
// plain copy reaches 5.15; what is left is the norms and rotations, two trips through memory a workgroup.  Rotations of a part of the head 62.
template <int KV, int ROPE>
__global__ __launch_bounds__(256) void paged_prepare_block_kernel(const PrepareParams p) {
    constexpr int BB = kv_block_bytes<KV>, STRIDE = kHeadDim + 8;                // (of a row of the values in LDS)
    __shared__ float2 turned[kKvBlock][kHeadDim / 2];
    __shared__ __align__(16) uint16_t rows[2][kKvBlock][STRIDE];
    __shared__ int prefix[kMaxSeqs];
    __shared__ int wave_sums[4];
    const PagedParams &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63, j = tid & 15, r0 = tid >> 4;
    const double per_position = turns_of_lane<ROPE>(p, lane);
    const int turned_lanes = ROPE == ROPE_THETA ? 16 : p.dims / 8;

    auto blocks_with_rows = [&](int s) {
        const SeqSpan a = seq_span(c, s);
        return a.n ? (a.len + a.n - 1) / kKvBlock - a.len / kKvBlock + 1 : 0;
    };
    const int units = prefix_sums<4>(c.n_seqs, prefix, wave_sums, blocks_with_rows);
    const int u = blockIdx.x;
    if (u >= units) return;
    int s = 0;
    for (int up = c.n_seqs; up - s > 1;) {
        const int mid = (s + up) >> 1;
        if (prefix[mid] <= u) s = mid; else up = mid;
    }
    const SeqSpan a = seq_span(c, s);
    const int blk = a.len / kKvBlock + u - prefix[s], pos0 = blk * kKvBlock, column = blk >> c.block_shift;
    const int lo = a.len - pos0, hi = a.len + a.n - pos0;                        // rows lo .. hi - 1 of the block are new
    const int page = column < c.columns ? c.table[s * c.table_ld + column] : -1;
    const bool stored = page_exists(page, c.n_pages);
    const long long base = stored ? ((((long long)page * c.Hkv) << c.block_shift) + (blk & ((1 << c.block_shift) - 1))) * (2 * BB) : 0;
    const long long head_step = (long long)(2 * BB) << c.block_shift;
    const int h0 = blockIdx.y * p.parts, h1 = min(h0 + p.parts, c.Hq + 2 * c.Hkv);
    auto is_new = [&](int r) { return r >= lo && r < hi; };
    auto row_of = [&](int r) { return (long long)(a.row0 + pos0 + r - a.len); };
    auto load = [&](int h, int i) {
        const int r = r0 + 16 * i;
        return is_new(r) ? *reinterpret_cast<const u32x4 *>(p.qkv + row_of(r) * p.ld + (long long)h * kHeadDim + 8 * j) : u32x4{0u, 0u, 0u, 0u};
    };
    u32x4 x[2] = {load(h0, 0), load(h0, 1)};
    float cosv[2][8], sinv[2][8];
    if (h0 < c.Hq + c.Hkv) {
        for (int r = tid >> 6; r < kKvBlock; r += 4) {
            float sn, cs;
            rotation(pos0 + r, per_position, sn, cs);
            turned[r][lane] = ROPE == ROPE_THETA ? float2{cs, sn} : float2{cs * p.magnitude, sn * p.magnitude};
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < (ROPE == ROPE_PAIRS ? 4 : 8); ++e) {
                const float2 v = turned[r0 + 16 * i][ROPE == ROPE_THETA ? 8 * (j & 7) + e : angle_of<ROPE>(j, e, turned_lanes)];
                cosv[i][e] = v.x;
                sinv[i][e] = ROPE != ROPE_PAIRS && j < turned_lanes / 2 ? -v.y : v.y;
            }
    }
    for (int h = h0; h < h1; ++h) {
        u32x4 next[2];
        if (h + 1 < h1) { next[0] = load(h + 1, 0); next[1] = load(h + 1, 1); }
        if (h < c.Hq + c.Hkv) {
            u32x4 graw = {0u, 0u, 0u, 0u};
            if (ROPE == ROPE_THETA || p.q_gamma) graw = *reinterpret_cast<const u32x4 *>((h < c.Hq ? p.q_gamma : p.k_gamma) + 8 * j);
            const float sc = KV == KV_E4M3 && h >= c.Hq && c.k_scale ? c.k_scale[h - c.Hq] : 1.0f;
            unsigned char *dst = c.pages + base + (h - c.Hq) * head_step;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + 16 * i;
                u32x4 o = x[i];
                if constexpr (ROPE == ROPE_THETA) {
                    o = norm_and_rotate(o, graw, p.eps, cosv[i], sinv[i]);
                } else {
                    if (p.q_gamma) o = normed(o, graw, p.eps);
                    o = rotated<ROPE>(o, turned_lanes, cosv[i], sinv[i]);
                }
                if (!is_new(r)) continue;
                if (h < c.Hq) *reinterpret_cast<u32x4 *>(p.q_out + row_of(r) * p.ldq + (long long)h * kHeadDim + 8 * j) = o;
                else if (!stored) continue;
                else if constexpr (KV == KV_BF16) *reinterpret_cast<u32x4 *>(dst + 2 * k_page_index<KV>(r, 8 * j)) = o;
                else *reinterpret_cast<u32x2 *>(dst + k_page_index<KV>(r, 8 * j)) = e4m3_codes(o, sc);
            }
        } else {
            const int hk = h - c.Hq - c.Hkv, buf = h & 1;                        // (two buffers: a barrier a head is enough)
#pragma unroll
            for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4 *>(&rows[buf][r0 + 16 * i][8 * j]) = x[i];
            __syncthreads();
            const float sc = KV == KV_E4M3 && c.v_scale ? c.v_scale[hk] : 1.0f;
            unsigned char *dst = c.pages + base + hk * head_step + BB;
            if (stored)
                for (int i = 0; i < 2; ++i) {
                    // unit (d, g4): positions 4 g4 .. + 3 and 16 + 4 g4 .. + 3 of one d
                    const int at = tid + 256 * i, d = (at >> 6) * 16 + (at & 15), g4 = (at >> 4) & 3;
                    u32x4 v;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int pos = 4 * g4 + 2 * (k & 1) + 16 * (k >> 1);
                        v[k] = rows[buf][pos][d] | (unsigned int)rows[buf][pos + 1][d] << 16;
                    }
                    const u32x2 codes = KV == KV_E4M3 ? e4m3_codes(v, sc) : u32x2{0u, 0u};
                    unsigned char *to = dst + (KV == KV_E4M3 ? 1 : 2) * v_page_index<KV>(4 * g4, d);
                    if (lo <= 0 && hi >= kKvBlock) {
                        if constexpr (KV == KV_BF16) *reinterpret_cast<u32x4 *>(to) = v;
                        else *reinterpret_cast<u32x2 *>(to) = codes;
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if (!is_new(4 * g4 + (k & 3) + 16 * (k >> 2))) continue;
                            if constexpr (KV == KV_BF16) *reinterpret_cast<uint16_t *>(to + 2 * k) = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
                            else to[k] = (unsigned char)(codes[k >> 2] >> (8 * (k & 3)));
                        }
                    }
                }
        }
        x[0] = next[0];
        x[1] = next[1];
    }
}

}  // namespace quasar
