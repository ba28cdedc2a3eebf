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
};

__device__ __forceinline__ SeqSpan seq_span(const PagedParams &p, int s) { return span_of(p.row_start[s], p.row_start[s + 1], p.lengths[s], p.T); }
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

template <int KV> __device__ __forceinline__ int k_page_index(int pib, int d) {
    if constexpr (KV == KV_BF16) return (int)k_cache_index(pib, d);
    return (((((pib >> 4) * 2 + (d >> 6)) * 4 + ((d & 31) >> 3)) * 16 + (pib & 15)) * 2 + ((d >> 5) & 1)) * 8 + (d & 7);
}
template <int KV> __device__ __forceinline__ int v_page_index(int pib, int d) {
    if constexpr (KV == KV_BF16) return (int)v_cache_index(pib, d);
    const int o = pib & 15;
    return ((((d >> 5) * 4 + (o >> 2)) * 16 + (d & 15)) * 2 + ((d >> 4) & 1)) * 8 + (o & 3) + ((pib >> 4) << 2);
}

// four fp32 -> four e4m3 codes (round to nearest even, saturating), value i in byte i
__device__ __forceinline__ unsigned int floats_to_e4m3x4(float a, float b, float c, float d) {
    auto sat = [](float x) { return __builtin_amdgcn_fmed3f(x, -kE4m3Max, kE4m3Max); };
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

// sum + both bf16 of a pair, in fp32: sums are taken of the rounded weights, so that the weights that are applied sum to one
__device__ __forceinline__ float add_bf16_pair(unsigned int pair, float sum) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
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
    int parts;                // waves that share a row's heads
};

// One wave takes four heads at a time, 16 lanes of 16 bytes each: lane 16 h + j holds d = 8 j .. 8 j + 7, its rotary partner
// (d +- 64) is lane j ^ 8.
template <int KV>
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
    // the angle in turns, reduced in double: positions reach tens of thousands of radians
    const int j = lane & 15;
    const double turns = (double)pos * exp2(-(2.0 * lane / kHeadDim) * p.log2_theta) * 0.15915494309189535;
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    float cosv[8], sinv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        cosv[e] = __shfl(cs, 8 * (j & 7) + e, 64);
        sinv[e] = __shfl(sn, 8 * (j & 7) + e, 64);
        if (j < 8) sinv[e] = -sinv[e];                       // first half: x1 cos - x2 sin
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
        const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, (float)kHeadDim) + p.eps));
        const u32x4 graw = *reinterpret_cast<const u32x4 *>((h < c.Hq ? p.q_gamma : p.k_gamma) + 8 * j);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float g = e & 1 ? __uint_as_float(graw[e >> 1] & 0xFFFF0000u) : __uint_as_float(graw[e >> 1] << 16);
            const float n = bf16_bits_to_float(float_to_bf16_bits(bf16_bits_to_float(float_to_bf16_bits(x[e] * r)) * g));
            const float other = __shfl_xor(n, 8, 64);
            o[e] = n * cosv[e] + other * sinv[e];
        }
        if (!live) continue;
        const bool value = h >= c.Hq + c.Hkv;
        u32x4 rounded = raw;                                    // (values are stored as they are)
        if (!value) {
#pragma unroll
            for (int e = 0; e < 4; ++e) rounded[e] = float2_to_bf16_pair(o[2 * e], o[2 * e + 1]);
        }
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
            const float sc = scale ? scale[hk] : 1.0f;
            float f[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[2 * e] = __fdiv_rn(__uint_as_float(rounded[e] << 16), sc);
                f[2 * e + 1] = __fdiv_rn(__uint_as_float(rounded[e] & 0xFFFF0000u), sc);
            }
            const u32x2 codes = {floats_to_e4m3x4(f[0], f[1], f[2], f[3]), floats_to_e4m3x4(f[4], f[5], f[6], f[7])};
            if (!value) {
                *reinterpret_cast<u32x2 *>(dst + k_page_index<KV>(pib, 8 * j)) = codes;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[v_page_index<KV>(pib, 8 * j + e)] = (unsigned char)(codes[e >> 2] >> (8 * (e & 3)));
            }
        }
    }
}

}  // namespace quasar
