// Causal attention of whole prompts, or chunks of them, over a paged key/value cache (gfx950): many rows per sequence.
//
// Rows are r = m * G + g: the G query heads of a key/value head side by side, so that a tile of rows covers few tokens
// (a narrow causal edge) and shares every key and value it loads.  A workgroup of NW waves takes 32 * NW rows of one kv head; the
// waves share tiles of 64 positions in LDS, loaded straight from the pages, two tiles in turn.
//
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 products: a lane owns one query column.  The
// rows of K are permuted, row 16 t + 8 c + 4 h + b of the product being position 16 c + 8 t + 4 h + b, which makes the scores that a lane
// holds after the first product the operand of the second as they lie, against values in the cache's own order.
#pragma once

#include <type_traits>

#include "paged.hpp"

namespace quasar {

struct PromptParams {
    PagedParams c;
    const uint16_t *q;        // [T, Hq * 128] bf16
    uint16_t *out;
    long long ldq, ldo;
    float scale_log2;         // log2(e) / sqrt(128)
};

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kPromptStep = 64;                          // positions in LDS at a time
constexpr int kPromptStepBytes = kPromptStep / kKvBlock * 2 * kKvBlockBytes;   // 32 KB: two blocks, keys and values
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

template <int KV, int NW>
__global__ __launch_bounds__(NW * 64) void prompt_attention_kernel(const PromptParams p) {
    constexpr int ROWS = 32 * NW;
    extern __shared__ __align__(16) unsigned char lds[];         // [2 steps][2 blocks][keys | values][8192], then the prefix sums
    int *prefix = reinterpret_cast<int *>(lds + 2 * kPromptStepBytes);   // [n_seqs + 1]
    int *wave_sums = prefix + kMaxSeqs + 1;
    int *there = wave_sums + NW;                                 // [step parity][block]: the block has a page
    const PagedParams &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hi = lane >> 5, col = lane & 31;
    const int h = blockIdx.x % c.Hkv;

    // row tiles of the sequences, prefix sums
    int tiles = 0;
    for (int s0 = 0; s0 < c.n_seqs; s0 += 64 * NW) {
        const int s = s0 + tid;
        int mine = 0;
        if (s < c.n_seqs) mine = (int)(((long long)seq_span(c, s).n * c.G + ROWS - 1) / ROWS);
        int sum = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(sum, off, 64);
            if (lane >= off) sum += up;
        }
        if (lane == 63) wave_sums[w] = sum;
        __syncthreads();
        int before = tiles;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            before += i < w ? wave_sums[i] : 0;
            tiles += wave_sums[i];
        }
        if (s < c.n_seqs) prefix[s] = before + sum - mine;
        __syncthreads();
    }
    // the last tiles, which see most, first
    const int f = tiles - 1 - (int)(blockIdx.x / c.Hkv);
    if (f < 0) return;
    int s = 0;
    {
        int up = c.n_seqs;
        while (up - s > 1) {
            const int mid = (s + up) >> 1;
            if (prefix[mid] <= f) s = mid; else up = mid;
        }
    }
    const SeqSpan a = seq_span(c, s);
    const int R = a.n * c.G, tile0 = (f - prefix[s]) * ROWS;
    const float ks = c.k_scale ? c.k_scale[h] : 1.0f, vs = c.v_scale ? c.v_scale[h] : 1.0f;
    const float scale_log2 = p.scale_log2 * ks;

    const int my_row = tile0 + w * 32 + col;
    const int row = min(my_row, R - 1);                          // (rows behind the last one repeat it and are not stored)
    const int token = row / c.G;
    const int limit = a.len + token;                             // last visible position of the lane's column
    const long long head_at = ((long long)h * c.G + row % c.G) * kHeadDim;
    bf16x8 qb[8];                                                // lane (column, hi) holds d = 16 k + 8 hi .. + 7
#pragma unroll
    for (int k = 0; k < 8; ++k)
        qb[k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p.q + (a.row0 + token) * p.ldq + head_at + 16 * k + 8 * hi));
    const int first_pos = a.len + tile0 / c.G;                   // positions up to here are visible to every row of the tile
    const int last_pos = a.len + (min(tile0 + ROWS, R) - 1) / c.G;
    const int nblk = blocks_of(c, last_pos + 1);
    const int steps = (nblk + 1) / 2;

    // ---- staging: the waves share the keys and values of the two blocks of a step in equal parts
    constexpr int BB = kv_block_bytes<KV>, PART = 4 * BB / NW, NL = PART / 1024;   // bytes and 16-byte loads a lane of a wave
    static_assert(PART <= BB && NL >= 1, "a wave's part lies in one block's keys or values");
    const int my_blk = w / (NW / 2), my_at = w * PART - my_blk * 2 * BB;         // (keys, then values, of a block are contiguous)
    const long long head_step = (long long)(2 * BB) << c.block_shift, page_step = head_step * c.Hkv;
    const int in_page = (1 << c.block_shift) - 1;
    const int32_t *pages_of = c.table + s * c.table_ld;
    const unsigned char *head = c.pages + h * head_step + my_at;
    int ids = -1, ids_at = -64;                                  // pages of steps ids_at .. + 63, one a lane
    u32x4 code[NL];
    auto request = [&](int step) {
        const int stage = step & 1;
        if (step >= ids_at + 64 || ids_at < 0) {
            ids_at = step;
            const int b = 2 * (step + lane) + my_blk;
            ids = b < nblk ? pages_of[b >> c.block_shift] : -1;
        }
        const int page = __builtin_amdgcn_readlane(ids, step - ids_at);
        const bool good = page_exists(page, c.n_pages);
        if (my_at == 0 && lane == 0) there[2 * stage + my_blk] = good;
        const unsigned char *from = head + (good ? page : 0) * page_step + ((2 * step + my_blk) & in_page) * (2 * BB);
        if constexpr (KV == KV_BF16) {
            const unsigned int to = lds_address_of(lds) + stage * kPromptStepBytes + w * PART;
#pragma unroll
            for (int i = 0; i < NL; ++i) load_to_lds_16(reinterpret_cast<unsigned long long>(from) + 1024 * i, 16 * lane, to + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) code[i] = reinterpret_cast<const u32x4 *>(from)[64 * i + lane];
        }
    };
    // what request() asked for is in LDS afterwards (for this wave; the others' behind a barrier)
    auto settle = [&](int stage) {
        if constexpr (KV == KV_BF16) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            u32x4 *to = reinterpret_cast<u32x4 *>(lds + stage * kPromptStepBytes + w * 2 * PART) + lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                to[64 * (2 * i)] = e4m3x8_to_bf16(code[i].x, code[i].y);
                to[64 * (2 * i + 1)] = e4m3x8_to_bf16(code[i].z, code[i].w);
            }
        }
    };

    f32x16 oacc[4];
    float mrow = -__builtin_inff(), lrow = 0.f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
    // this lane's place in a block: row col of the keys, d = col of the values
    const int k_lane = (((col >> 3) & 1) * 16 * 16 + ((col >> 4) * 8 + (col & 7)) + 16 * hi) * 16;   // [sub 2][kstep 4][g4 4][p 16] of 16 bytes
    const int v_lane = ((col >> 4) * 64 + (col & 15) + 16 * hi) * 16;                             // [dt 8][g4 4][dd 16] of 16 bytes

    // the 64 positions of a step; edge: some are hidden from some row, or are nobody's; between(): called while the scores are computed
    auto attend = [&](auto edge, int step, bool there0, bool there1, auto between) {
        constexpr bool EDGE = decltype(edge)::value;
        const unsigned char *buf = lds + (step & 1) * kPromptStepBytes;
        const int pos0 = step * kPromptStep;
        f32x16 sc[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[blk][i] = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(buf + blk * 2 * kKvBlockBytes + k_lane + k * 512);
                sc[blk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[k], sc[blk], 0, 0, 0);
            }
        if constexpr (EDGE) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                // register 4 (2 t + c) + b: position 16 c + 8 t + 4 hi + b
                const int left = (blk ? there1 : there0) ? limit - pos0 - 32 * blk - 4 * hi : -1;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (16 * ((i >> 2) & 1) + 8 * (i >> 3) + (i & 3) > left) sc[blk][i] = -__builtin_inff();
            }
        }
        between();                                               // (dozens of scalar instructions: while the products are under way)
        u32x4 v0[2][4];                                          // the first values, ahead of the softmax: its exponentials cover the way
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) v0[t][dt] = *reinterpret_cast<const u32x4 *>(buf + kKvBlockBytes + v_lane + dt * 2048 + t * 512);
        float mx = larger(sc[0][0], sc[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = larger(mx, larger(sc[0][i], sc[1][i]));
        mx = max_halves(mx);
        if (__builtin_amdgcn_ballot_w64((mx - mrow) * scale_log2 > kLazyMax) != 0ull) {          // (the first visible score, too)
            const float m_new = larger(mrow, mx);
            const float alpha = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((mrow - m_new) * scale_log2);
            mrow = m_new;
            lrow *= alpha;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) oacc[dt] *= alpha;
        }
        const float mc = mrow == -__builtin_inff() ? 0.f : -mrow * scale_log2;
        u32x4 pb[2][2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[blk][2 * i], scale_log2, mc));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[blk][2 * i + 1], scale_log2, mc));
                const unsigned int pk = float2_to_bf16_pair(e0, e1);
                pb[blk][i >> 2][i & 3] = pk;
                // the sum of the rounded values, so that the weights that are applied sum to one
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                lrow = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), __builtin_bit_cast(bf16x2, 0x3F803F80u), lrow, false);
            }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    u32x4 va = blk == 0 ? v0[t][dt] : *reinterpret_cast<const u32x4 *>(buf + (2 * blk + 1) * kKvBlockBytes + v_lane + dt * 2048 + t * 512);
                    if constexpr (EDGE) {
                        // positions that no row sees hold whatever the page held: they must not reach the product (0 x NaN)
                        const int end = (blk ? there1 : there0) ? last_pos - pos0 - 32 * blk - 4 * (2 * t + hi) : -1;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int at = 16 * (j >> 1) + 2 * (j & 1);
                            va[j] &= (at <= end ? 0x0000FFFFu : 0u) | (at + 1 <= end ? 0xFFFF0000u : 0u);
                        }
                    }
                    oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va), __builtin_bit_cast(bf16x8, pb[blk][t]), oacc[dt], 0, 0, 0);
                }
    };
    // The steps that every row sees whole, then the others (and all from the first that lacks a page on): two loops, since the outputs'
    // registers would be copied once a step where the two ways met.
    const int whole = min((first_pos + 1) / kPromptStep, steps);
    int step = 0;
    bool settled = false;
    auto arrive = [&] {
        settle(step & 1);
        lds_barrier();
    };
    auto request_next = [&] {
        if (step + 1 < steps) request(step + 1);
    };
    if (steps > 0) request(0);
    for (; step < whole; step = step + 1) {
        arrive();
        settled = !(there[2 * (step & 1)] && there[2 * (step & 1) + 1]);
        if (settled) break;
        attend(std::false_type{}, step, true, true, request_next);
    }
    for (; step < steps; step = step + 1) {
        if (!settled) arrive();
        settled = false;
        const bool there0 = there[2 * (step & 1)], there1 = there[2 * (step & 1) + 1];
        attend(std::true_type{}, step, there0, there1, request_next);
    }
    float sum = lrow + __shfl_xor(lrow, 32, 64);
    const float inv = sum > 0.f ? __fdiv_rn(vs, sum) : 0.f;      // a row that sees nothing: zeros
    if (my_row >= R) return;
    uint16_t *to = p.out + (a.row0 + token) * p.ldo + head_at + 4 * hi;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {                            // registers 4 i .. + 3: d = 32 dt + 8 i + 4 hi ..
            const u32x2 o = {float2_to_bf16_pair(oacc[dt][4 * i] * inv, oacc[dt][4 * i + 1] * inv),
                             float2_to_bf16_pair(oacc[dt][4 * i + 2] * inv, oacc[dt][4 * i + 3] * inv)};
            *reinterpret_cast<u32x2 *>(to + 32 * dt + 8 * i) = o;
        }
}

}  // namespace quasar
