// Causal attention of whole prompts, or chunks of them, over a paged key/value cache (gfx950): many rows per sequence.
//
// Rows are r = m * G + g: the G query heads of a key/value head side by side, so that a tile of rows covers few tokens
// (a narrow causal edge) and shares every key and value it loads.  A workgroup of four waves takes 128 * NT rows of one kv head; the
// waves share tiles of 64 positions in LDS, loaded straight from the pages, two tiles in turn.
//
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 products: a lane owns one query column of each of the wave's NT row tiles.  The
// rows of K are permuted, row 16 t + 8 c + 4 h + b of the product being position 16 c + 8 t + 4 h + b, which makes the scores that a lane
// holds after the first product the operand of the second as they lie, against values in the cache's own order.
#pragma once

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
constexpr int kPromptWaves = 4;
constexpr int kPromptStep = 64;                          // positions in LDS at a time
constexpr int kPromptStepBytes = kPromptStep / kKvBlock * 2 * kKvBlockBytes;   // 32 KB: two blocks, keys and values
// Scores may pass the running maximum by this much (in powers of two) before sums and outputs are scaled down: p up to 2^8 costs neither
// product nor sum any precision.
constexpr float kLazyMax = 8.f;

template <int KV, int NT>
__global__ __launch_bounds__(kPromptWaves * 64) void prompt_attention_kernel(const PromptParams p) {
    constexpr int ROWS = 32 * NT * kPromptWaves;
    extern __shared__ __align__(16) unsigned char lds[];         // [2 steps][2 blocks][keys | values][8192], then the prefix sums
    int *prefix = reinterpret_cast<int *>(lds + 2 * kPromptStepBytes);   // [n_seqs + 1]
    int *wave_sums = prefix + kMaxSeqs + 1;
    const PagedParams &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hi = lane >> 5, col = lane & 31;
    const int h = blockIdx.x % c.Hkv;

    // row tiles of the sequences, prefix sums
    int tiles = 0;
    for (int s0 = 0; s0 < c.n_seqs; s0 += 64 * kPromptWaves) {
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
        for (int i = 0; i < kPromptWaves; ++i) {
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

    bf16x8 qb[NT][8];                                            // lane (column, hi) holds d = 16 k + 8 hi .. + 7
    int limit[NT];                                               // last visible position of the lane's column
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = min(tile0 + (w * NT + nt) * 32 + col, R - 1);   // (rows behind the last one repeat it and are not stored)
        const int m = r / c.G, g = r % c.G;
        limit[nt] = a.len + m;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            qb[nt][k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p.q + (a.row0 + m) * p.ldq + ((long long)h * c.G + g) * kHeadDim + 16 * k + 8 * hi));
    }
    const int first_pos = a.len + tile0 / c.G;                   // positions up to here are visible to every row of the tile
    const int last_pos = a.len + (min(tile0 + ROWS, R) - 1) / c.G;
    const int nblk = blocks_of(c, last_pos + 1);
    const int steps = (nblk + 1) / 2;

    // ---- staging: wave w brings keys (w even) or values (w odd) of block w / 2 of every step
    constexpr int BB = kv_block_bytes<KV>, NL = BB / 1024;
    const long long head_step = (long long)(2 * BB) << c.block_shift, page_step = head_step * c.Hkv;
    const int in_page = (1 << c.block_shift) - 1;
    const int32_t *pages_of = c.table + s * c.table_ld;
    const unsigned char *head = c.pages + h * head_step + (w & 1) * BB;
    int ids = -1, ids_at = -64;                                  // pages of steps ids_at .. + 63, one a lane
    auto page_of_step = [&](int step) {
        if (step >= ids_at + 64 || ids_at < 0) {
            ids_at = step;
            const int b = 2 * (step + lane) + (w >> 1);
            ids = b < nblk ? pages_of[b >> c.block_shift] : -1;
        }
        return __builtin_amdgcn_readlane(ids, step - ids_at);
    };
    int *there = wave_sums + kPromptWaves;                       // [step parity][block]: the block has a page
    u32x4 code[NL];
    auto request = [&](int step) {
        const int page = page_of_step(step);
        const bool good = page_exists(page, c.n_pages);
        if (!(w & 1) && lane == 0) there[2 * (step & 1) + (w >> 1)] = good;
        const unsigned char *from = head + (good ? page : 0) * page_step + ((2 * step + (w >> 1)) & in_page) * (2 * BB);
        if constexpr (KV == KV_BF16) {
            const unsigned int to = lds_address_of(lds) + (step & 1) * kPromptStepBytes + w * kKvBlockBytes;
#pragma unroll
            for (int i = 0; i < NL; ++i) load_to_lds_16(reinterpret_cast<unsigned long long>(from) + 1024 * i, 16 * lane, to + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) code[i] = reinterpret_cast<const u32x4 *>(from)[64 * i + lane];
        }
    };
    // what request() asked for is in LDS afterwards (for this wave; the others' behind a barrier)
    auto settle = [&](int step) {
        if constexpr (KV == KV_BF16) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            u32x4 *to = reinterpret_cast<u32x4 *>(lds + (step & 1) * kPromptStepBytes + w * kKvBlockBytes) + lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                to[64 * (2 * i)] = e4m3x8_to_bf16(code[i].x, code[i].y);
                to[64 * (2 * i + 1)] = e4m3x8_to_bf16(code[i].z, code[i].w);
            }
        }
    };

    f32x16 oacc[4][NT];
    float mrow[NT], lrow[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        mrow[nt] = -__builtin_inff();
        lrow[nt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[dt][nt][i] = 0.f;
    }
    // this lane's place in a block: row col of the keys, d = col of the values
    const int k_lane = (((col >> 3) & 1) * 16 * 16 + ((col >> 4) * 8 + (col & 7)) + 16 * hi) * 16;   // [sub 2][kstep 4][g4 4][p 16] of 16 bytes
    const int v_lane = ((col >> 4) * 64 + (col & 15) + 16 * hi) * 16;                             // [dt 8][g4 4][dd 16] of 16 bytes

    if (steps > 0) request(0);
    for (int step = 0; step < steps; ++step) {
        settle(step);
        __syncthreads();
        const bool there0 = there[2 * (step & 1)], there1 = there[2 * (step & 1) + 1], gap = !(there0 && there1);
        if (step + 1 < steps) request(step + 1);
        const unsigned char *buf = lds + (step & 1) * kPromptStepBytes;
        const int pos0 = step * kPromptStep;
        const bool edge = pos0 + kPromptStep - 1 > first_pos || gap;

        f32x16 sc[2][NT];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[blk][nt][i] = 0.f;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(buf + blk * 2 * kKvBlockBytes + k_lane + k * 512);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) sc[blk][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[nt][k], sc[blk][nt], 0, 0, 0);
            }
        if (edge) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        // register 4 (2 t + c) + b: position 16 c + 8 t + 4 hi + b
                        const int pos = pos0 + 32 * blk + 16 * ((i >> 2) & 1) + 8 * (i >> 3) + 4 * hi + (i & 3);
                        if (pos > limit[nt] || !(blk ? there1 : there0)) sc[blk][nt][i] = -__builtin_inff();
                    }
        }
        u32x4 pb[2][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = -__builtin_inff();
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[blk][nt][i]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const bool moved = (mx - mrow[nt]) * scale_log2 > kLazyMax;          // (the first visible score, too)
            if (__builtin_amdgcn_ballot_w64(moved) != 0ull) {
                const float m_new = fmaxf(mrow[nt], mx);
                const float alpha = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((mrow[nt] - m_new) * scale_log2);
                mrow[nt] = m_new;
                lrow[nt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) oacc[dt][nt] *= alpha;
            }
            const float mc = mrow[nt] == -__builtin_inff() ? 0.f : -mrow[nt] * scale_log2;
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[blk][nt][2 * i], scale_log2, mc));
                    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[blk][nt][2 * i + 1], scale_log2, mc));
                    const unsigned int pk = float2_to_bf16_pair(e0, e1);
                    pb[blk][nt][i >> 2][i & 3] = pk;
                    // the sum of the rounded values, so that the weights that are applied sum to one
                    lrow[nt] += __uint_as_float(pk << 16) + __uint_as_float(pk & 0xFFFF0000u);
                }
        }
        const bool behind = pos0 + kPromptStep - 1 > last_pos || gap;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    u32x4 va = *reinterpret_cast<const u32x4 *>(buf + (2 * blk + 1) * kKvBlockBytes + v_lane + dt * 2048 + t * 512);
                    if (behind) {
                        // positions that no row sees hold whatever the page held: they must not reach the product (0 x NaN)
                        const int end = (blk ? there1 : there0) ? last_pos : -1;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int pos = pos0 + 32 * blk + 16 * (j >> 1) + 4 * (2 * t + hi) + 2 * (j & 1);
                            va[j] &= (pos <= end ? 0x0000FFFFu : 0u) | (pos + 1 <= end ? 0xFFFF0000u : 0u);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        oacc[dt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va), __builtin_bit_cast(bf16x8, pb[blk][nt][t]), oacc[dt][nt], 0, 0, 0);
                }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float sum = lrow[nt] + __shfl_xor(lrow[nt], 32, 64);
        const float inv = sum > 0.f ? __fdiv_rn(vs, sum) : 0.f;  // a row that sees nothing: zeros
        const int r = tile0 + (w * NT + nt) * 32 + col;
        if (r >= R) continue;
        const int m = r / c.G, g = r % c.G;
        uint16_t *to = p.out + (a.row0 + m) * p.ldo + ((long long)h * c.G + g) * kHeadDim + 4 * hi;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                        // registers 4 i .. + 3: d = 32 dt + 8 i + 4 hi ..
                const u32x2 o = {float2_to_bf16_pair(oacc[dt][nt][4 * i] * inv, oacc[dt][nt][4 * i + 1] * inv),
                                 float2_to_bf16_pair(oacc[dt][nt][4 * i + 2] * inv, oacc[dt][nt][4 * i + 3] * inv)};
                *reinterpret_cast<u32x2 *>(to + 32 * dt + 8 * i) = o;
            }
    }
}

}  // namespace quasar
