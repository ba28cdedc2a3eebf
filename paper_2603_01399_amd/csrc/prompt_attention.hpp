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

#include "paged_attention.hpp"

namespace quasar {

struct PromptParams {
    PagedParams c;
    const uint16_t *q;        // [T, Hq * 128] bf16
    uint16_t *out;
    long long ldq, ldo;
    f32x4 *part_o;            // FLAT: [Hkv][2 workers][NW][16][64], what workers leave of a tile that they share
    float *part_ml;           // [Hkv][2 workers][NW][64][2]
    int *pieces;              // [workers][4]: sequence of the tile that begins with a worker and goes on (-1: none), its first row, last worker, slot
    int workers;
    float scale_log2;         // log2(e) / sqrt(128)
};

constexpr int kPromptWaves = 4;                          // 128 rows a workgroup, two workgroups a compute unit
constexpr int kMaxFlatTiles = 2048;                      // of a launch that shares tiles: their prefix sums live in LDS
constexpr int kFlatLeast = 4;                            // steps that a worker takes at least

// A tile of rows: its sequence, its first row there, and what its rows see.
struct PromptTile {
    int s, tile0, R, first_pos, last_pos, steps;
    SeqSpan a;
};

template <int ROWS>
__device__ __forceinline__ PromptTile prompt_tile(const PagedParams &c, const int *prefix, int f) {
    PromptTile t;
    int s = 0, up = c.n_seqs;
    while (up - s > 1) {
        const int mid = (s + up) >> 1;
        if (prefix[mid] <= f) s = mid; else up = mid;
    }
    t.s = s;
    t.a = seq_span(c, s);
    t.R = t.a.n * c.G;
    t.tile0 = (f - prefix[s]) * ROWS;
    t.first_pos = t.a.len + t.tile0 / c.G;                       // positions up to here are visible to every row of the tile
    t.last_pos = t.a.len + (min(t.tile0 + ROWS, t.R) - 1) / c.G;
    t.steps = (blocks_of(c, t.last_pos + 1) + 1) / 2;
    return t;
}

constexpr int kPromptStep = 64;                          // positions in LDS at a time
constexpr int kPromptStepBytes = kPromptStep / kKvBlock * 2 * kKvBlockBytes;   // 32 KB: two blocks, keys and values

// FLAT: the steps of all tiles as one line, in equal pieces for `workers` workgroups of a kv head (as the blocks of a step's sequences,
// paged_attention.hpp), for launches whose tiles would leave compute units idle; else a workgroup a tile, the last ones, which see most,
// first.
template <int KV, bool FLAT>
__global__ __launch_bounds__(kPromptWaves * 64, 2) void prompt_attention_kernel(const PromptParams p) {
    constexpr int NW = kPromptWaves, ROWS = 32 * NW;
    extern __shared__ __align__(16) unsigned char lds[];         // [2 steps][2 blocks][keys | values][8192], then the prefix sums
    int *prefix = reinterpret_cast<int *>(lds + 2 * kPromptStepBytes);   // tiles ahead of a sequence
    int *wave_sums = prefix + kMaxSeqs;
    int *there = wave_sums + NW;                                 // [step parity][block]: the block has a page
    int *line = there + 4;                                       // FLAT: steps ahead of a tile
    const PagedParams &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hi = lane >> 5, col = lane & 31;
    const int h = blockIdx.x % c.Hkv, worker = blockIdx.x / c.Hkv;
    const float ks = c.k_scale ? c.k_scale[h] : 1.0f, vs = c.v_scale ? c.v_scale[h] : 1.0f;
    const float scale_log2 = p.scale_log2 * ks;

    int tiles = prefix_sums<NW>(c.n_seqs, prefix, wave_sums, [&](int s) { return (int)(((long long)seq_span(c, s).n * c.G + ROWS - 1) / ROWS); });
    int tile = tiles - 1 - worker, at = 0, end = 0;              // FLAT: steps at .. end - 1 of the line
    FlatShare mine{};
    int goes_on = -1, goes_on_at = 0, last_worker = 0, first_slot = 0;
    if constexpr (FLAT) {
        tiles = min(tiles, kMaxFlatTiles);                       // (more only where the rows' starts do not fit the tensor)
        const int total = prefix_sums<NW>(tiles, line, wave_sums, [&](int f) { return prompt_tile<ROWS>(c, prefix, f).steps; });
        mine = flat_share(total, p.workers, kFlatLeast, worker);
        at = mine.begin;
        end = mine.end;
        tile = 0;
        for (int up = tiles; up - tile > 1;) {
            const int mid = (tile + up) >> 1;
            if (line[mid] <= at) tile = mid; else up = mid;
        }
    }
    for (; FLAT ? at < end : tile >= 0; tile = FLAT ? tile + 1 : -1) {
    const PromptTile pt = prompt_tile<ROWS>(c, prefix, tile);
    const SeqSpan a = pt.a;
    const int R = pt.R, tile0 = pt.tile0, first_pos = pt.first_pos, last_pos = pt.last_pos, s = pt.s;
    const int nblk = blocks_of(c, last_pos + 1);
    int step0 = 0, steps = pt.steps;                             // the piece's part of the tile's steps
    if constexpr (FLAT) {
        step0 = at - line[tile];
        steps = min(pt.steps, step0 + end - at);
        at += steps - step0;
        lds_barrier();                                           // (the last tile's values may still be read)
    }
    const int my_row = tile0 + w * 32 + col;
    const int row = min(my_row, R - 1);                          // (rows behind the last one repeat it and are not stored)
    const int token = row / c.G;
    const int limit = a.len + token;                             // last visible position of the lane's column
    const long long head_at = ((long long)h * c.G + row % c.G) * kHeadDim;
    bf16x8 qb[8];                                                // lane (column, hi) holds d = 16 k + 8 hi .. + 7
#pragma unroll
    for (int k = 0; k < 8; ++k)
        qb[k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p.q + (a.row0 + token) * p.ldq + head_at + 16 * k + 8 * hi));

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
                lrow = add_bf16_pair(pk, lrow);
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
    int step = step0;
    bool settled = false;
    auto arrive = [&] {
        settle(step & 1);
        lds_barrier();
    };
    auto request_next = [&] {
        if (step + 1 < steps) request(step + 1);
    };
    if (step < steps) request(step);
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
    if (FLAT && (step0 > 0 || steps < pt.steps)) {
        const int slot = flat_slot(mine, worker, line[tile]);
        const long long part = ((long long)h * 2 * p.workers + slot) * NW + w;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                p.part_o[(part * 16 + 4 * dt + i) * 64 + lane] = f32x4{oacc[dt][4 * i], oacc[dt][4 * i + 1], oacc[dt][4 * i + 2], oacc[dt][4 * i + 3]};
        *reinterpret_cast<u32x2 *>(p.part_ml + (part * 64 + lane) * 2) = u32x2{__float_as_uint(mrow * scale_log2), __float_as_uint(lrow)};
        if (step0 == 0) {
            goes_on = s;
            goes_on_at = tile0;
            last_worker = (line[tile] + pt.steps - 1) / mine.share;
            first_slot = slot;
        }
        continue;
    }
    float sum = lrow + __shfl_xor(lrow, 32, 64);
    const float inv = sum > 0.f ? __fdiv_rn(vs, sum) : 0.f;      // a row that sees nothing: zeros
    if (my_row < R) {
        uint16_t *to = p.out + (a.row0 + token) * p.ldo + head_at + 4 * hi;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                        // registers 4 i .. + 3: d = 32 dt + 8 i + 4 hi ..
                const u32x2 o = {float2_to_bf16_pair(oacc[dt][4 * i] * inv, oacc[dt][4 * i + 1] * inv),
                                 float2_to_bf16_pair(oacc[dt][4 * i + 2] * inv, oacc[dt][4 * i + 3] * inv)};
                *reinterpret_cast<u32x2 *>(to + 32 * dt + 8 * i) = o;
            }
    }
    }
    if (FLAT && h == 0 && tid == 0) {
        int *piece = p.pieces + worker * 4;
        piece[0] = goes_on;
        piece[1] = goes_on_at;
        piece[2] = last_worker;
        piece[3] = first_slot;
    }
}

// Joins the parts of the tiles that several workers share.  A unit is 32 rows (a wave's) and 32 d of a kv head of such a tile: the four waves
// of a workgroup share its parts, four of them requested at a time, and meet in LDS; the workgroups walk the units.
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptParams p) {
    constexpr int NW = kPromptWaves;
    __shared__ f32x4 sacc[3][4][64];
    __shared__ u32x2 sml[3][64];
    __shared__ int list[kMaxWorkers];
    const PagedParams &c = p.c;
    const int units = shared_pieces(p.pieces, 4, p.workers, list) * c.Hkv * NW * 4;
    const int lane = threadIdx.x & 63, sg = threadIdx.x >> 6, hi = lane >> 5, col = lane & 31;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int dt = u & 3, w = (u >> 2) % NW, h = (u >> 2) / NW % c.Hkv, worker = list[(u >> 2) / NW / c.Hkv];
        const int *piece = p.pieces + worker * 4;
        const int s = piece[0], row = piece[1] + w * 32 + col, count = piece[2] - worker + 1, first_slot = piece[3];
        const SeqSpan a = seq_span(c, s);
        if (piece[1] + w * 32 >= a.n * c.G) continue;
        float m = -__builtin_inff(), l = 0.f;
        f32x4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto join = [&](const u32x2 ml, const f32x4 (&o)[4]) {   // another part of the same rows
            const float m_new = fmaxf(m, __uint_as_float(ml.x));
            const float m_use = m_new == -__builtin_inff() ? 0.f : m_new;        // nothing visible in these parts
            const float keep = exp2f(m - m_use), f = exp2f(__uint_as_float(ml.x) - m_use);
            l = l * keep + f * __uint_as_float(ml.y);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = acc[i] * keep + o[i] * f;
            m = m_new;
        };
        for (int k0 = sg; k0 < count; k0 += 16) {
            f32x4 o[4][4];
            u32x2 ml[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int slot = flat_part_slot(worker, first_slot, min(k0 + 4 * j, count - 1));
                const long long part = ((long long)h * 2 * p.workers + slot) * NW + w;
                ml[j] = *reinterpret_cast<const u32x2 *>(p.part_ml + (part * 64 + lane) * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j][i] = p.part_o[(part * 16 + 4 * dt + i) * 64 + lane];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k0 + 4 * j < count) join(ml[j], o[j]);
        }
        if (sg) {
            sml[sg - 1][lane] = u32x2{__float_as_uint(m), __float_as_uint(l)};
#pragma unroll
            for (int i = 0; i < 4; ++i) sacc[sg - 1][i][lane] = acc[i];
        }
        __syncthreads();
        if (sg == 0) {
            for (int k = 0; k < 3; ++k) {
                const f32x4 o[4] = {sacc[k][0][lane], sacc[k][1][lane], sacc[k][2][lane], sacc[k][3][lane]};
                join(sml[k][lane], o);
            }
            const float sum = l + __shfl_xor(l, 32, 64);
            const float vs = c.v_scale ? c.v_scale[h] : 1.0f;
            const float inv = sum > 0.f ? __fdiv_rn(vs, sum) : 0.f;
            if (row < a.n * c.G) {
                uint16_t *to = p.out + (a.row0 + row / c.G) * p.ldo + ((long long)h * c.G + row % c.G) * kHeadDim + 32 * dt + 4 * hi;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x2 o = {float2_to_bf16_pair(acc[i].x * inv, acc[i].y * inv), float2_to_bf16_pair(acc[i].z * inv, acc[i].w * inv)};
                    *reinterpret_cast<u32x2 *>(to + 8 * i) = o;
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace quasar
