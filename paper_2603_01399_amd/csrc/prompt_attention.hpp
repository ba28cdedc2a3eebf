// Causal attention of whole prompts, or chunks of them, over a paged key/value cache (gfx950): many rows per sequence, or the more than
// 32 rows of a draft.
//
// Rows are r = m * G + g: the G query heads of a key/value head side by side, so that a tile of rows covers few tokens
// (a narrow causal edge) and shares every key and value it loads.  A workgroup of four waves takes 128 (or 64) rows of one kv
// head; the waves share steps of 64 positions in LDS, loaded straight from the pages, two steps in turn.
//
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 products: a lane owns one query column.  The
// rows of K are permuted, row 16 t + 8 c + 4 h + b of the product being position 16 c + 8 t + 4 h + b, which makes the scores that a lane
// holds after the first product the operand of the second as they lie, against values in the cache's own order.
//
// Bound by the matrix cores and the power they draw: 8192 rows of 64 / 8 heads take 1.01 to 1.10 ms (1.0 to 1.09 PFLOP/s, in 8-bit pages 1.16 ms; a large library
// product reaches 1.36 on the same card).  Matrix cores are busy 52 % of the cycles there and the vector units 37 % with the softmax (32
// exponentials, 32 multiply-adds, 25 maxima, 16 conversions and 16 sums a wave and step of 32 products), at about 2.0 GHz; the products
// alone, without the softmax, took 0.82 to 0.88 ms.  LDS is busy 27 %, without bank conflicts.  Tried and slower or the same: 64 rows a
// wave (the accumulators' registers are copied), three steps in LDS, steps of 32 positions, priorities by phase or by wave.  Scores a block ahead, their
// products among the instructions of the softmax before: 5 % fewer cycles, 1056 us against 1072 on one card for 8192 rows, but 209 against 196 for
// 512 rows of 40 / 8 heads behind 16000 positions in 8-bit pages, whose start is a trip to memory longer.
// Many short prompts are bound by memory and the start of a tile: 60 of up to 300 rows 73 us, of which 32 for queries and outputs; 9 of up to 1531 107.
// (Tiles in the order of their steps, of whichever sequence, share fewer keys and values at a time: 9 of up to 1531 112.6, 30 of up to 700 118
// where the order of sequences took 108.)
#pragma once

#include <type_traits>

#include "paged_attention.hpp"

namespace quasar {

struct PromptParams {
    PagedParams c;
    const uint16_t *q;        // [T, Hq * 128] bf16
    uint16_t *out;
    long long ldq, ldo;
    f32x4 *part_o;            // FLAT: [Hkv][2 workers][32 rows of a tile][16][64], what workers leave of a tile that they share
    float *part_ml;           // [Hkv][2 workers][32 rows of a tile][64][2]
    int *pieces;              // [workers][4]: sequence of the tile that begins with a worker and goes on (-1: none), its first row, last worker, slot
    int workers;              // of a kv head
    int whole_more;           // steps that the longest tile may have beyond a worker's share while tiles stay whole
    float scale_log2;         // log2(e) / sqrt(128)
    Window window;            // WINDOW
};

constexpr int kPromptStep = 64, kStepShift = 6;          // positions in LDS at a time
constexpr int kPromptWaves = 4;                          // of a workgroup, two workgroups a compute unit
// Steps of a worker at least, where steps are shared: with fewer, what the join reads costs more than the worker saves (8 tokens over up to 8000
// positions, 64 / 8 heads, 20.5 us; two steps 24.1, three 22.7; over up to 1000, 8-bit, 15.6, 14.5 and 14.8).
constexpr int kFlatLeast = 4;
constexpr int kMaxFlatTiles = 2048;                      // of a launch that shares tiles: their prefix sums live in LDS

// A tile of rows: its sequence, its first row there, and what its rows see.
struct PromptTile {
    int s, tile0, R, first_pos, last_pos, steps;
    SeqSpan a;
    TileUnits units;          // WINDOW: which steps they are
};

// What the search of a tile needs: WINDOW or not, at compile time.
template <bool WINDOW> struct TileView {
    const PagedParams &c;
    Window window;
};
template <bool WINDOW>
__device__ __forceinline__ PromptTile prompt_tile(const TileView<WINDOW> &view, int rows, int s, const SeqSpan &a, int tile0) {
    const PagedParams &c = view.c;
    PromptTile t;
    t.s = s;
    t.a = a;
    t.R = a.n * c.G;
    t.tile0 = tile0;
    t.first_pos = a.len + tile0 / c.G;                           // positions up to here are visible to every row of the tile
    t.last_pos = a.len + (min(tile0 + rows, t.R) - 1) / c.G;
    t.steps = (blocks_of(c, t.last_pos + 1) + 1) / 2;
    if constexpr (WINDOW) {
        t.units = tile_units(view.window, t.first_pos, t.last_pos, t.steps, kStepShift);
        t.steps = t.units.u.count;
    }
    return t;
}

// Tile f of the line of all sequences' tiles.  UNIFORM: f is the same for the wave, and so is what it finds (LDS does not say so).
template <int ROWS, bool UNIFORM, bool WINDOW>
__device__ __forceinline__ PromptTile tile_of_line(const TileView<WINDOW> &view, const int *prefix, int f) {
    const PagedParams &c = view.c;
    int s = 0, up = c.n_seqs;
    while (up - s > 1) {
        const int mid = (s + up) >> 1;
        if (prefix[mid] <= f) s = mid; else up = mid;
    }
    if (UNIFORM) s = __builtin_amdgcn_readfirstlane(s);
    return prompt_tile(view, ROWS, s, seq_span(c, s), (f - (UNIFORM ? __builtin_amdgcn_readfirstlane(prefix[s]) : prefix[s])) * ROWS);
}

// Tile `back` from the end of the line; R = 0: there are fewer.  Each wave for itself, a sequence a lane: no LDS, and nothing is read twice.  Of up to
// kSortedSeqs sequences the longest one's tiles are first, which evens out what is left at the end: 9 prompts of up to 1531 rows 107.3 us, in the order
// of sequences 111.8; 4 of up to 2048 85.4 and 90.2; 16 of up to 300 26.3 and 29.1.  Of more, finding the order costs what it gives: 60 of up to
// 300 79.8 and 74.8, behind up to 2000 positions 308 and 324.
constexpr int kSortedSeqs = 32;
template <int ROWS, bool WINDOW>
__device__ __forceinline__ PromptTile tile_from_end(const TileView<WINDOW> &view, int back) {
    const PagedParams &c = view.c;
    constexpr int AT_ONCE = 4;
    const int lane = threadIdx.x & 63;
    auto tile_of = [&](const SeqSpan &a, int s, int &all, PromptTile &t) {       // of the sequences s of the lanes; all: their tiles
        const int upto = lane_sums((a.n * c.G + ROWS - 1) / ROWS);
        all = __builtin_amdgcn_readlane(upto, 63);
        if (back >= all) return false;
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > back));
        const SeqSpan of = {__builtin_amdgcn_readlane(a.row0, l), __builtin_amdgcn_readlane(a.n, l), __builtin_amdgcn_readlane(a.len, l)};
        t = prompt_tile(view, ROWS, __builtin_amdgcn_readlane(s, l), of, (__builtin_amdgcn_readlane(upto, l) - 1 - back) * ROWS);
        return true;
    };
    PromptTile t{};
    int all;
    if (c.n_seqs > 1 && c.n_seqs <= kSortedSeqs) {
        const SeqSpan a = lane < c.n_seqs ? seq_span(c, lane) : SeqSpan{0, 0, 0};
        const int reach = lane < c.n_seqs ? a.len + a.n : -1;
        int rank = 0;
        // how many come first: those that reach further, or as far from a lower lane (lanes without a sequence: behind all, where they carry nothing)
        for (int j0 = 0; j0 < c.n_seqs; j0 += 8)
#pragma unroll
            for (int j = j0; j < j0 + 8; ++j) {
                const int other = __builtin_amdgcn_readlane(reach, j);
                rank += other + (j < lane) > reach;
            }
        auto to_rank = [&](int v) { return __builtin_amdgcn_ds_permute(4 * rank, v); };          // (0 in the lanes that none goes to)
        tile_of(SeqSpan{to_rank(a.row0), to_rank(a.n), to_rank(a.len)}, to_rank(lane), all, t);
        return t;
    }
    for (int end = c.n_seqs; end > 0; end -= 64 * AT_ONCE) {
        SeqSpan a[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int s = end - 1 - 64 * k - lane;
            a[k] = s >= 0 ? seq_span(c, s) : SeqSpan{0, 0, 0};
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (tile_of(a[k], end - 1 - 64 * k - lane, all, t)) return t;
            back -= all;
        }
    }
    return t;
}

constexpr int kPromptStepBytes = kPromptStep / kKvBlock * 2 * kKvBlockBytes;   // 32 KB: two blocks, keys and values

// FLAT: the steps of all tiles as one line, in equal pieces for `workers` workgroups of a kv head (as the blocks of a step's sequences,
// paged_attention.hpp), for launches whose tiles would leave compute units idle; where the longest tile has hardly more steps than a piece, each
// tile goes to a worker as it is, and the join finds nothing (whole_more).  Else a workgroup a tile, the last ones, which see most, first.
// PW: waves that share rows.  1: four times 32 rows, each wave over both blocks of a step.  2: twice 32 rows, each wave over one of the
// blocks, joined at the end: for up to 64 rows a sequence, where half of four times 32 would be nobody's.
// 8-bit pages are widened on the way into LDS, once for all waves.  (In LDS as they are, four steps of half the size with three under way, and
// widened by each wave that reads them, 2 x 8 tokens of 64 / 8 heads over 100003 positions take 75.7 us, and 76.6 so.)
// WINDOW: a tile's steps are those that its rows see some position of, the ones that every row sees whole first (the order is free), so that the two
// loops over them are the same.  (Steps of any two blocks of 32, which leave no half of a step unused at the first tokens and the window's ends, are 5 % fewer and
// took 6 to 8 % longer, for prompts as for a draft's shared tiles.)  9 prompts of up to 1531 rows of 32 / 8 heads, a window of 333 and 4 first tokens: 92 us, 97 in 8-bit pages.  8192 rows of 64 / 8 heads,
// windows of 1024: 314 us, 0.82 PFLOP/s of what the rows see; of the 17 or 18 steps of a tile's 16 positions two or three are seen in part.
template <int KV, bool FLAT, int PW, bool WINDOW>
__global__ __launch_bounds__(kPromptWaves * 64, 2) void prompt_attention_kernel(const PromptParams p) {
    constexpr int NW = kPromptWaves, RW = NW / PW, ROWS = 32 * RW, NB = 2 / PW;  // row groups; blocks of a step for a wave
    constexpr bool DIRECT = KV == KV_BF16;                       // from memory into LDS
    extern __shared__ __align__(16) unsigned char lds[];         // [2 steps][2 blocks][keys | values][8192], then the prefix sums
    int *prefix = reinterpret_cast<int *>(lds + 2 * kPromptStepBytes);   // tiles ahead of a sequence
    int *wave_sums = prefix + kMaxSeqs;
    int *there = wave_sums + NW;                                 // [step & 3][block]: the block has a page
    int *line = there + 8;                                       // FLAT: steps ahead of a tile
    const PagedParams &c = p.c;
    const TileView<WINDOW> view{c, p.window};
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = w % RW, pw = w / RW;
    const int hi = lane >> 5, col = lane & 31;
    const int h = blockIdx.x % c.Hkv, worker = blockIdx.x / c.Hkv;
    const float ks = c.k_scale ? c.k_scale[h] : 1.0f, vs = c.v_scale ? c.v_scale[h] : 1.0f;
    const float scale_log2 = p.scale_log2 * ks;

    int tile = 0, at = 0, end = 0;                               // FLAT: steps at .. end - 1 of the line
    int tiles = 0, total = 0;
    bool shared = false;
    FlatShare mine{};
    int goes_on = -1, goes_on_at = 0, last_worker = 0, first_slot = 0;
    PromptTile pt{};
    if constexpr (FLAT) {
        // (more tiles than kMaxFlatTiles only where the rows' starts do not fit the tensor)
        tiles = min(kMaxFlatTiles, prefix_sums<NW>(c.n_seqs, prefix, wave_sums, [&](int s) {
            return (int)(((long long)seq_span(c, s).n * c.G + ROWS - 1) / ROWS);
        }));
        int longest = 0;                                         // steps of a tile, of those that this thread counts
        total = prefix_sums<NW>(tiles, line, wave_sums, [&](int f) {
            const int n = tile_of_line<ROWS, false>(view, prefix, f).steps;
            longest = max(longest, n);
            return n;
        });
        mine = flat_share(total, p.workers, kFlatLeast, worker);
        const bool pays = __builtin_amdgcn_ballot_w64(longest > mine.share + p.whole_more) != 0ull;
        if (lane == 0) wave_sums[w] = pays;
        __syncthreads();
        for (int i = 0; i < NW; ++i) shared |= wave_sums[i] != 0;
        shared = __builtin_amdgcn_readfirstlane(shared);
        if (shared) {
            at = __builtin_amdgcn_readfirstlane(mine.begin);
            end = __builtin_amdgcn_readfirstlane(mine.end);
            for (int up = tiles; up - tile > 1;) {
                const int mid = (tile + up) >> 1;
                if (line[mid] <= at) tile = mid; else up = mid;
            }
            tile = __builtin_amdgcn_readfirstlane(tile);
        } else {
            tile = worker;
            end = __builtin_amdgcn_readfirstlane(total);
            at = tile < tiles ? __builtin_amdgcn_readfirstlane(line[tile]) : end;
        }
    } else {
        pt = tile_from_end<ROWS>(view, worker);
    }
    auto next_tile = [&] {
        tile += shared ? 1 : p.workers;
        if (!shared) at = tile < tiles ? __builtin_amdgcn_readfirstlane(line[tile]) : end;
        return at < end;
    };
    for (bool more = FLAT ? at < end : pt.R > 0; more; more = FLAT && next_tile()) {
    if constexpr (FLAT) pt = tile_of_line<ROWS, true>(view, prefix, tile);
    const SeqSpan a = pt.a;
    const int R = pt.R, tile0 = pt.tile0, first_pos = pt.first_pos, last_pos = pt.last_pos, s = pt.s;
    const int nblk = blocks_of(c, last_pos + 1);
    auto step_at = [&](int i) {                                  // the i-th of the tile's steps
        if constexpr (WINDOW) return pt.units.at(i);
        return i;
    };
    int step0 = 0, steps = pt.steps;                             // the piece's part of the tile's steps
    if constexpr (FLAT) {
        step0 = at - __builtin_amdgcn_readfirstlane(line[tile]);
        steps = min(pt.steps, step0 + end - at);
        at += steps - step0;
        lds_barrier();                                           // (the last tile's values may still be read)
    }
    const int my_row = tile0 + rw * 32 + col;
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
    static_assert(PART == BB, "a wave's part is one block's keys or values");
    const int my_blk = w / (NW / 2), my_at = w * PART - my_blk * 2 * BB;         // (keys, then values, of a block are contiguous)
    const long long head_step = (long long)(2 * BB) << c.block_shift, page_step = head_step * c.Hkv;
    const int in_page = (1 << c.block_shift) - 1;
    const int32_t *pages_of = c.table + s * c.table_ld;
    const unsigned char *head = c.pages + h * head_step + my_at;
    int ids = -1, ids_at = -64;                                  // pages of steps ids_at .. + 63, one a lane
    u32x4 code[NL];
    auto request = [&](int step) {
        if (step >= ids_at + 64 || ids_at < 0) {
            ids_at = step;
            const int b = 2 * step_at(step + lane) + my_blk;
            ids = b < nblk ? pages_of[b >> c.block_shift] : -1;
        }
        const int page = __builtin_amdgcn_readlane(ids, step - ids_at);
        const bool good = page_exists(page, c.n_pages);
        if (my_at == 0 && lane == 0) there[2 * (step & 3) + my_blk] = good;
        const unsigned char *from = head + (good ? page : 0) * page_step + ((2 * step_at(step) + my_blk) & in_page) * (2 * BB);
        if constexpr (DIRECT) {
            // (scalar registers, which the load takes; the compiler may have them in vector ones)
            const unsigned int to = __builtin_amdgcn_readfirstlane(lds_address_of(lds) + (step & 1) * kPromptStepBytes + w * PART);
            const unsigned long long from64 = reinterpret_cast<unsigned long long>(from);
            const unsigned long long at = (unsigned long long)(unsigned int)__builtin_amdgcn_readfirstlane((int)(from64 >> 32)) << 32 |
                                          (unsigned int)__builtin_amdgcn_readfirstlane((int)from64);
#pragma unroll
            for (int i = 0; i < NL; ++i) load_to_lds_16(at + 1024 * i, 16 * lane, to + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) code[i] = reinterpret_cast<const u32x4 *>(from)[64 * i + lane];
        }
    };
    // what request() asked for is in LDS afterwards (for this wave; the others' behind a barrier)
    auto settle = [&](int step) {
        if constexpr (DIRECT) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            u32x4 *to = reinterpret_cast<u32x4 *>(lds + (step & 1) * kPromptStepBytes + w * 2 * PART) + lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                // (a wave's part is keys or values)
                to[64 * (2 * i)] = my_at ? e4m3x8_to_f16(code[i].x, code[i].y) : e4m3x8_to_bf16(code[i].x, code[i].y);
                to[64 * (2 * i + 1)] = my_at ? e4m3x8_to_f16(code[i].z, code[i].w) : e4m3x8_to_bf16(code[i].z, code[i].w);
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
    const int k_lane = (((col >> 3) & 1) * 256 + (col >> 4) * 8 + (col & 7) + 16 * hi) * 16;     // [sub 2][kstep 4][g4 4][p 16] of 16 bytes
    const int v_lane = ((col >> 4) * 64 + (col & 15) + 16 * hi) * 16;                         // [dt 8][g4 4][dd 16] of 16 bytes
    auto keys = [&](const unsigned char *at, int k) { return *reinterpret_cast<const bf16x8 *>(at + k_lane + k * 512); };
    auto values = [&](const unsigned char *at, int dt, int t) { return *reinterpret_cast<const u32x4 *>(at + v_lane + dt * 2048 + t * 512); };

    // the wave's blocks of a step; edge: some are hidden from some row, or are nobody's; between(): called while the scores are computed
    auto attend = [&](auto edge, int step, bool there0, bool there1, auto between) {
        constexpr bool EDGE = decltype(edge)::value;
        const unsigned char *buf = lds + (step & 1) * kPromptStepBytes;
        const int pos0 = step_at(step) * kPromptStep;
        auto block = [&](int b) { return PW == 1 ? b : pw; };    // the wave's b-th block
        auto has_page = [&](int b) { return block(b) ? there1 : there0; };
        f32x16 sc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bf16x8 ka = keys(buf + block(b) * 2 * kKvBlockBytes, k);
                sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[k], sc[b], 0, 0, 0);
            }
        if constexpr (EDGE) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // register 4 (2 t + c) + b: position 16 c + 8 t + 4 hi + b
                if constexpr (WINDOW) {
                    const unsigned int seen = has_page(b) ? seen_of_block(p.window, limit, pos0 + 32 * block(b)) >> (4 * hi) : 0u;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!(seen & 1u << (16 * ((i >> 2) & 1) + 8 * (i >> 3) + (i & 3)))) sc[b][i] = -__builtin_inff();
                } else {
                    const int left = has_page(b) ? limit - pos0 - 32 * block(b) - 4 * hi : -1;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (16 * ((i >> 2) & 1) + 8 * (i >> 3) + (i & 3) > left) sc[b][i] = -__builtin_inff();
                }
            }
        }
        between();                                               // (dozens of scalar instructions: while the products are under way)
        u32x4 v0[2][4];                                          // the first values, ahead of the softmax: its exponentials cover the way
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) v0[t][dt] = values(buf + (2 * block(0) + 1) * kKvBlockBytes, dt, t);
        float mx = larger(sc[0][0], sc[NB - 1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = larger(mx, larger(sc[0][i], sc[NB - 1][i]));
        mx = max_halves(mx);
        if (__builtin_amdgcn_ballot_w64((mx - mrow) * scale_log2 > kLazyMax) != 0ull) {          // (the first visible score, too)
            const float m_new = larger(mrow, mx);
            const float alpha = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((mrow - m_new) * scale_log2);
            mrow = m_new;
            lrow *= alpha;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) oacc[dt] *= alpha;
        }
        const float mc = kWeightShift<KV> + (mrow == -__builtin_inff() ? 0.f : -mrow * scale_log2);
        u32x4 pb[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * i], scale_log2, mc));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][2 * i + 1], scale_log2, mc));
                const unsigned int pk = weight_pair<KV>(e0, e1);
                pb[b][i >> 2][i & 3] = pk;
                lrow = add_pair<KV>(pk, lrow);
            }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    u32x4 va = b == 0 ? v0[t][dt] : values(buf + (2 * block(b) + 1) * kKvBlockBytes, dt, t);
                    if constexpr (EDGE) {
                        // positions that no row sees hold whatever the page held: they must not reach the product (0 x NaN)
                        const int end = has_page(b) ? last_pos - pos0 - 32 * block(b) - 4 * (2 * t + hi) : -1;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int at = 16 * (j >> 1) + 2 * (j & 1);
                            va[j] &= (at <= end ? 0x0000FFFFu : 0u) | (at + 1 <= end ? 0xFFFF0000u : 0u);
                        }
                        if (any_nonfinite<KV>(va)) {
                            if constexpr (WINDOW) {
                                const unsigned int bad = drop_nonfinite_of_block<KV>(va, 4 * (2 * t + hi));
                                if (bad & seen_of_block(p.window, limit, pos0 + 32 * block(b))) lrow = __builtin_nanf("");
                            } else {
                                const int first = drop_nonfinite<KV>(va, pos0 + 32 * block(b) + 4 * (2 * t + hi));
                                if (limit >= first) lrow = __builtin_nanf("");
                            }
                        }
                    }
                    oacc[dt] = values_times_weights<KV>(va, pb[b][t], oacc[dt]);
                }
    };
    // The steps that every row sees whole, then the others (and all from the first that lacks a page on): two loops, since the outputs'
    // registers would be copied once a step where the two ways met.
    const int whole = min(WINDOW ? pt.units.whole : (first_pos + 1) / kPromptStep, steps);
    int step = step0;
    bool settled = false;
    auto arrive = [&] {
        if constexpr (DIRECT) settle(step);
        lds_barrier();
    };
    // (codes that pass through registers are widened while the scores of the step before are computed, and those of the step behind requested)
    auto request_next = [&] {
        if constexpr (DIRECT) {
            if (step + 1 < steps) request(step + 1);
        } else {
            if (step + 1 < steps) settle(step + 1);
            if (step + 2 < steps) request(step + 2);
        }
    };
    auto has = [&](int blk) { return __builtin_amdgcn_readfirstlane(there[2 * (step & 3) + blk]) != 0; };
    if (step < steps) request(step);
    if constexpr (!DIRECT) {
        if (step < steps) settle(step);
        if (step + 1 < steps) request(step + 1);
    }
    for (; step < whole; step = step + 1) {
        arrive();
        settled = !(has(0) && has(1));
        if (settled) break;
        attend(std::false_type{}, step, true, true, request_next);
    }
    for (; step < steps; step = step + 1) {
        if (!settled) arrive();
        settled = false;
        attend(std::true_type{}, step, has(0), has(1), request_next);
    }
    if constexpr (PW > 1) {
        // waves that share rows: the second leaves its part in LDS (in the place of the steps), the first takes it in
        f32x4 *lo = reinterpret_cast<f32x4 *>(lds);              // [RW][16][64]
        u32x2 *lml = reinterpret_cast<u32x2 *>(lds + RW * 16 * 64 * 16);
        lds_barrier();
        if (pw) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                lo[(rw * 16 + i) * 64 + lane] = f32x4{oacc[i >> 2][4 * (i & 3)], oacc[i >> 2][4 * (i & 3) + 1], oacc[i >> 2][4 * (i & 3) + 2], oacc[i >> 2][4 * (i & 3) + 3]};
            lml[rw * 64 + lane] = u32x2{__float_as_uint(mrow), __float_as_uint(lrow)};
        }
        lds_barrier();
        if (!pw) {
            const u32x2 ml = lml[rw * 64 + lane];
            const float m_new = fmaxf(mrow, __uint_as_float(ml.x)), m_use = m_new == -__builtin_inff() ? 0.f : m_new;
            const float keep = __builtin_amdgcn_exp2f((mrow - m_use) * scale_log2), fac = __builtin_amdgcn_exp2f((__uint_as_float(ml.x) - m_use) * scale_log2);
            lrow = lrow * keep + fac * __uint_as_float(ml.y);
            mrow = m_new;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const f32x4 o = lo[(rw * 16 + i) * 64 + lane];
#pragma unroll
                for (int j = 0; j < 4; ++j) oacc[i >> 2][4 * (i & 3) + j] = oacc[i >> 2][4 * (i & 3) + j] * keep + o[j] * fac;
            }
        }
    }
    if (FLAT && (step0 > 0 || steps < pt.steps)) {
        const int slot = flat_slot(mine, worker, line[tile]);
        const long long part = ((long long)h * 2 * p.workers + slot) * RW + rw;
        if (pw == 0) {
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p.part_o[(part * 16 + 4 * dt + i) * 64 + lane] = f32x4{oacc[dt][4 * i], oacc[dt][4 * i + 1], oacc[dt][4 * i + 2], oacc[dt][4 * i + 3]};
            *reinterpret_cast<u32x2 *>(p.part_ml + (part * 64 + lane) * 2) = u32x2{__float_as_uint(mrow * scale_log2), __float_as_uint(lrow)};
        }
        if (step0 == 0) {
            goes_on = s;
            goes_on_at = tile0;
            last_worker = (line[tile] + pt.steps - 1) / mine.share;
            first_slot = slot;
        }
        continue;
    }
    float sum = lrow + __shfl_xor(lrow, 32, 64);
    const float inv = sum == 0.f ? 0.f : __fdiv_rn(vs, sum);      // a row that sees nothing: zeros
    if (pw == 0 && my_row < R) {
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

// Joins the parts of the tiles that several workers share.  A unit is 32 rows (a wave's) and 32 d of a kv head of such a tile.  As in
// paged_merge_kernel, the four waves of a workgroup share its parts, four of them requested at a time, and meet in LDS, or each takes units of its
// own where there are more of them than workgroups (4 x 700 tokens of 32 / 8 heads behind 3000
// positions, with the attention: 110.7 us, and 115.5 by workgroups that walk the units).
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptParams p, int RW /* 32 rows of a tile */) {
    __shared__ f32x4 sacc[3][4][64];
    __shared__ u32x2 sml[3][64];
    __shared__ int list[kMaxWorkers];
    const PagedParams &c = p.c;
    const int units = shared_pieces(p.pieces, 4, p.workers, list) * c.Hkv * RW * 4;
    const int lane = threadIdx.x & 63, sg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5, col = lane & 31;
    auto unit = [&](auto each_wave, int u) {
        constexpr bool alone = decltype(each_wave)::value;       // a wave for itself
        const int dt = u & 3, w = (u >> 2) % RW, h = (u >> 2) / RW % c.Hkv, worker = __builtin_amdgcn_readfirstlane(list[(u >> 2) / RW / c.Hkv]);
        const int *piece = p.pieces + worker * 4;
        const int s = piece[0], row = piece[1] + w * 32 + col, count = piece[2] - worker + 1, first_slot = piece[3];
        const SeqSpan a = seq_span(c, s);
        if (piece[1] + w * 32 >= a.n * c.G) return;
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
        const int step = alone ? 1 : 4;
        for (int k0 = alone ? 0 : sg; k0 < count; k0 += 4 * step) {
            f32x4 o[4][4];
            u32x2 ml[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int slot = flat_part_slot(worker, first_slot, min(k0 + step * j, count - 1));
                const long long part = ((long long)h * 2 * p.workers + slot) * RW + w;
                ml[j] = *reinterpret_cast<const u32x2 *>(p.part_ml + (part * 64 + lane) * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[j][i] = p.part_o[(part * 16 + 4 * dt + i) * 64 + lane];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k0 + step * j < count) join(ml[j], o[j]);
        }
        if constexpr (!alone) {
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
            }
        }
        const float sum = l + __shfl_xor(l, 32, 64);
        const float vs = c.v_scale ? c.v_scale[h] : 1.0f;
        const float inv = sum == 0.f ? 0.f : __fdiv_rn(vs, sum);
        if ((alone || sg == 0) && row < a.n * c.G) {
            uint16_t *to = p.out + (a.row0 + row / c.G) * p.ldo + ((long long)h * c.G + row % c.G) * kHeadDim + 32 * dt + 4 * hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x2 o = {float2_to_bf16_pair(acc[i].x * inv, acc[i].y * inv), float2_to_bf16_pair(acc[i].z * inv, acc[i].w * inv)};
                *reinterpret_cast<u32x2 *>(to + 8 * i) = o;
            }
        }
    };
    if (units > (int)gridDim.x) {
        for (int u = blockIdx.x * 4 + sg; u < units; u += gridDim.x * 4) unit(std::true_type{}, u);
    } else if ((int)blockIdx.x < units) {
        unit(std::false_type{}, blockIdx.x);
    }
}

}  // namespace quasar
