// Attention of the new tokens of a step - one, or a short draft, per sequence - over a paged key/value cache (gfx950): up to 32 rows
// m * G + g of a sequence and kv head; more go the way of prompts (prompt_attention.hpp).
//
// The arithmetic is that of verify_attention_kernel: S^T = K Q^T and O^T = V^T P^T, a lane owning one query column.  What differs is the
// work split.  The lengths are on the device and as ragged as the traffic, so a grid over sequences leaves the card to the longest
// one; instead the blocks of all sequences are ONE line, cut into equal pieces for the workers of a kv head:
//   flat blocks   |--- sequence 0 ---|- 1 -|-------- sequence 2 --------|
//   workers       |    0    |    1    |    2    |    3    |    4    |
// A worker walks the sequences in its piece.  One that lies in it whole is finished there; of the (at most two) that it shares with a
// neighbour it leaves maximum, sum and output to the merge, in the slot of the piece's beginning or of its end.
//
// Bound by memory where the cache is long: 64 sequences of one token over up to 8192 positions (1.21 GB, 32 / 8 heads) take 191 us with the
// merge, 6.3 TB/s where a plain read reaches 6.7; in 8-bit pages 99.5, 6.1 TB/s; one sequence over up to 100003 positions 68, 6.0 TB/s.  Bound by
// the way to memory and back where it is short: 4 over up to 1000 12.6 to 13.1 us, 8.0 and 3.4 in the kernels, of which 3 go by until the page table
// is known, and 2 for each trip.  One workgroup a compute unit: two take 200 us for the first, since more pieces are shared.
#pragma once

#include <type_traits>

#include "paged.hpp"

namespace quasar {

struct PagedAttnParams {
    PagedParams c;
    const uint16_t *q;        // [T, Hq * 128] bf16
    uint16_t *out;
    long long ldq, ldo;
    f32x4 *part_o;            // [Hkv][2 workers][NQT][8][64]
    float *part_ml;           // [Hkv][2 workers][NQT][16][2]
    int *pieces;              // [workers][4]: sequence that begins here and goes on (-1: none), last worker, slot
    int workers;
    float scale_log2;         // log2(e) / sqrt(128)
    Window window;            // WINDOW
    bool each;                // WINDOW: a worker has a sequence, nothing is shared
};

constexpr int kPagedWaves = 4, kLoneWaves = 8;           // of a workgroup; where it has a compute unit and a sequence to itself
constexpr int kMaxWorkers = 512;             // of a kv head

// WINDOW: a sequence's blocks are those that its rows see some position of; those between the first tokens and the window have no place in
// the line, whatever the context's length.  64 sequences of one token over up to 16000 positions in 8-bit pages, 64 / 8 heads, windows of 4096 (518 MB): 81.5 us,
// 6.4 TB/s.
template <int KV, int NQT, bool WINDOW, int NW = kPagedWaves>
__global__ __launch_bounds__(NW * 64, NQT == 1 ? 2 : 1) void paged_attention_kernel(const PagedAttnParams p) {
    constexpr int BB = kv_block_bytes<KV>, NL = BB / 1024;     // 16-byte loads of a lane per block
    extern __shared__ __align__(16) unsigned char lds[];
    f32x4 *lo = reinterpret_cast<f32x4 *>(lds);                                  // [NW][NQT][8][64]
    float *lml = reinterpret_cast<float *>(lds + NW * NQT * 8 * 64 * 16);        // [NW][NQT][16][2]
    int *wave_sums = reinterpret_cast<int *>(lml + NW * NQT * 16 * 2);
    int *prefix = wave_sums + NW;                                                // [n_seqs + 1]
    SeqSpan *spans = reinterpret_cast<SeqSpan *>(prefix + p.c.n_seqs + 1);       // [n_seqs]: read once, not again from memory
    const PagedParams &c = p.c;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g4 = lane >> 4, col = lane & 15;
    const int h = blockIdx.y, worker = blockIdx.x;

    const int total = prefix_sums<NW>(c.n_seqs, prefix, wave_sums, [&](int s) {
        const SeqSpan a = seq_span(c, s);
        spans[s] = a;
        const int blocks = a.n ? blocks_of(c, a.len + a.n) : 0;
        if constexpr (WINDOW) return window_units(p.window, a.len, blocks, kBlockShift).count;
        return blocks;
    });
    if (tid == 0) prefix[c.n_seqs] = total;
    __syncthreads();
    FlatShare mine = flat_share(total, p.workers, NW, worker);                   // (a block for each wave)
    if (WINDOW && p.each) mine = FlatShare{1, prefix[worker], prefix[worker + 1]};
    int f = mine.begin;
    const int f_end = mine.end;
    int *piece = p.pieces + worker * 4;
    int goes_on = -1, last_worker = 0, first_slot = 0;
    // first sequence of the piece: the last one that begins at or before f (those without blocks are skipped by the search)
    int s = 0;
    if (f < f_end) {
        int hi = c.n_seqs;
        while (hi - s > 1) {
            const int mid = (s + hi) >> 1;
            if (prefix[mid] <= f) s = mid; else hi = mid;
        }
    }
    const float ks = c.k_scale ? c.k_scale[h] : 1.0f, vs = c.v_scale ? c.v_scale[h] : 1.0f;
    const float scale_log2 = p.scale_log2 * ks;
    const long long head_step = (long long)(2 * BB) << c.block_shift, page_step = head_step * c.Hkv;
    const int in_page = (1 << c.block_shift) - 1;

    for (; f < f_end; ++s) {
        const int s_begin = prefix[s], s_end = prefix[s + 1];
        if (s_end <= f) continue;
        const SeqSpan a = spans[s];
        const int n = a.n, R = n * c.G;
        const int b0 = f - s_begin, b1 = (s_end < f_end ? s_end : f_end) - s_begin;
        const int32_t *pages_of = c.table + s * c.table_ld;
        WindowUnits units{};
        if constexpr (WINDOW) units = window_units(p.window, a.len, blocks_of(c, a.len + n), kBlockShift);
        auto block_at = [&](int i) {          // the i-th of the sequence's blocks
            if constexpr (WINDOW) return units.at(i);
            return i;
        };

        // queries as B operands: lane (query column col, k group g4) holds d = 32 ks + 8 g4 .. + 7
        bf16x8 qb[NQT][4];
        int limit[NQT];                       // last visible position of this lane's query column
#pragma unroll
        for (int qt = 0; qt < NQT; ++qt) {
            const int r = 16 * qt + col;
            const int m = r < R ? r / c.G : n - 1, g = r < R ? r % c.G : 0;
            limit[qt] = a.len + m;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (r < R)
                    v = *reinterpret_cast<const u32x4 *>(p.q + (a.row0 + m) * p.ldq + ((long long)h * c.G + g) * kHeadDim + 32 * k + 8 * g4);
                qb[qt][k] = __builtin_bit_cast(bf16x8, v);
            }
        }
        f32x4 oacc[8][NQT];
        float mrow[NQT], lrow[NQT];
#pragma unroll
        for (int qt = 0; qt < NQT; ++qt) {
            mrow[qt] = -__builtin_inff();
            lrow[qt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) oacc[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        u32x4 kc[NL], vc[NL];
        auto load_block = [&](int b, int page, u32x4 (&k)[NL], u32x4 (&v)[NL]) {
            const u32x4 *from = reinterpret_cast<const u32x4 *>(c.pages + page * page_step + h * head_step + (b & in_page) * (2 * BB)) + lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) k[i] = __builtin_nontemporal_load(from + 64 * i);
#pragma unroll
            for (int i = 0; i < NL; ++i) v[i] = __builtin_nontemporal_load(from + 64 * (NL + i));
        };
        auto k_operand = [&](int sub, int k) {
            if constexpr (KV == KV_BF16) return kc[sub * 4 + k];
            const u32x4 v = kc[sub * 2 + (k >> 1)];
            return k & 1 ? e4m3x8_to_bf16(v.z, v.w) : e4m3x8_to_bf16(v.x, v.y);
        };
        auto v_operand = [&](int dt) {
            if constexpr (KV == KV_BF16) return vc[dt];
            const u32x4 v = vc[dt >> 1];
            return dt & 1 ? e4m3x8_to_f16(v.z, v.w) : e4m3x8_to_f16(v.x, v.y);
        };
        // `there`: the table names a page of the cache for the block; else its positions count as hidden
        auto process = [&](int b, bool there) {
            const int pos0 = b * kKvBlock, end = there ? a.len + n : 0;
            bool edge = pos0 + kKvBlock - 1 > a.len || !there;         // some position may be hidden from some query
            if constexpr (WINDOW) edge |= pos0 <= a.len + n - 1 - p.window.size && pos0 + kKvBlock > p.window.sinks;
            unsigned int keep[4] = {~0u, ~0u, ~0u, ~0u};
            if (edge) {
                // positions behind the sequence hold whatever the page held: values there must not reach the product (0 x NaN)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int oa = pos0 + 4 * g4 + (j & 1) * 2 + (j >> 1) * 16;
                    keep[j] = (oa < end ? 0x0000FFFFu : 0u) | (oa + 1 < end ? 0xFFFF0000u : 0u);
                }
                if constexpr (WINDOW) {                        // (nor values that the first row's window has passed)
                    const unsigned int seen = seen_of_block(p.window, a.len, pos0) | ~bits_through(a.len - pos0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned int pair = seen >> (4 * g4 + (j & 1) * 2 + (j >> 1) * 16);
                        keep[j] &= (pair & 1u ? 0x0000FFFFu : 0u) | (pair & 2u ? 0xFFFF0000u : 0u);
                    }
                }
            }
            f32x4 sc[NQT][2];
#pragma unroll
            for (int qt = 0; qt < NQT; ++qt) sc[qt][0] = sc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int sub = 0; sub < 2; ++sub) {
                    const bf16x8 ka = __builtin_bit_cast(bf16x8, k_operand(sub, k));
#pragma unroll
                    for (int qt = 0; qt < NQT; ++qt) sc[qt][sub] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[qt][k], sc[qt][sub], 0, 0, 0);
                }
            if (edge) {
#pragma unroll
                for (int qt = 0; qt < NQT; ++qt) {
                    unsigned int seen = 0;
                    if constexpr (WINDOW) seen = there ? seen_of_block(p.window, limit[qt], pos0) >> (4 * g4) : 0u;
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (WINDOW ? !(seen & 1u << (16 * sub + i)) : pos0 + 16 * sub + 4 * g4 + i > limit[qt] || !there) sc[qt][sub][i] = -__builtin_inff();
                        }
                }
            }
            u32x4 pb16[NQT];
            bool moved = false;
            float alpha[NQT];
#pragma unroll
            for (int qt = 0; qt < NQT; ++qt) {
                float mx = fmaxf(fmaxf(fmaxf(sc[qt][0].x, sc[qt][0].y), fmaxf(sc[qt][0].z, sc[qt][0].w)),
                                 fmaxf(fmaxf(sc[qt][1].x, sc[qt][1].y), fmaxf(sc[qt][1].z, sc[qt][1].w)));
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float m_new = fmaxf(mrow[qt], mx);
                const float mc = m_new == -__builtin_inff() ? 0.f : -m_new * scale_log2;                                      // nothing visible yet
                const float ms = mc + kWeightShift<KV>;
                alpha[qt] = __builtin_amdgcn_exp2f(__builtin_fmaf(mrow[qt], scale_log2, mc));   // 0 while mrow is -inf
                mrow[qt] = m_new;
                float psum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qt][i >> 1][2 * (i & 1)], scale_log2, ms));
                    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qt][i >> 1][2 * (i & 1) + 1], scale_log2, ms));
                    pb16[qt][i] = weight_pair<KV>(e0, e1);
                    psum = add_pair<KV>(pb16[qt][i], psum);
                }
                lrow[qt] = lrow[qt] * alpha[qt] + psum;
                moved |= alpha[qt] != 1.0f;
            }
            if (__builtin_amdgcn_ballot_w64(moved) != 0ull) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                    for (int qt = 0; qt < NQT; ++qt) oacc[dt][qt] *= alpha[qt];
            }
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                u32x4 v = v_operand(dt);
                if (edge) {
                    v.x &= keep[0];
                    v.y &= keep[1];
                    v.z &= keep[2];
                    v.w &= keep[3];
                    if (n > 1 && any_nonfinite<KV>(v)) {
                        if constexpr (WINDOW) {
                            const unsigned int bad = drop_nonfinite_of_block<KV>(v, 4 * g4);
#pragma unroll
                            for (int qt = 0; qt < NQT; ++qt)
                                if (bad & seen_of_block(p.window, limit[qt], pos0)) lrow[qt] = __builtin_nanf("");
                        } else {
                            const int first = drop_nonfinite<KV>(v, pos0 + 4 * g4);
#pragma unroll
                            for (int qt = 0; qt < NQT; ++qt)
                                if (limit[qt] >= first) lrow[qt] = __builtin_nanf("");
                        }
                    }
                }
#pragma unroll
                for (int qt = 0; qt < NQT; ++qt)
                    oacc[dt][qt] = values_times_weights<KV>(v, pb16[qt], oacc[dt][qt]);
            }
        };
        // a wave's blocks are b0 + w, b0 + w + NW, ...; 64 of their page ids are fetched at a time, one a lane
        for (int bs = b0 + w; bs < b1; bs += 64 * NW) {
            const int ahead = bs + NW * lane;
            int id = -1;
            if (ahead < b1) id = pages_of[block_at(ahead) >> c.block_shift];
            const int cnt = min(64, (b1 - bs + NW - 1) / NW);
            auto page_at = [&](int i) { return __builtin_amdgcn_readlane(id, i); };
            auto good = [&](int page) { return page_exists(page, c.n_pages); };
            // one block of prefetch, the last block of a wave without one: the number of loads in flight is known at every use
            int page = page_at(0);
            load_block(block_at(bs), good(page) ? page : 0, kc, vc);
            for (int i = 0; i + 1 < cnt; ++i) {
                u32x4 kn[NL], vn[NL];
                const int next = page_at(i + 1), b = bs + NW * i;
                load_block(block_at(b + NW), good(next) ? next : 0, kn, vn);
                process(block_at(b), good(page));
#pragma unroll
                for (int l = 0; l < NL; ++l) { kc[l] = kn[l]; vc[l] = vn[l]; }
                page = next;
            }
            process(block_at(bs + NW * (cnt - 1)), good(page));
        }
        // the four lanes of a query column hold partial row sums; the maxima go on in log2 units
#pragma unroll
        for (int qt = 0; qt < NQT; ++qt) {
            lrow[qt] += __shfl_xor(lrow[qt], 16, 64);
            lrow[qt] += __shfl_xor(lrow[qt], 32, 64);
            mrow[qt] *= scale_log2;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) lo[((w * NQT + qt) * 8 + dt) * 64 + lane] = oacc[dt][qt];
            if (g4 == 0) {
                lml[((w * NQT + qt) * 16 + col) * 2 + 0] = mrow[qt];
                lml[((w * NQT + qt) * 16 + col) * 2 + 1] = lrow[qt];
            }
        }
        __syncthreads();
        const bool whole = b0 == 0 && b1 == s_end - s_begin;
        const int slot = flat_slot(mine, worker, s_begin);
        const long long pbase = ((long long)h * (2 * p.workers) + slot) * NQT;
        if (!whole && b0 == 0) {
            goes_on = s;
            last_worker = (s_end - 1) / mine.share;
            first_slot = slot;
        }
#pragma unroll
        for (int qt = 0; qt < NQT; ++qt) {
            float mstar = -__builtin_inff();
            for (int ww = 0; ww < NW; ++ww) mstar = fmaxf(mstar, lml[((ww * NQT + qt) * 16 + col) * 2]);
            const float m_use = mstar == -__builtin_inff() ? 0.f : mstar;
            float fac[NW], lsum = 0.f;
            for (int ww = 0; ww < NW; ++ww) {
                fac[ww] = exp2f(lml[((ww * NQT + qt) * 16 + col) * 2] - m_use);
                lsum += fac[ww] * lml[((ww * NQT + qt) * 16 + col) * 2 + 1];
            }
            const int r = 16 * qt + col;
            const float inv = lsum == 0.f ? 0.f : __fdiv_rn(vs, lsum);            // a row that sees nothing: zeros
            for (int dt = w; dt < 8; dt += NW) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                for (int ww = 0; ww < NW; ++ww) acc += lo[((ww * NQT + qt) * 8 + dt) * 64 + lane] * fac[ww];
                if (!whole) {
                    p.part_o[((pbase + qt) * 8 + dt) * 64 + lane] = acc;
                } else if (r < R) {
                    const int m = r / c.G, g = r % c.G;
                    const u32x2 o = {float2_to_bf16_pair(acc.x * inv, acc.y * inv), float2_to_bf16_pair(acc.z * inv, acc.w * inv)};
                    *reinterpret_cast<u32x2 *>(p.out + (a.row0 + m) * p.ldo + ((long long)h * c.G + g) * kHeadDim + 16 * dt + 4 * g4) = o;
                }
            }
            if (!whole && w == 0 && g4 == 0) {
                p.part_ml[((pbase + qt) * 16 + col) * 2 + 0] = mstar;
                p.part_ml[((pbase + qt) * 16 + col) * 2 + 1] = lsum;
            }
        }
        __syncthreads();                                                         // (the next sequence's merge reuses the LDS)
        f = s_begin + b1;
    }
    if (h == 0 && tid == 0 && !(WINDOW && p.each)) {
        piece[0] = goes_on;
        piece[1] = last_worker;
        piece[2] = first_slot;
    }
}

// The workers in whose pieces a shared sequence (or tile) begins, in order, into list; how many.  records: of each worker `words` ints, the
// first of them < 0 where none begins.
__device__ __forceinline__ int shared_pieces(const int *records, int words, int workers, int *list) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int i = 0; i < workers; i += 64) {
        const bool begins = i + lane < workers && records[(i + lane) * words] >= 0;
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(begins);
        if (begins && threadIdx.x < 64) list[n + __popcll(mask & ((1ull << lane) - 1))] = i + lane;
        n += __popcll(mask);
    }
    __syncthreads();
    return n;
}

// Joins the pieces of the sequences that several workers share.  A unit is 16 rows and 16 d of a kv head of such a sequence.  Where a workgroup
// has one unit, its eight waves share the pieces, four of them requested at a time, and meet in LDS; where there are more units than
// workgroups, many sequences are shared by few workers each, and every wave takes units of its own (64 x 1 tokens over up to 8192 positions, with the
// attention: 191.9 us, and 197.5 by workgroups that walk the units; 16 x 8 over 4000: 39.2 and 44.5).
__global__ __launch_bounds__(512) void paged_merge_kernel(const PagedAttnParams p, int NQT) {
    __shared__ float smax[8][16];
    __shared__ float slsum[8][16];
    __shared__ f32x4 sacc[8][64];
    __shared__ int list[kMaxWorkers];
    const PagedParams &c = p.c;
    const int *records = p.pieces;
    const int units = shared_pieces(records, 4, p.workers, list) * c.Hkv * NQT * 8;
    const int sg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g4 = lane >> 4, col = lane & 15;
    auto unit = [&](auto each_wave, int u) {
        constexpr bool alone = decltype(each_wave)::value;       // a wave for itself
        const int dt = u & 7, qt = (u >> 3) % NQT, h = (u >> 3) / NQT % c.Hkv, worker = __builtin_amdgcn_readfirstlane(list[(u >> 3) / NQT / c.Hkv]);
        const int s = records[worker * 4], last = records[worker * 4 + 1], first_slot = records[worker * 4 + 2];
        const SeqSpan a = seq_span(c, s);
        const int R = a.n * c.G, r = 16 * qt + col;
        if (16 * qt >= R) return;
        const int count = last - worker + 1, step = alone ? 1 : 8;
        float mw = -__builtin_inff(), lsum = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int k0 = alone ? 0 : sg; k0 < count; k0 += 4 * step) {
            f32x4 o[4];
            u32x2 ml[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = flat_part_slot(worker, first_slot, min(k0 + step * i, count - 1));
                const long long pb = ((long long)h * (2 * p.workers) + slot) * NQT + qt;
                ml[i] = reinterpret_cast<const u32x2 *>(p.part_ml)[pb * 16 + col];
                o[i] = p.part_o[(pb * 8 + dt) * 64 + lane];
            }
            float m_new = mw;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + step * i < count) m_new = fmaxf(m_new, __uint_as_float(ml[i].x));
            const float m_use = m_new == -__builtin_inff() ? 0.f : m_new;        // nothing visible in these pieces
            const float keep = exp2f(mw - m_use);
            acc *= keep;
            lsum *= keep;
            mw = m_new;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + step * i < count) {
                    const float f = exp2f(__uint_as_float(ml[i].x) - m_use);
                    lsum += f * __uint_as_float(ml[i].y);
                    acc += o[i] * f;
                }
        }
        if constexpr (!alone) {
            sacc[sg][lane] = acc;
            if (g4 == 0) { smax[sg][col] = mw; slsum[sg][col] = lsum; }
            __syncthreads();
            if (sg == 0) {
                float mstar = smax[0][col];
#pragma unroll
                for (int i = 1; i < 8; ++i) mstar = fmaxf(mstar, smax[i][col]);
                const float m_use = mstar == -__builtin_inff() ? 0.f : mstar;
                acc = f32x4{0.f, 0.f, 0.f, 0.f};
                lsum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float f = exp2f(smax[i][col] - m_use);
                    acc += sacc[i][lane] * f;
                    lsum += slsum[i][col] * f;
                }
            }
        }
        if ((alone || sg == 0) && r < R) {
            const float vs = c.v_scale ? c.v_scale[h] : 1.0f;
            const float inv = lsum == 0.f ? 0.f : __fdiv_rn(vs, lsum);
            const int m = r / c.G, g = r % c.G;
            const u32x2 o = {float2_to_bf16_pair(acc.x * inv, acc.y * inv), float2_to_bf16_pair(acc.z * inv, acc.w * inv)};
            *reinterpret_cast<u32x2 *>(p.out + (a.row0 + m) * p.ldo + ((long long)h * c.G + g) * kHeadDim + 16 * dt + 4 * g4) = o;
        }
    };
    if (units > (int)gridDim.x) {
        for (int u = blockIdx.x * 8 + sg; u < units; u += gridDim.x * 8) unit(std::true_type{}, u);
    } else if ((int)blockIdx.x < units) {
        unit(std::false_type{}, blockIdx.x);
    }
}

}  // namespace quasar
