// What the kernels take from the books of a paged cache, bounded before it is an address, and how a step's blocks are shared among
// workers.  Plain C++ for both sides: the kernels run it on the GPU, the tests run the same functions on the CPU.
#pragma once

#include <stdint.h>

#include "draw.hpp"

namespace quasar {

constexpr int kMaxSeqs = 1024;               // sequences of a batch: their prefix sums live in LDS
constexpr int kMaxPositions = 1 << 24;       // of a sequence, as in the contiguous cache
constexpr int kPositionsPerBlock = 32;

// Rows and cached positions of a sequence: no rows where they do not fit the T packed ones, or the length is none.
struct SeqSpan { int row0, n, len; };
QUASAR_BOTH SeqSpan span_of(int begin, int end, int len, int T) {
    const bool fits = begin >= 0 && end >= begin && end <= T && len >= 0 && len <= kMaxPositions;
    return SeqSpan{fits ? begin : 0, fits ? end - begin : 0, fits ? len : 0};
}

// Blocks of 32 positions that hold positions 0 .. total - 1, as far as a row of the table (columns pages of 1 << block_shift blocks) reaches.
QUASAR_BOTH int blocks_reached(int total, int columns, int block_shift) {
    const int most = columns << block_shift, want = (total + kPositionsPerBlock - 1) / kPositionsPerBlock;
    return want < most ? want : most;
}

QUASAR_BOTH bool page_exists(int id, int n_pages) { return (unsigned int)id < (unsigned int)n_pages; }

// A window: the row at position p sees p - size + 1 .. p and, of what is ahead of those, the first `sinks` positions.
struct Window { int size, sinks; };
constexpr int kMostWindow = 1 << 25;         // of size and sinks: more than any two positions are apart, and sums with positions stay below 2^31
QUASAR_BOTH int window_low(const Window &w, int pos) { return pos >= w.size ? pos - w.size + 1 : 0; }

// What rows at positions `first` and behind see of a sequence of `units` units of 1 << shift positions: units 0 .. head - 1, which hold the
// first positions, and from head + skip on; the i-th of them is unit i, or i + skip from i = head on.  Of units > 0 at least one, the last, so that
// rows that see none of them (a window beyond what the table reaches) are somebody's, who writes their zeros.
struct WindowUnits {
    int head, skip, count;
    QUASAR_BOTH int at(int i) const { return i < head ? i : i + skip; }
};
QUASAR_BOTH WindowUnits window_units(const Window &w, int first, int units, int shift) {
    const int low = window_low(w, first);
    int from = low >> shift, head = ((w.sinks < low ? w.sinks : low) + (1 << shift) - 1) >> shift;
    if (from > units) from = units;
    if (head > from) head = from;
    if (head == 0 && from == units && units > 0) from = units - 1;
    return WindowUnits{head, from - head, units - (from - head)};
}

// The same for a tile of rows at positions first .. last, with the units that every row sees whole, and whose positions are all in the
// windows, ahead of the others: units w0 .. w0 + whole - 1, then the others in order.
struct TileUnits {
    WindowUnits u;
    int w0, whole;
    QUASAR_BOTH int at(int i) const {
        if (i < whole) return w0 + i;
        const int x = u.at(i - whole);
        return x < w0 ? x : x + whole;
    }
};
QUASAR_BOTH TileUnits tile_units(const Window &w, int first, int last, int units, int shift) {
    TileUnits t;
    t.u = window_units(w, first, units, shift);
    const int from = t.u.head + t.u.skip, behind = (first + 1) >> shift;         // (units ahead of `behind` hold no position behind the first row)
    t.w0 = (window_low(w, last) + (1 << shift) - 1) >> shift;
    if (t.w0 < from) t.w0 = from;
    t.whole = (behind < units ? behind : units) - t.w0;
    if (t.whole < 0) t.whole = 0;
    return t;
}

// Positions of a block of 32 from `pos0` on that a row at position `pos` sees, one bit each.
QUASAR_BOTH unsigned int bits_through(int n) { return n < 0 ? 0u : n >= 31 ? ~0u : (2u << n) - 1u; }
QUASAR_BOTH unsigned int seen_of_block(const Window &w, int pos, int pos0) {
    return bits_through(pos - pos0) & (~bits_through(pos - w.size - pos0) | bits_through(w.sinks - 1 - pos0));
}

// Columns of a sequence's table, of pages of 1 << page_shift positions, that no row at position len or behind sees anything of.
struct Columns { int begin, end; };
QUASAR_BOTH Columns columns_behind(const Window &w, int len, int page_shift) {
    return Columns{(w.sinks + (1 << page_shift) - 1) >> page_shift, window_low(w, len) >> page_shift};
}

// The blocks of all sequences as one line, cut into equal pieces for the workers; `least`: blocks that a worker takes at least.
struct FlatShare { int share, begin, end; };
QUASAR_BOTH FlatShare flat_share(int total, int workers, int least, int worker) {
    FlatShare f;
    f.share = (total + workers - 1) / workers;
    if (f.share < least) f.share = least;
    const long long begin = (long long)worker * f.share;
    f.begin = begin < total ? (int)begin : total;
    f.end = total - f.begin < f.share ? total : f.begin + f.share;
    return f;
}
// Where a worker leaves its part of a sequence that it shares: at most one goes on from the worker before (or begins with the piece),
// and at most one begins inside and goes on.
QUASAR_BOTH int flat_slot(const FlatShare &f, int worker, int seq_begin) { return 2 * worker + (seq_begin > f.begin ? 1 : 0); }
// The slot of part k of a sequence whose first part lies in `worker` at `first_slot`.
QUASAR_BOTH int flat_part_slot(int worker, int first_slot, int k) { return k == 0 ? first_slot : 2 * (worker + k); }

}  // namespace quasar
