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
