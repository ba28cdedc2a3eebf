// CPU model of what the kernels take from a paged cache's books: the library's own host and device functions.
#include "../paper_2603_01399_amd/csrc/books.hpp"

using namespace quasar;

extern "C" void span_model(int begin, int end, int len, int T, int *out) {
    const SeqSpan s = span_of(begin, end, len, T);
    out[0] = s.row0; out[1] = s.n; out[2] = s.len;
}
extern "C" int blocks_model(int total, int columns, int block_shift) { return blocks_reached(total, columns, block_shift); }
extern "C" int page_model(int id, int n_pages) { return page_exists(id, n_pages); }
extern "C" void share_model(int total, int workers, int least, int worker, int *out) {
    const FlatShare f = flat_share(total, workers, least, worker);
    out[0] = f.share; out[1] = f.begin; out[2] = f.end;
}
extern "C" int slot_model(int total, int workers, int least, int worker, int seq_begin) {
    return flat_slot(flat_share(total, workers, least, worker), worker, seq_begin);
}
extern "C" int part_slot_model(int worker, int first_slot, int k) { return flat_part_slot(worker, first_slot, k); }
