// CPU model of what the windowed kernels read: the library's own host and device functions.
#include "../paper_2603_01399_amd/csrc/books.hpp"

using namespace quasar;

extern "C" int units_model(int size, int sinks, int first, int units, int shift, int *out) {
    const WindowUnits u = window_units(Window{size, sinks}, first, units, shift);
    for (int i = 0; i < u.count; ++i) out[i] = u.at(i);
    return u.count;
}
// -> count; whole[0]: how many of them come first because every row sees them whole
extern "C" int tile_model(int size, int sinks, int first, int last, int units, int shift, int *out, int *whole) {
    const TileUnits t = tile_units(Window{size, sinks}, first, last, units, shift);
    for (int i = 0; i < t.u.count; ++i) out[i] = t.at(i);
    whole[0] = t.whole;
    return t.u.count;
}
extern "C" unsigned int seen_model(int size, int sinks, int pos, int pos0) { return seen_of_block(Window{size, sinks}, pos, pos0); }
extern "C" void columns_model(int size, int sinks, int len, int page_shift, int *out) {
    const Columns c = columns_behind(Window{size, sinks}, len, page_shift);
    out[0] = c.begin; out[1] = c.end;
}
