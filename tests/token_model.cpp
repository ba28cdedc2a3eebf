// CPU model of the arithmetic behind a draw: the library's own host and device functions.
#include "../paper_2603_01399_amd/csrc/token_math.hpp"

using namespace quasar;

extern "C" double weight_model(float z, float ref, double rate) { return weight_of(z, ref, rate); }
extern "C" u64 units_model(float z, float ref, double rate, int bits) { return weight_units(z, ref, rate, bits); }
extern "C" float value_model(float z) { return logit_value(z); }
extern "C" u64 key_model(float z, int v, int bf16) { return bf16 ? rank_key<1>(z, v) : rank_key<0>(z, v); }
extern "C" float key_value_model(u64 key, int bf16) { return bf16 ? key_value<1>(key) : key_value<0>(key); }
extern "C" u64 first_key_model(float most, int bf16) { return bf16 ? first_key<1>(ordered_bits(most)) : first_key<0>(ordered_bits(most)); }
extern "C" u64 last_key_model(float least, int bf16) { return bf16 ? last_key<1>(ordered_bits(least)) : last_key<0>(ordered_bits(least)); }
extern "C" int key_token_model(u64 key) { return key_token(key); }
extern "C" int bucket_model(float z, float scale, float most) { return bucket_of(z, scale, bucket_line(most, scale)); }
extern "C" float least_model(float most, double rate, float min_p) { return least_logit(most, rate, min_p); }
extern "C" void filters_model(float t, int k, float p, float min_p, int V, double *out) {
    const Filters f = filters_of(t, k, p, min_p, V);
    out[0] = f.rate; out[1] = f.scale; out[2] = f.k; out[3] = f.p; out[4] = f.min_p;
}
