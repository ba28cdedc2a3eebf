// CPU model of the line of buckets (csrc/token_math.hpp): where a logit lies, the smallest logit of some buckets, the last bucket that min_p asks for.
#include "../paper_2603_01399_amd/csrc/token_math.hpp"

using namespace quasar;

// Buckets of n logits in a row whose largest is `most`.
extern "C" void buckets_model(const float *z, long long n, float most, float temperature, int *out) {
    const Filters f = filters_of(temperature, 0, 1.0f, 0.0f, 1 << 20);
    const auto top = bucket_line(most, f.scale);
    for (long long i = 0; i < n; ++i) out[i] = bucket_of(z[i], f.scale, top);
}
// The smallest logit of buckets 0 .. j, with a wave's ballots in a loop.
extern "C" float least_model(int j, float most, float temperature) {
    const Filters f = filters_of(temperature, 0, 1.0f, 0.0f, 1 << 20);
    return value_of_ordered(least_of_buckets(j, f, bucket_line(most, f.scale), most, [](auto holds) {
        u64 mask = 0;
        for (int i = 0; i < 64; ++i) mask |= (u64)(holds(i) ? 1 : 0) << i;
        return mask;
    }));
}
extern "C" int last_model(float min_p) { return last_bucket(log2f(min_p)); }
extern "C" float least_left_model(float most, float temperature, float min_p) {
    const Filters f = filters_of(temperature, 0, 1.0f, min_p, 1 << 20);
    return least_logit(most, f.rate, f.min_p);
}
