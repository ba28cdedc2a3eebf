// Drawing tokens from the logits of a batch's rows, with temperature, top-k, top-p and min-p of each (gfx950), and the verification of
// drafts from them (Sec. 3.1, the acceptance and resampling rules, with a deterministic drafter).
//
// All filters keep a beginning of one order, larger logits first and equal ones by their place, so together they are one cut in it.  Sorting a
// vocabulary to find the cut would move it many times; instead
//   token_parts_kernel   reads it once, in parts of 8192 tokens: the largest logit of a part and of its chunks, and how many tokens and what mass lie in each of
//                        512 buckets of 1/16 (in units of the temperature) below the part's largest;
//   token_draw_kernel    a workgroup a row: adds the parts' buckets up, finds the bucket in which a cut falls, gathers that bucket's tokens from the chunks
//                        that can hold some, finds the cut among them digit by digit, and draws: from what each part has left, the part, then the token;
//   token_verify_kernel  drafts: the leading accepted ones of each sequence, and the token that its first refusal (or last row) has drawn.
// Weights are whole numbers (token_math.hpp), sums of them exact, and what is added up in fp64 is added in a fixed order: results are determined by the
// arguments alone.
#pragma once

#include "books.hpp"
#include "quasar_device.hpp"
#include "token_math.hpp"

namespace quasar {

constexpr int kPartTokens = 8192, kPartThreads = 512, kPartWaves = kPartThreads / 64, kPartLane = kPartTokens / kPartThreads;
constexpr int kMaxTokenParts = ((1 << kIndexBits) + 7 + kPartTokens - 1) / kPartTokens;
constexpr int kDrawThreads = 1024, kDrawWaves = kDrawThreads / 64;
constexpr int kListed = 3584;                // tokens of a bucket that are kept in LDS; more are read again where they are asked for

struct TokenParams {
    const void *logits;
    long long ld;
    const float *temperature, *top_p, *min_p;    // of a row, or of a sequence where there are drafts; NULL: 1, no limit, no limit
    const int32_t *top_k;
    const int32_t *row_start, *draft;            // drafts: rows of the sequences, tokens proposed; else NULL
    const float *u_accept, *u;
    int32_t *token;                              // [T]
    float *p;                                    // [T], of the token or of the draft; may be NULL
    int32_t *accepted;                           // [T]: drafts: the row's is accepted
    // of the rows of this launch
    float *part_max, *chunk_max;                 // [rows][nb], [rows][nb][chunks of a part]
    u64 *mass;                                   // [rows][nb][kBuckets]
    unsigned int *count;
    int V, T, n_seqs, nb;
    int row0;                                    // row of the first of them
};

template <int DT> constexpr int lane_tokens = DT == 1 ? 8 : 4;               // of a 16-byte load: bf16, fp32
template <int DT> constexpr int chunk_tokens = 64 * lane_tokens<DT>;         // of a wave's load
template <int DT> constexpr int part_chunks = kPartTokens / chunk_tokens<DT>;

// Whose parameters a row goes by (-1: nobody's row), and whether it is the last of its sequence.
struct RowOf { int who; bool last; };
__device__ __forceinline__ RowOf row_of(const TokenParams &p, int row) {
    if (!p.row_start) return RowOf{row, true};
    const int lane = threadIdx.x & 63;
    int s = 0;
    for (int i = 0; i < p.n_seqs; i += 64) {
        const bool before = i + lane < p.n_seqs && p.row_start[i + lane + 1] <= row;
        s += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    if (s >= p.n_seqs) return RowOf{-1, true};
    const SeqSpan a = span_of(p.row_start[s], p.row_start[s + 1], 0, p.T);
    return row >= a.row0 && row < a.row0 + a.n ? RowOf{s, row == a.row0 + a.n - 1} : RowOf{-1, true};
}
__device__ __forceinline__ Filters filters_at(const TokenParams &p, int who) {
    return filters_of(p.temperature ? p.temperature[who] : 1.0f, p.top_k ? p.top_k[who] : 0, p.top_p ? p.top_p[who] : 1.0f, p.min_p ? p.min_p[who] : 0.0f, p.V);
}

// A row whose first token may lie anywhere: places are counted from the 16-byte border ahead of it.
template <int DT> struct LogitRow {
    const unsigned char *border;
    int skew, V;
    __device__ LogitRow(const TokenParams &p, int row) : V(p.V) {
        constexpr int E = DT == 1 ? 2 : 4;
        const u64 at = reinterpret_cast<u64>(p.logits) + (u64)row * p.ld * E;
        border = reinterpret_cast<const unsigned char *>(at & ~15ull);
        skew = (int)(at & 15) / E;
    }
    __device__ __forceinline__ float one(int v) const {
        if constexpr (DT == 1) return logit_value(bf16_bits_to_float(reinterpret_cast<const uint16_t *>(border)[skew + v]));
        else return logit_value(reinterpret_cast<const float *>(border)[skew + v]);
    }
    // the tokens at places at .. (a whole load); -inf where there are none
    __device__ __forceinline__ void load(int at, float (&x)[lane_tokens<DT>]) const {
        constexpr int N = lane_tokens<DT>;
        if (at >= skew && at + N <= skew + V) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(border + 16ll * (at / N));
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if constexpr (DT == 1) x[e] = logit_value(__uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16));
                else x[e] = logit_value(__uint_as_float(v[e]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = at + e >= skew && at + e < skew + V ? one(at + e - skew) : -__builtin_inff();
        }
    }
};

// the largest over the wave, in every lane
__device__ __forceinline__ float wave_max(float v) {
    auto step = [&](auto ctrl, auto mask) {
        const int o = __builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), decltype(ctrl)::value, decltype(mask)::value, 0xf, false);
        v = fmaxf(v, __int_as_float(o));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});      // from 1, 2, 4 and 8 lanes before, within 16 lanes
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});      // lane 15 to the 16 lanes behind it, lane 47 likewise
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});      // lane 31 to the 32 lanes behind it
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Grid (parts, rows).  A part's 16 tokens a thread stay in registers between its largest logit and the buckets.
template <int DT>
__global__ __launch_bounds__(kPartThreads) void token_parts_kernel(const TokenParams p) {
    constexpr int N = lane_tokens<DT>, LOADS = kPartLane / N, CHUNKS = part_chunks<DT>;
    __shared__ u64 mass[kBuckets];
    __shared__ unsigned int count[kBuckets];
    __shared__ float wave_largest[kPartWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x, r = blockIdx.y;
    const LogitRow<DT> row(p, p.row0 + r);
    float x[LOADS][N];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) row.load(b * kPartTokens + (w * LOADS + i) * chunk_tokens<DT> + lane * N, x[i]);
    const RowOf of = row_of(p, p.row0 + r);
    if (of.who < 0) return;
    const Filters f = filters_at(p, of.who);
    for (int i = tid; i < kBuckets; i += kPartThreads) mass[i] = 0, count[i] = 0;
    float largest = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        float m = x[i][0];
#pragma unroll
        for (int e = 1; e < N; ++e) m = fmaxf(m, x[i][e]);
        m = wave_max(m);
        if (lane == 0) p.chunk_max[((long long)r * p.nb + b) * CHUNKS + w * LOADS + i] = m;
        largest = fmaxf(largest, m);
    }
    if (lane == 0) wave_largest[w] = largest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPartWaves; ++i) largest = fmaxf(largest, wave_largest[i]);
    if (tid == 0) p.part_max[(long long)r * p.nb + b] = largest;
    const float top = bucket_line(largest, f.scale);
    if (largest > -__builtin_inff()) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int at = bucket_of(x[i][e], f.scale, top);
                if (at >= kBuckets) continue;
                atomicAdd(&mass[at], weight_units(x[i][e], largest, f.rate, kPartBits));
                if (f.k) atomicAdd(&count[at], 1u);
            }
    }
    __syncthreads();
    const long long to = ((long long)r * p.nb + b) * kBuckets;
    for (int i = tid; i < kBuckets; i += kPartThreads) {
        p.mass[to + i] = mass[i];
        if (f.k) p.count[to + i] = count[i];
    }
}

// Sum of v over the threads up to each one, of a workgroup of kDrawThreads; wave_sums: [kDrawWaves] of LDS.
template <class N>
__device__ __forceinline__ N sums_through(N v, N *wave_sums) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const N up = __shfl_up(v, off, 64);
        if (lane >= off) v += up;
    }
    __syncthreads();                                             // (wave_sums may still be read from the last call)
    if (lane == 63) wave_sums[w] = v;
    __syncthreads();
    N before = 0;
#pragma unroll
    for (int i = 0; i < kDrawWaves; ++i) before += i < w ? wave_sums[i] : N(0);
    return before + v;
}

// A workgroup a row.
template <int DT>
__global__ __launch_bounds__(kDrawThreads) void token_draw_kernel(const TokenParams p) {
    constexpr int N = lane_tokens<DT>, CHUNKS = part_chunks<DT>;
    constexpr u64 ALL = ~0ull;
    __shared__ double bucket_mass[kBuckets], through_mass[kBuckets];
    __shared__ unsigned int through_count[kBuckets];
    __shared__ u64 list[kListed];                                // rank keys of a bucket's tokens, in no order
    __shared__ u64 bin_mass[kDrawThreads];
    __shared__ unsigned int bin_count[kDrawThreads];
    __shared__ double factor[kMaxTokenParts];                    // of a part's units in the row's
    __shared__ u64 part_mass[kMaxTokenParts];
    __shared__ float part_max[kMaxTokenParts];
    __shared__ int shift[kMaxTokenParts];                        // of a part's buckets in the row's
    __shared__ unsigned short chunks[kMaxTokenParts * CHUNKS];   // that may hold some of the bucket
    __shared__ u64 wave_units[kDrawWaves];
    __shared__ double wave_mass[kDrawWaves];
    __shared__ unsigned int wave_count[kDrawWaves];
    __shared__ int found, n_chunks, n_listed;
    __shared__ u64 chosen[4];
    __shared__ double drawn_total;
    __shared__ int drawn_part;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x, row_at = p.row0 + r;
    const RowOf of = row_of(p, row_at);
    if (of.who < 0) return;
    const Filters f = filters_at(p, of.who);
    const LogitRow<DT> row(p, row_at);
    const int nb = p.nb;

    // ---- the row's largest logit, and how the parts' buckets lie on its line
    float most = -__builtin_inff();
    for (int b = lane; b < nb; b += 64) most = fmaxf(most, p.part_max[(long long)r * nb + b]);
    most = wave_max(most);
    if (!(most > -__builtin_inff())) {                           // nothing to draw from
        if (tid == 0) {
            p.token[row_at] = -1;
            if (p.p) p.p[row_at] = 0.0f;
            if (p.accepted) p.accepted[row_at] = 0;
        }
        return;
    }
    const float top = bucket_line(most, f.scale);
    for (int b = tid; b < nb; b += kDrawThreads) {
        const float m = p.part_max[(long long)r * nb + b];
        part_max[b] = m;
        shift[b] = bucket_of(m, f.scale, top);
        factor[b] = m > -__builtin_inff() ? weight_of(m, most, f.rate) : 0.0;
    }
    __syncthreads();

    // ---- buckets of the row: count and mass of each, and through it
    {
        const int j = tid % kBuckets;
        double mass = 0.0;
        unsigned int count = 0;
        for (int b = tid / kBuckets; b < nb; b += kDrawThreads / kBuckets) {
            const int from = j - shift[b];
            if (from < 0) continue;
            const long long at = ((long long)r * nb + b) * kBuckets + from;
            mass += (double)p.mass[at] * (factor[b] * (1.0 / (double)(1ull << kPartBits)));
            if (f.k) count += p.count[at];
        }
        reinterpret_cast<double *>(bin_mass)[tid] = mass;
        bin_count[tid] = count;
        __syncthreads();
        mass = 0.0;
        count = 0;
        if (tid < kBuckets) {
            mass = reinterpret_cast<double *>(bin_mass)[tid] + reinterpret_cast<double *>(bin_mass)[tid + kBuckets];
            count = bin_count[tid] + bin_count[tid + kBuckets];
        }
        const double mass_through = sums_through(mass, wave_mass);
        const unsigned int count_through = sums_through(count, wave_count);
        if (tid < kBuckets) bucket_mass[tid] = mass, through_mass[tid] = mass_through, through_count[tid] = count_through;
        __syncthreads();
    }

    // The tokens of a bucket: their keys into the list, as many as it takes; how many.
    auto each_of_chunks = [&](int bucket, auto body) {
        for (int q0 = w; q0 < n_chunks; q0 += 4 * kDrawWaves) {
            float x[4][N];
            int at[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                at[i] = q0 + i * kDrawWaves < n_chunks ? chunks[q0 + i * kDrawWaves] * chunk_tokens<DT> + lane * N : -1;
                if (at[i] >= 0) row.load(at[i], x[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (at[i] >= 0 && bucket_of(x[i][e], f.scale, top) == bucket) body(rank_key(x[i][e], at[i] + e - row.skew));
        }
    };
    int listed_bucket = -1;
    auto gather = [&](int bucket) {
        if (tid == 0) n_chunks = 0, n_listed = 0;
        __syncthreads();
        for (int i = tid; i < nb * CHUNKS; i += kDrawThreads)
            if (bucket_of(p.chunk_max[(long long)r * nb * CHUNKS + i], f.scale, top) <= bucket) chunks[atomicAdd(&n_chunks, 1)] = (unsigned short)i;
        __syncthreads();
        each_of_chunks(bucket, [&](u64 key) {
            const int at = atomicAdd(&n_listed, 1);
            if (at < kListed) list[at] = key;
        });
        __syncthreads();
        listed_bucket = bucket;
    };
    auto each = [&](auto body) {                                 // of the gathered bucket
        if (n_listed <= kListed) {
            for (int i = tid; i < n_listed; i += kDrawThreads) body(list[i]);
        } else {
            each_of_chunks(listed_bucket, body);
        }
    };
    // Of the gathered bucket's tokens up to `cut`, in their order: the first `need` (by_mass: those ahead of which less than `limit` of the row's mass
    // lies).  The last of them becomes the cut; their mass.  A digit of ten bits of the keys at a time, until one token is left: keys differ.
    auto select = [&](bool by_mass, unsigned int need, double limit, u64 &cut) {
        u64 lo = ALL, hi = 0;
        each([&](u64 key) {
            if (key > cut) return;
            lo = key < lo ? key : lo;
            hi = key > hi ? key : hi;
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            const u64 a = __shfl_xor(lo, off, 64), b = __shfl_xor(hi, off, 64);
            lo = a < lo ? a : lo;
            hi = b > hi ? b : hi;
        }
        if (lane == 0) bin_mass[w] = lo, bin_mass[kDrawWaves + w] = hi;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kDrawWaves; ++i) {
            lo = bin_mass[i] < lo ? bin_mass[i] : lo;
            hi = bin_mass[kDrawWaves + i] > hi ? bin_mass[kDrawWaves + i] : hi;
        }
        if (lo > hi) return 0.0;                                 // (no token: nothing is cut)
        const float ref = key_value(lo);
        const double to_row = weight_of(ref, most, f.rate) * (1.0 / (double)(1ull << kListBits));
        const double units = __builtin_ceil(limit / to_row);
        const u64 want = by_mass ? (units < 1.0 ? 1ull : units < 0x1p62 ? (u64)units : 1ull << 62) : ALL;
        u64 mass_before = 0;
        unsigned int count_before = 0;
        for (;;) {
            const u64 span = hi - lo;
            const int digit = span < kDrawThreads ? 0 : 54 - __builtin_clzll(span);
            __syncthreads();
            bin_mass[tid] = 0;
            bin_count[tid] = 0;
            if (tid == 0) found = kDrawThreads, chosen[3] = 0;
            __syncthreads();
            each([&](u64 key) {
                if (key < lo || key > hi) return;
                const int at = (int)((key - lo) >> digit);
                atomicAdd(&bin_count[at], 1u);
                atomicAdd(&bin_mass[at], weight_units(key_value(key), ref, f.rate, kListBits));
            });
            __syncthreads();
            const u64 mass = bin_mass[tid];
            const unsigned int count = bin_count[tid];
            const u64 mass_through = mass_before + sums_through(mass, wave_units);
            const unsigned int count_through = count_before + sums_through(count, wave_count);
            if (count) {
                if (by_mass ? mass_through >= want : count_through >= need) atomicMin(&found, tid);
                atomicMax(&chosen[3], (u64)tid + 1);             // (none reaches it: the last that holds any)
            }
            __syncthreads();
            const int bin = found < kDrawThreads ? found : (int)chosen[3] - 1;
            if (tid == bin) chosen[0] = mass_through, chosen[1] = mass, chosen[2] = (u64)count_through << 32 | count;
            __syncthreads();
            const u64 end = lo + ((u64)(bin + 1) << digit) - 1;
            hi = end < hi ? end : hi;
            const unsigned int inside = (unsigned int)chosen[2];
            if (inside <= 1 || digit == 0) {
                cut = hi;
                return (double)chosen[0] * to_row;
            }
            lo += (u64)bin << digit;
            mass_before = chosen[0] - chosen[1];
            count_before = (unsigned int)(chosen[2] >> 32) - inside;
        }
    };
    // The first bucket below `limit` that a condition holds for, or `limit`.
    auto first_bucket = [&](int limit, auto holds) {
        if (tid == 0) found = limit;
        __syncthreads();
        if (tid < limit && holds(tid)) atomicMin(&found, tid);
        __syncthreads();
        const int at = found;
        __syncthreads();
        return at;
    };

    // ---- the cut
    u64 cut = ALL;
    int border = kBuckets;                                       // the bucket in which it lies
    double total = through_mass[kBuckets - 1];
    if (f.k) {
        const int at = first_bucket(kBuckets, [&](int j) { return through_count[j] >= (unsigned int)f.k; });
        if (at < kBuckets) {                                     // (else what is beyond the buckets has no mass)
            gather(at);
            border = at;
            total = (at ? through_mass[at - 1] : 0.0) + select(false, (unsigned int)f.k - (at ? through_count[at - 1] : 0u), 0.0, cut);
        }
    }
    if (f.p < 1.0f) {
        const double target = (double)f.p * total;
        const int at = first_bucket(border, [&](int j) { return bucket_mass[j] > 0.0 && through_mass[j] >= target; });
        if (at < kBuckets) {
            if (listed_bucket != at) gather(at);
            border = at;
            select(true, 0u, target - (through_mass[at] - bucket_mass[at]), cut);
        }
    }
    if (f.min_p > 0.0f) {
        const float least = least_logit(most, f.rate, f.min_p);
        const u64 key = rank_key(least, (1 << kIndexBits) - 1);
        if (key < cut) {
            cut = key;
            border = bucket_of(least, f.scale, top);
        }
    }
    auto kept = [&](float z, int v) {
        const int at = bucket_of(z, f.scale, top);
        return at < border || (at == border && at < kBuckets && rank_key(z, v) <= cut);
    };

    // ---- what is left of each part
    __syncthreads();
    for (int b = w; b < nb; b += kDrawWaves) {
        u64 sum = 0;
        for (int j = lane; j < border - shift[b]; j += 64) sum += p.mass[((long long)r * nb + b) * kBuckets + j];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if (lane == 0) part_mass[b] = sum;
    }
    if (border < kBuckets) {
        if (listed_bucket != border) gather(border);
        __syncthreads();
        each([&](u64 key) {
            if (key > cut) return;
            const int b = (key_token(key) + row.skew) / kPartTokens;
            atomicAdd(&part_mass[b], weight_units(key_value(key), part_max[b], f.rate, kPartBits));
        });
    }
    __syncthreads();
    int banned = -1;
    if (tid == 0) {
        double whole = 0.0;
        for (int b = 0; b < nb; ++b) whole += (double)part_mass[b] * factor[b];
        if (p.draft) {
            const int d = p.draft[row_at];
            double of_draft = 0.0;
            if (!of.last && d >= 0 && d < p.V) {
                const float z = row.one(d);
                if (kept(z, d)) {
                    const int b = (d + row.skew) / kPartTokens;
                    const u64 units = weight_units(z, part_max[b], f.rate, kPartBits);
                    of_draft = (double)units * factor[b] / whole;
                    part_mass[b] -= units;                       // what a refusal draws from
                }
                banned = d;
                whole = 0.0;
                for (int b = 0; b < nb; ++b) whole += (double)part_mass[b] * factor[b];
            } else if (d >= 0 && d < p.V && kept(row.one(d), d)) {
                const int b = (d + row.skew) / kPartTokens;
                of_draft = (double)weight_units(row.one(d), part_max[b], f.rate, kPartBits) * factor[b] / whole;
            }
            if (p.p) p.p[row_at] = (float)of_draft;
            p.accepted[row_at] = !of.last && (double)p.u_accept[row_at] < of_draft;
        }
        // the part that the draw falls in: the first whose running mass exceeds it, else the last that has any
        const float u = p.u[row_at];
        const double target = u > 0.0f ? (double)u * whole : 0.0;
        double through = 0.0, ahead = 0.0;
        int part = -1;
        for (int b = 0; b < nb; ++b) {
            if (!part_mass[b]) continue;
            part = b;
            ahead = through;
            through += (double)part_mass[b] * factor[b];
            if (through > target) break;
        }
        u64 units = 0;
        if (part >= 0) {
            const double left = (target - ahead) / factor[part];
            units = left > 0.0 ? (left < 0x1p62 ? (u64)left : 1ull << 62) : 0;
            if (units >= part_mass[part]) units = part_mass[part] - 1;
        }
        drawn_part = part;
        drawn_total = whole;
        chosen[0] = units;
        chosen[1] = (u64)(banned + 1);
    }
    __syncthreads();
    const int part = drawn_part;
    if (part < 0) {                                              // (all mass was the draft's)
        if (tid == 0) {
            p.token[row_at] = -1;
            if (p.p && !p.draft) p.p[row_at] = 0.0f;
        }
        return;
    }
    // ---- the token: eight places a thread, in order
    banned = (int)chosen[1] - 1;
    const u64 ahead = chosen[0];
    float x[kPartTokens / kDrawThreads / N][N];
    const int at0 = part * kPartTokens + tid * (kPartTokens / kDrawThreads);
    u64 units[kPartTokens / kDrawThreads], sum = 0;
#pragma unroll
    for (int i = 0; i < kPartTokens / kDrawThreads / N; ++i) row.load(at0 + i * N, x[i]);
#pragma unroll
    for (int i = 0; i < kPartTokens / kDrawThreads; ++i) {
        const int v = at0 + i - row.skew;
        const float z = x[i / N][i % N];
        units[i] = kept(z, v) && v != banned ? weight_units(z, part_max[part], f.rate, kPartBits) : 0;
        sum += units[i];
    }
    const u64 through = sums_through(sum, wave_units);
    if (through > ahead && through - sum <= ahead) {
        u64 at = through - sum;
#pragma unroll
        for (int i = 0; i < kPartTokens / kDrawThreads; ++i) {
            if (at <= ahead && at + units[i] > ahead) {
                p.token[row_at] = at0 + i - row.skew;
                if (p.p && !p.draft) p.p[row_at] = (float)((double)units[i] * factor[part] / drawn_total);
            }
            at += units[i];
        }
    }
}

// A wave a sequence: how many of its drafts are accepted ahead of the first refusal, and what the row behind them has drawn.
__global__ __launch_bounds__(256) void token_verify_kernel(const int32_t *row_start, int n_seqs, int T, const int32_t *accepted, const int32_t *token,
                                                           int32_t *out_accept_len, int32_t *out_token) {
    const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (s >= n_seqs) return;
    const SeqSpan a = span_of(row_start[s], row_start[s + 1], 0, T);
    int n = 0;
    for (; n < a.n; n += 64) {
        const bool goes_on = n + lane < a.n && accepted[a.row0 + n + lane] != 0;
        const unsigned long long stops = ~__builtin_amdgcn_ballot_w64(goes_on);
        if (stops) {
            n += __builtin_ctzll(stops);
            break;
        }
    }
    if (lane == 0) {
        out_accept_len[s] = a.n ? n : 0;
        out_token[s] = a.n ? token[a.row0 + n] : -1;
    }
}

}  // namespace quasar
