// Drawing tokens from the logits of a batch's rows, with temperature, top-k, top-p and min-p of each (gfx950), and the verification of
// drafts from them (Sec. 3.1, the acceptance and resampling rules, with a deterministic drafter).
//
// All filters keep a beginning of one order, larger logits first and equal ones by their place, so together they are one cut in it.  Sorting a
// vocabulary to find the cut would move it many times; instead
//   token_parts_kernel   reads it once, in parts of 8192 tokens: the largest logit of a part and of its chunks, and how many tokens and what mass lie in each of
//                        512 buckets of 1/16 (in units of the temperature) below the part's largest;
//   token_draw_kernel    a workgroup a row: adds the parts' buckets up, finds the bucket in which a cut falls, gathers that bucket's tokens from the chunks
//                        that can hold some, finds the cut among them digit by digit, and draws: from what each part has left, the part, then the token;
//                        Of a sequence's rows with drafts the workgroup that is done last says how many of them are accepted, and what the row behind them has drawn.
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
constexpr int kChunkTurn = 16;               // chunks that a wave reads at a time
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
    // drafts: a row's is accepted [T]; rows of a sequence that are done, and what it comes to [n_seqs]
    int32_t *accepted, *done, *out_accept_len, *out_token;
    // of the rows of this launch
    float *part_max, *chunk_max;                 // [rows][nb], [rows][nb][chunks of a part]
    u64 *mass;                                   // [rows][nb][kBuckets]
    unsigned int *count;
    int V, T, n_seqs, nb;
    int row0;                                    // row of the first of them
};

template <int DT> constexpr int lane_tokens = DT == 1 ? 8 : 4;               // of a 16-byte load: bf16, fp32
template <int DT> constexpr int chunk_tokens = 16 * lane_tokens<DT>;         // of sixteen lanes' load: whose largest logit is kept
template <int DT> constexpr int part_chunks = kPartTokens / chunk_tokens<DT>;

// Whose parameters a row goes by (-1: nobody's row), and the rows of its sequence.
struct RowOf {
    int who, row0, n;
    __device__ bool last(int row) const { return row == row0 + n - 1; }
};
__device__ __forceinline__ RowOf row_of(const TokenParams &p, int row) {
    if (!p.row_start) return RowOf{row, row, 1};
    const int lane = threadIdx.x & 63;
    int s = 0;
    for (int i = 0; i < p.n_seqs; i += 64) {
        const bool before = i + lane < p.n_seqs && p.row_start[i + lane + 1] <= row;
        s += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    if (s >= p.n_seqs) return RowOf{-1, 0, 0};
    const SeqSpan a = span_of(p.row_start[s], p.row_start[s + 1], 0, p.T);
    return RowOf{row >= a.row0 && row < a.row0 + a.n ? s : -1, a.row0, a.n};
}
__device__ __forceinline__ Filters filters_at(const TokenParams &p, int who) {
    return filters_of(p.temperature ? p.temperature[who] : 1.0f, p.top_k ? p.top_k[who] : 0, p.top_p ? p.top_p[who] : 1.0f, p.min_p ? p.min_p[who] : 0.0f, p.V);
}

// A row whose first token may lie anywhere: places are counted from the 16-byte border ahead of it, in units of 16 bytes.  Requests are made by every
// lane, without a branch, so that many are under way together: a unit that is not whole, or not there, asks for the nearest whole one, and what it has is
// read one by one where the request is used (two units of a row at most have some).
template <int DT> struct LogitRow {
    static constexpr int N = lane_tokens<DT>;
    const unsigned char *border;
    int skew, V, first, last;                                    // first and last whole unit; last < first: none
    __device__ LogitRow(const TokenParams &p, int row) : V(p.V) {
        constexpr int E = DT == 1 ? 2 : 4;
        const u64 at = reinterpret_cast<u64>(p.logits) + (u64)row * p.ld * E;
        border = reinterpret_cast<const unsigned char *>(at & ~15ull);
        skew = (int)(at & 15) / E;
        first = skew ? 1 : 0;
        last = (skew + V) / N - 1;
    }
    __device__ __forceinline__ float one(int v) const {
        if constexpr (DT == 1) return logit_value(bf16_bits_to_float(reinterpret_cast<const uint16_t *>(border)[skew + v]));
        else return logit_value(reinterpret_cast<const float *>(border)[skew + v]);
    }
    __device__ __forceinline__ u32x4 request(int unit) const {
        if (last < first) return u32x4{0u, 0u, 0u, 0u};          // (the same for every lane)
        return *reinterpret_cast<const u32x4 *>(border + (unsigned int)(16 * min(max(unit, first), last)));    // (a row has at most 4 MB)
    }
    // the tokens of a requested unit as form(logit) has them; -inf where there are none
    template <class Form>
    __device__ __forceinline__ void as_whole(const u32x4 v, float (&x)[N], Form form) const {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float z = DT == 1 ? __uint_as_float(e & 1 ? v[DT == 1 ? e >> 1 : 0] & 0xFFFF0000u : v[DT == 1 ? e >> 1 : 0] << 16) : __uint_as_float(v[e & 3]);
            x[e] = form(z);
        }
    }
    template <class Form> __device__ __forceinline__ void values(int unit, const u32x4 v, float (&x)[N], Form form) const {
        as_whole(v, x, form);
        if (!whole(unit)) at_end(unit, x);
    }
    __device__ __forceinline__ bool whole(int unit) const { return unit >= first && unit <= last; }
    __device__ __forceinline__ bool partial(int unit) const { return !whole(unit) && unit * N < skew + V; }     // (unit 0 has the row's first place, if any)
    __device__ __forceinline__ void at_end(int unit, float (&x)[N]) const {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int at = unit * N + e;
            x[e] = at >= skew && at < skew + V ? one(at - skew) : -__builtin_inff();
        }
    }
};

// v of the lanes up to each one combined by op, whose neutral value is `none`: within 16 lanes, then from their last lanes on.
template <int CTRL, int ROWS, class N>
__device__ __forceinline__ N from_lane(N v, N none) {
    if constexpr (sizeof(N) == 4) {
        return __builtin_bit_cast(N, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    } else {
        const u32x2 x = __builtin_bit_cast(u32x2, v), o = __builtin_bit_cast(u32x2, none);
        return __builtin_bit_cast(N, u32x2{(unsigned int)__builtin_amdgcn_update_dpp((int)o.x, (int)x.x, CTRL, ROWS, 0xf, false),
                                           (unsigned int)__builtin_amdgcn_update_dpp((int)o.y, (int)x.y, CTRL, ROWS, 0xf, false)});
    }
}
template <bool ALL_LANES, class N, class Op>
__device__ __forceinline__ N lanes_through(N v, N none, Op op) {
    v = op(v, from_lane<0x111, 0xf>(v, none));
    v = op(v, from_lane<0x112, 0xf>(v, none));
    v = op(v, from_lane<0x114, 0xf>(v, none));
    v = op(v, from_lane<0x118, 0xf>(v, none));
    if constexpr (ALL_LANES) {
        v = op(v, from_lane<0x142, 0xa>(v, none));
        v = op(v, from_lane<0x143, 0xc>(v, none));
    }
    return v;
}
template <class N> __device__ __forceinline__ N lane_sums_through(N v) {
    return lanes_through<true>(v, N(0), [](N a, N b) { return a + b; });
}
template <class N> __device__ __forceinline__ N of_lane(N v, int lane) {
    if constexpr (sizeof(N) == 4) {
        return __builtin_bit_cast(N, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const u32x2 x = __builtin_bit_cast(u32x2, v);
        return __builtin_bit_cast(N, u32x2{(unsigned int)__builtin_amdgcn_readlane((int)x.x, lane), (unsigned int)__builtin_amdgcn_readlane((int)x.y, lane)});
    }
}
__device__ __forceinline__ float wave_max(float v) {             // in every lane
    return of_lane(lanes_through<true>(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); }), 63);
}
template <class N> __device__ __forceinline__ N wave_sum(N v) { return of_lane(lane_sums_through(v), 63); }

// How a row is drawn.  FIRST: the first token is all that is left.  ALL: nothing is filtered.  FEW: top-k of at most kFew, so that all that is left can be gathered.  MANY: a cut anywhere.
enum { DRAW_ALL = 0, DRAW_FEW = 1, DRAW_MANY = 2, DRAW_FIRST = 3 };
constexpr int kFew = 2048;
__device__ __forceinline__ int draw_mode(const Filters &f) {
    if (f.k == 1) return DRAW_FIRST;
    if (f.k && f.k <= kFew) return DRAW_FEW;
    return f.k || f.p < 1.0f || f.min_p > 0.0f ? DRAW_MANY : DRAW_ALL;
}

// Grid (parts, rows).  A part's 16 tokens a thread stay in registers between its largest logit and the buckets.  What the row asks for is counted and nothing
// else: nothing (FIRST), the whole part's mass (ALL), counts (FEW), masses, and counts where there is a top-k (MANY).  Bound by instructions: a compute unit does one for 64 tokens a
// cycle, 0.25 us for each that is done for every token of 64 rows of 152 K; vector instructions fill 79 to 88 % of the cycles.  64 rows more of fp32 logits take 7.0 us
// (FEW: 39 MB, 5.6 TB/s), 10.8 (ALL) and 13.9 (MANY).  Tried: two, four or eight copies of the buckets in LDS for the lanes of a wave, fewer workgroups a compute unit,
// so that some load while others compute: the same; 256 threads of 32 tokens 2 to 4 us more, 1024 of 8 up to 4 more where there are many rows.
template <int DT>
__global__ __launch_bounds__(kPartThreads) void token_parts_kernel(const TokenParams p) {
    constexpr int N = lane_tokens<DT>, LOADS = kPartLane / N, CHUNKS = part_chunks<DT>;
    __shared__ u64 mass[kBuckets];
    __shared__ unsigned int count[kBuckets];
    __shared__ float wave_largest[kPartWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x, r = blockIdx.y;
    const LogitRow<DT> row(p, p.row0 + r);
    u32x4 raw[LOADS];
    auto unit = [&](int i) { return b * (kPartTokens / N) + (w * LOADS + i) * 64 + lane; };
#pragma unroll
    for (int i = 0; i < LOADS; ++i) raw[i] = row.request(unit(i));
    if (p.row_start && b == 0 && p.row0 + r == 0)                // (what sequences come to that no rows speak for)
        for (int s = tid; s < p.n_seqs; s += kPartThreads) p.out_accept_len[s] = 0, p.out_token[s] = -1, p.done[s] = 0;
    const RowOf of = row_of(p, p.row0 + r);
    if (of.who < 0) return;
    const Filters f = filters_at(p, of.who);
    float x[LOADS][N];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) row.values(unit(i), raw[i], x[i], [](float z) { return logit_weighed(z); });
    const int mode = draw_mode(f);
    const bool counts = f.k != 0, masses = mode == DRAW_MANY;
    static_assert(kBuckets == kPartThreads, "a bucket a thread");
    mass[tid] = 0;
    count[tid] = 0;
    float largest = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        float m = x[i][0];
#pragma unroll
        for (int e = 1; e < N; ++e) m = fmaxf(m, x[i][e]);
        m = lanes_through<false>(m, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
        if ((lane & 15) == 15) p.chunk_max[((long long)r * p.nb + b) * CHUNKS + (w * LOADS + i) * 4 + (lane >> 4)] = m;
        largest = fmaxf(largest, m);
    }
    largest = wave_max((lane & 15) == 15 ? largest : -__builtin_inff());
    if (lane == 0) wave_largest[w] = largest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPartWaves; ++i) largest = fmaxf(largest, wave_largest[i]);
    if (tid == 0) p.part_max[(long long)r * p.nb + b] = largest + 0.0f;      // (as it is ordered: one zero)
    if (mode == DRAW_FIRST) return;
    const double top = bucket_line(largest, f.scale);
    const long long to = ((long long)r * p.nb + b) * kBuckets;
    // (a token that min_p keeps from being left in its part cannot be left in the row; where top-p counts it for the whole all the same, it is taken)
    int last = kBuckets - 1;
    if (mode == DRAW_MANY && !counts && f.p >= 1.0f) last = last_bucket(__log2f(f.min_p));
    if (mode == DRAW_ALL) {
        u64 whole = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) whole += weight_units<true>(x[i][e], largest, f.rate, kPartBits);
        whole = wave_sum(whole);
        if (lane == 0) mass[w] = whole;
        __syncthreads();
        if (tid == 0) {
            for (int i = 1; i < kPartWaves; ++i) whole += mass[i];
            p.mass[to] = whole;
        }
        return;
    }
    if (largest > -__builtin_inff()) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int at = bucket_of(x[i][e], f.scale, top);
                if (at > last) continue;
                if (masses) atomicAdd(&mass[at], weight_units<true>(x[i][e], largest, f.rate, kPartBits));
                if (counts) atomicAdd(&count[at], 1u);
            }
    }
    __syncthreads();
    if (masses) p.mass[to + tid] = mass[tid];
    if (counts) p.count[to + tid] = count[tid];
}

// What the waves of a workgroup tell each other: a value a wave, combined by every wave.  One barrier: the places are taken in turn, and a place comes again
// only behind another's barrier.
constexpr int kTurns = 4;
struct WaveTalk {
    u64 (*places)[kDrawWaves];                                   // [kTurns] of LDS
    int turn;
    template <class N> __device__ __forceinline__ N told(N v) {                  // lane i: what wave i % kDrawWaves has said
        static_assert(kDrawWaves == 16, "sixteen lanes");
        N *place = reinterpret_cast<N *>(places[turn]);
        turn = (turn + 1) % kTurns;
        if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = v;
        __syncthreads();
        return place[threadIdx.x & 15];
    }
    template <class N, class Op> __device__ __forceinline__ N all(N v, N none, Op op) {        // v: the wave's
        return of_lane(lanes_through<false>(told(v), none, op), 15);
    }
    // sum of v over the threads up to this one
    template <class N> __device__ __forceinline__ N sum_through(N v) {
        v = lane_sums_through(v);
        const N other = told(of_lane(v, 63));
        const bool ahead = (int)(threadIdx.x & 15) < __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return v + of_lane(lanes_through<false>(ahead ? other : N(0), N(0), [](N a, N b) { return a + b; }), 15);
    }
    template <class N> __device__ __forceinline__ N sum(N v) {
        return all(wave_sum(v), N(0), [](N a, N b) { return a + b; });
    }
    // the first thread that a holds for (kDrawThreads: none), and the last that b holds for (-1).  (By ballots: what many threads add to one place in LDS is
    // added one after the other, ten cycles each.)
    __device__ __forceinline__ void ends(bool a, bool b, int &first, int &last) {
        const unsigned long long as = __builtin_amdgcn_ballot_w64(a), bs = __builtin_amdgcn_ballot_w64(b);
        const int w = threadIdx.x >> 6;
        const unsigned int f = as ? kDrawThreads - (64 * w + __builtin_ctzll(as)) : 0, l = bs ? 64 * w + 64 - __builtin_clzll(bs) : 0;
        const unsigned int r = all(f << 16 | l, 0u, [](unsigned int x, unsigned int y) {
            return max(x & 0xFFFF0000u, y & 0xFFFF0000u) | max(x & 0xFFFFu, y & 0xFFFFu);
        });
        first = kDrawThreads - (int)(r >> 16);
        last = (int)(r & 0xFFFFu) - 1;
    }
};

__device__ __forceinline__ uint32_t least_ordered_of_bucket(int j, const Filters &f, double top, float most) {
    const int lane = threadIdx.x & 63;
    return least_of_buckets(j, f, top, most, [&](auto holds) { return (u64)__builtin_amdgcn_ballot_w64(holds(lane)); });
}

// A workgroup a row.  Two things bound it.  It is a chain of steps that each wait for the one before (a trip to memory 1 us, a barrier of sixteen waves 0.2): requests are made
// together and ahead, and no step is one thread's.  And a compute unit does one instruction for 64 tokens a cycle, 1 us for each that is done for every token of
// 152 K: what chunks hold is compared with the ends of the gathered buckets, two instructions, and only what lies between is worked on.  One row of 152 K tokens takes
// 7 us without filters (where the first is all that is left a call takes 6.6), 13 to 16 with top-k, and 34 with a top-p whose cut lies in a bucket of thousands, where every chunk is read: buckets 7, chunks 10, their keys and the
// digits 8, the rest 9.  Tried: two to eight workgroups that read such a row's chunks together and the last of which goes on: what each has to make visible to the others
// costs more than it reads (64 rows with top-p 52 us, 61 by two, 69 by four).  A thread has 128 vector registers: of bf16 logits three are spilled, of fp32 ones one, and 41 to 43 scalar
// ones lie in lanes of vector ones.
template <int DT>
__global__ __launch_bounds__(kDrawThreads) void token_draw_kernel(const TokenParams p) {
    constexpr int N = lane_tokens<DT>, CHUNKS = part_chunks<DT>;
    constexpr int AHEAD = 4;                                     // chunks' largest logits of a thread that are requested at the start: of vocabularies up to 2^18 or 2^19 all
    // Loads of a turn of a wave that reads chunks (a bit a token: 32 at most); two turns are under way.  (fp32 logits with six: 18 vector registers spilled, one row with top-k
    // 20.3 us, 64 with top-k 37.5 and with top-p 59.6; with four none, 19.4, 34.7 and 56.9.)
    constexpr int DEPTH = 4;
    constexpr u64 ALL = ~0ull;
    constexpr int kPairs = 128;                                  // tokens up to which each is compared with each (of 16 bytes from LDS a pair: 512 tokens take 15 us, a digit 3)
    extern __shared__ unsigned short chunks[];                   // that may hold some of the gathered buckets
    __shared__ double bucket_mass[kBuckets], through_mass[kBuckets];
    __shared__ unsigned int through_count[kBuckets];
    __shared__ u64 list[kListed];                                // rank keys of the gathered tokens, in no order
    __shared__ u64 bin_mass[kDrawThreads];
    __shared__ unsigned int bin_count[kDrawThreads];
    __shared__ u64 edge[kPairs + 16];                                //  those among which the cut lies
    __shared__ double factor[kMaxTokenParts];                    // of a part's units in the row's
    __shared__ u64 part_mass[kMaxTokenParts];
    __shared__ float part_max[kMaxTokenParts];
    __shared__ int shift[kMaxTokenParts];                        // of a part's buckets in the row's
    __shared__ u64 talk_places[kTurns][kDrawWaves];
    __shared__ int n_chunks, n_listed, n_edge;
    __shared__ u64 chosen[3];
    __shared__ double drawn_total;
    __shared__ int drawn_part, drawn_banned, drawn_token;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x, row_at = p.row0 + r;
    const int nb = p.nb, maxima = nb * CHUNKS;
    const LogitRow<DT> row(p, row_at);
    auto chunk_max_at = [&](int i) {
        const int at = tid + i * kDrawThreads;
        return at < maxima ? p.chunk_max[(long long)r * maxima + at] : -__builtin_inff();
    };
    float chunk_max[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) chunk_max[i] = chunk_max_at(i);
    float most = -__builtin_inff();
    for (int b = lane; b < nb; b += 64) most = fmaxf(most, p.part_max[(long long)r * nb + b]);
    const float mine_max = tid < nb ? p.part_max[(long long)r * nb + tid] : -__builtin_inff();
    const u64 mine_mass = tid < nb ? p.mass[((long long)r * nb + tid) * kBuckets] : 0;           // (of the whole part in DRAW_ALL)
    const float u_at = p.u[row_at];
    const int draft = p.draft ? p.draft[row_at] : -1;
    const float u_accept = p.draft ? p.u_accept[row_at] : 0.0f;
    const RowOf of = row_of(p, row_at);
    if (of.who < 0) return;
    const bool last_row = of.last(row_at);
    Filters f = filters_at(p, of.who);
    f.scale = of_lane(f.scale, 0);                               // (into scalar registers, as the place below)
    const int mode = draw_mode(f);
    WaveTalk talk{talk_places, 0};

    // ---- the row's largest logit, and how the parts' buckets lie on its line
    most = wave_max(most);
    // The row is done.  Drafts: the last of a sequence's rows to be done finds how many of them are accepted ahead of the first that is not.
    auto finish = [&](int token, bool accepted) {                // (thread 0's arguments)
        if (!p.row_start) {
            if (tid == 0) p.token[row_at] = token;
            return;
        }
        if (tid == 0) {
            p.token[row_at] = token;
            p.accepted[row_at] = accepted;
            n_edge = __hip_atomic_fetch_add(&p.done[of.who], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == of.n - 1;
        }
        __syncthreads();
        if (!n_edge || w) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        int n = 0, drawn = -1;
        for (; n < of.n; n += 64) {
            const int at = of.row0 + min(n + lane, of.n - 1);
            const int candidate = __hip_atomic_load(&p.token[at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const int goes_on = __hip_atomic_load(&p.accepted[at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const unsigned long long stops = __builtin_amdgcn_ballot_w64(n + lane >= of.n || !goes_on);
            if (stops) {                                         // (a sequence's last row never goes on)
                drawn = __builtin_amdgcn_readlane(candidate, __builtin_ctzll(stops));
                n += __builtin_ctzll(stops);
                break;
            }
        }
        if (lane == 0) {
            p.out_accept_len[of.who] = n;
            p.out_token[of.who] = drawn;
        }
    };
    if (!(most > -__builtin_inff())) {                           // nothing to draw from
        if (tid == 0 && p.p) p.p[row_at] = 0.0f;
        finish(-1, false);
        return;
    }
    if (mode == DRAW_FIRST) {                                    // of the first chunk that has the largest logit the first place that has it
        int chunk = 0;
#pragma unroll 1
        for (int i = 0; i * kDrawThreads < maxima; ++i) {
            int first, last;
            talk.ends((i == 0 ? chunk_max[0] : chunk_max_at(i)) == most, false, first, last);
            if (first == kDrawThreads) continue;
            chunk = first + i * kDrawThreads;
            break;
        }
        const int unit = chunk * 16 + (lane & 15);
        float x[N];
        row.values(unit, row.request(unit), x, [](float z) { return logit_weighed(z); });
        int place = N;
#pragma unroll
        for (int e = N - 1; e >= 0; --e) place = x[e] == most ? e : place;
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(place < N)), token = (chunk * 16 + l) * N + __builtin_amdgcn_readlane(place, l) - row.skew;
        const bool all = draft == token;                         // the draft has all mass
        if (tid == 0 && p.p) p.p[row_at] = !p.draft || all ? 1.0f : 0.0f;
        finish(all && !last_row ? -1 : token, all && !last_row && u_accept < 1.0f);
        return;
    }
    const double top = of_lane(bucket_line(most, f.scale), 0);
    const float draft_logit = draft >= 0 && draft < p.V ? row.one(draft) : -__builtin_inff();    // (one address for the workgroup)
    static_assert(kMaxTokenParts <= kDrawThreads, "a part a thread");
    if (tid < nb) {
        part_max[tid] = mine_max;
        if (mode != DRAW_ALL) shift[tid] = bucket_of(mine_max, f.scale, top);
        factor[tid] = mine_max > -__builtin_inff() ? weight_of(mine_max, most, f.rate) : 0.0;
        part_mass[tid] = mode == DRAW_ALL ? mine_mass : 0;
    }
    __syncthreads();

    // Ten requests at a time of what the parts have in this thread's bucket, of every other part: take(part, what it has).
    auto merged = [&](auto place, auto take) {
        const int j = tid % kBuckets;
#pragma unroll 1
        for (int b0 = tid / kBuckets; b0 < nb; b0 += 20) {
            decltype(place(0ll)) v[10];
            bool ok[10];
#pragma unroll
            for (int i = 0; i < 10; ++i) {
                const int b = b0 + 2 * i;
                ok[i] = b < nb && j >= shift[min(b, nb - 1)];
                v[i] = place(((long long)r * nb + (ok[i] ? b : 0)) * kBuckets + (ok[i] ? j - shift[b] : 0));
            }
#pragma unroll
            for (int i = 0; i < 10; ++i)
                if (ok[i]) take(b0 + 2 * i, v[i]);
        }
    };
    // ---- buckets of the row: how many tokens, or what mass, through each
    if (f.k) {
        unsigned int count = 0;
        merged([&](long long at) { return p.count[at]; }, [&](int, unsigned int n) { count += n; });
        bin_count[tid] = count;
        __syncthreads();
        const unsigned int through = talk.sum_through(tid < kBuckets ? bin_count[tid] + bin_count[tid + kBuckets] : 0u);
        if (tid < kBuckets) through_count[tid] = through;
        __syncthreads();
    }
    if (mode == DRAW_MANY) {
        double mass = 0.0;
        merged([&](long long at) { return p.mass[at]; }, [&](int b, u64 units) { mass += (double)units * (factor[b] * (1.0 / (double)(1ull << kPartBits))); });
        reinterpret_cast<double *>(bin_mass)[tid] = mass;
        __syncthreads();
        mass = tid < kBuckets ? reinterpret_cast<double *>(bin_mass)[tid] + reinterpret_cast<double *>(bin_mass)[tid + kBuckets] : 0.0;
        const double through = talk.sum_through(mass);
        if (tid < kBuckets) bucket_mass[tid] = mass, through_mass[tid] = through;
        __syncthreads();
    }

    // The gathered tokens: their keys in the list, as many as it takes, or, where there are more, read again wherever they are asked for.  (The steps below are one loop, so that
    // gathering and selecting stand in the code once: as often as they are called it was 216 KB.)
    float gathered_from = 0.0f, gathered_to = 0.0f;              // their smallest and largest logit
    int gathered = -1;                                           // buckets: first << 16 | last
    auto each = [&](auto body) {
        if (n_listed <= kListed) {
            for (int i = tid; i < n_listed; i += kDrawThreads) body(list[i]);
            return;
        }
        for (int q = 4 * w + (lane >> 4); q < n_chunks; q += 4 * kDrawWaves) {
            const int unit = chunks[q] * 16 + (lane & 15);
            float x[N];
            row.values(unit, row.request(unit), x, [](float z) { return z; });
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (x[e] >= gathered_from && x[e] <= gathered_to) body(rank_key<DT>(logit_value(x[e]), unit * N + e - row.skew));
        }
    };

    // ---- the cut: by top-k, then by top-p, then by min_p; at last the tokens of the bucket in which it lies
    enum { BY_COUNT, BY_MASS, OF_BORDER, STEPS };
    u64 cut = ALL;
    int border = kBuckets;                                       // the bucket in which it lies (FEW: the last one gathered)
    double total = mode == DRAW_MANY ? through_mass[kBuckets - 1] : 0.0;
#pragma unroll 1
    for (int step = mode == DRAW_ALL ? (int)STEPS : (int)BY_COUNT; step < STEPS; ++step) {
        int from = 0, to = border, last;
        double limit = 0.0;
        unsigned int need = 0;
        if (step == BY_COUNT) {
            if (!f.k) continue;
            talk.ends(tid < kBuckets && through_count[tid % kBuckets] >= (unsigned int)f.k, false, to, last);
            if (mode == DRAW_MANY && to >= kBuckets) continue;   // (what is beyond the buckets has no mass)
            to = min(to, kBuckets - 1);
            from = mode == DRAW_FEW ? 0 : to;
            need = (unsigned int)f.k - (to ? through_count[to - 1] : 0u);        // of bucket `to`
        } else if (step == BY_MASS) {
            if (!(f.p < 1.0f)) continue;
            limit = (double)f.p * total;
            if (mode == DRAW_MANY) {
                talk.ends(tid < border && bucket_mass[tid % kBuckets] > 0.0 && through_mass[tid % kBuckets] >= limit, false, to, last);
                to = min(to, border);
                if (to == kBuckets) continue;
                from = to;
                limit -= through_mass[to] - bucket_mass[to];
            }
        } else {
            if (f.min_p > 0.0f) {
                const float least = least_logit(most, f.rate, f.min_p);
                const u64 key = last_key<DT>(ordered_bits(least));
                if (key < cut) {
                    cut = key;
                    if (mode == DRAW_MANY) border = bucket_of(least, f.scale, top);
                }
            }
            if (mode == DRAW_FEW || border == kBuckets) break;
            from = to = border;
        }
        const uint32_t least = least_ordered_of_bucket(to, f, top, most);
        if (gathered != (from << 16 | to)) {
            gathered = from << 16 | to;
            gathered_from = value_of_ordered(least);
            gathered_to = from ? value_of_ordered(least_ordered_of_bucket(from - 1, f, top, most) - 1) : __builtin_inff();
            if (tid == 0) n_chunks = 0, n_listed = 0;
            __syncthreads();
#pragma unroll 1
            for (int i = 0; i * kDrawThreads < maxima; ++i) {
                const float largest = i == 0 ? chunk_max[0] : i == 1 ? chunk_max[1] : i == 2 ? chunk_max[2] : i == 3 ? chunk_max[3] : chunk_max_at(i);
                const bool may = largest >= gathered_from;
                const unsigned long long mask = __builtin_amdgcn_ballot_w64(may);
                if (!mask) continue;
                int at = 0;
                if (lane == 0) at = atomicAdd(&n_chunks, (int)__popcll(mask));
                at = __builtin_amdgcn_readfirstlane(at);
                if (may) chunks[at + __popcll(mask & ((1ull << lane) - 1))] = (unsigned short)(tid + i * kDrawThreads);
            }
            __syncthreads();
            // (to a whole number of a wave's turns, of chunks behind the last one, which hold nothing)
            constexpr int TURN = 4 * DEPTH;
            static_assert(TURN <= kChunkTurn, "room behind the chunks");
            const int turns = (n_chunks + TURN - 1) / TURN;
            if (tid < turns * TURN - n_chunks) chunks[n_chunks + tid] = (unsigned short)maxima;
            __syncthreads();
            const int in_chunk = lane & 15;
            u32x4 next[DEPTH];
            int next_unit[DEPTH];
            auto ask = [&](int turn) {
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) next_unit[i] = chunks[turn * TURN + 4 * i + (lane >> 4)] * 16 + in_chunk;
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) next[i] = row.request(next_unit[i]);
            };
            if (w < turns) ask(w);
#pragma unroll 1
            for (int turn = w; turn < turns; turn += kDrawWaves) {
                const unsigned short *ids = chunks + turn * TURN + (lane >> 4);
                u32x4 raw[DEPTH];
                int unit[DEPTH];
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) raw[i] = next[i], unit[i] = next_unit[i];
                if (turn + kDrawWaves < turns) ask(turn + kDrawWaves);
                unsigned int in = 0;
                bool ends = false;
                auto between = [&](const float (&x)[N]) {
                    unsigned int bits = 0;
#pragma unroll
                    for (int e = 0; e < N; ++e) bits |= x[e] >= gathered_from && x[e] <= gathered_to ? 1u << e : 0u;
                    return bits;
                };
#pragma unroll
                for (int i = 0; i < DEPTH; ++i) {
                    float x[N];
                    row.as_whole(raw[i], x, [](float z) { return z; });
                    const unsigned int bits = between(x) << (i * N);
                    in |= row.whole(unit[i]) ? bits : 0u;
                    ends |= row.partial(unit[i]);
                }
                if (__builtin_amdgcn_ballot_w64(ends)) {         // a row's first and last places
#pragma unroll 1
                    for (int i = 0; i < DEPTH; ++i) {
                        const int u = ids[4 * i] * 16 + in_chunk;
                        if (!row.partial(u)) continue;
                        float x[N];
                        row.at_end(u, x);
                        in |= between(x) << (i * N);
                    }
                }
                const int n = __popc(in), through = lane_sums_through(n), all = __builtin_amdgcn_readlane(through, 63);
                if (!all) continue;
                int at = 0;
                if (lane == 0) at = atomicAdd(&n_listed, all);
                at = __builtin_amdgcn_readfirstlane(at) + through - n;
                for (; in; in &= in - 1, ++at) {                 // (as often as the lane that has most; the places alone: logits are indexed at compile time)
                    const int bit = __builtin_ctz(in);
                    if (at < kListed) list[at] = (u64)((ids[4 * (bit / N)] * 16 + in_chunk) * N + bit % N - row.skew);
                }
            }
            __syncthreads();
            // their keys: the logits once more, side by side
            if (n_listed <= kListed) {
#pragma unroll 1
                for (int i0 = tid; i0 < n_listed; i0 += 4 * kDrawThreads) {
                    int v[4];
                    float z[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (int)list[i0 + i * kDrawThreads < n_listed ? i0 + i * kDrawThreads : i0];    // (its own: others become keys)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = row.one(v[i]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i0 + i * kDrawThreads < n_listed) list[i0 + i * kDrawThreads] = rank_key<DT>(z[i], v[i]);
                }
            }
            __syncthreads();
        }
        if (step == OF_BORDER) break;
        border = to;
        // Among the keys lo .. hi, `inside` of them, the first `want` (tokens, or units of mass: those ahead of which less lies).  Masses are multiples of 2^-43 of the largest
        // logit's weight that there may be in the one bucket that is gathered: off by 2^-43.9 of the bucket's at most, however little that is of the row's.  Where all that is
        // left is gathered, up to kFew tokens of many buckets, they are multiples of 2^-51 of the row's largest.
        const bool by_mass = step == BY_MASS, one = !by_mass || from;            // (one bucket's)
        const uint32_t largest = one && to ? least_ordered_of_bucket(to - 1, f, top, most) - 1 : ordered_bits(most);
        const int bits = mode == DRAW_FEW ? kFewBits : kListBits;
        const float ref = mode == DRAW_FEW ? most : value_of_ordered(largest);
        const double to_row = of_lane(weight_of(ref, most, f.rate) * (mode == DRAW_FEW ? 1.0 / (1ull << kFewBits) : 1.0 / (1ull << kListBits)), 0);
        u64 lo = first_key<DT>(largest), hi = last_key<DT>(least), before = 0;
        hi = cut < hi ? cut : hi;
        int inside = from || by_mass ? n_listed : (int)(through_count[to] - (to ? through_count[to - 1] : 0u));
        const double units = by_mass ? __builtin_ceil(limit / to_row) : (double)need;
        const u64 want = units < 1.0 ? 1ull : units < 0x1p63 ? (u64)units : 1ull << 63;
        if (by_mass || need < (unsigned int)inside) {
#pragma unroll 1
            while (inside > kPairs && lo < hi) {                 // a digit of ten bits at a time
                const u64 span = hi - lo;
                const int digit = span < kDrawThreads ? 0 : 54 - __builtin_clzll(span);
                bin_mass[tid] = 0;
                bin_count[tid] = 0;
                __syncthreads();
                each([&](u64 key) {
                    if (key < lo || key > hi) return;
                    const int at = (int)((key - lo) >> digit);
                    atomicAdd(&bin_count[at], 1u);
                    if (by_mass) atomicAdd(&bin_mass[at], weight_units(key_value<DT>(key), ref, f.rate, bits));
                });
                __syncthreads();
                const unsigned int count = bin_count[tid];
                const u64 mine = by_mass ? bin_mass[tid] : count, through = before + talk.sum_through(mine);
                int bin, last;
                talk.ends(count && through >= want, count != 0, bin, last);
                if (bin == kDrawThreads) bin = max(last, 0);     // (none reaches it: the last that holds any)
                if (tid == bin) chosen[0] = through - mine, chosen[1] = count;
                __syncthreads();
                const u64 end = lo + ((u64)(bin + 1) << digit) - 1;
                hi = end < hi ? end : hi;
                lo += (u64)bin << digit;
                before = chosen[0];
                inside = (int)chosen[1];
            }
            if (inside > 1 && lo < hi) {                         // each is compared with each, four lanes to a token
                if (tid == 0) n_edge = 0, chosen[2] = hi;
                __syncthreads();
                each([&](u64 key) {
                    if (key < lo || key > hi) return;
                    const int at = atomicAdd(&n_edge, 1);
                    if (at < kPairs) edge[at] = key;             // (there are no more)
                });
                __syncthreads();
                const int n = min(n_edge, kPairs), mine = tid / 4, part = tid % 4;
                if (tid < n) bin_mass[tid] = by_mass ? weight_units(key_value<DT>(edge[tid]), ref, f.rate, bits) : 1;
                else if (tid < n + 16) edge[tid] = ALL;          // (ahead of none)
                __syncthreads();
                if (4 * n > (tid & ~63)) {                       // (whole waves)
                    const u64 key = mine < n ? edge[mine] : ALL;
                    u64 ahead = 0;
                    for (int i = part; i < n; i += 16) {
                        u64 other[4], units[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) other[e] = edge[i + 4 * e], units[e] = bin_mass[i + 4 * e];
#pragma unroll
                        for (int e = 0; e < 4; ++e) ahead += other[e] < key ? units[e] : 0;
                    }
                    ahead += __shfl_xor(ahead, 1, 64);
                    ahead += __shfl_xor(ahead, 2, 64);
                    ahead += before;
                    if (mine < n && part == 0 && ahead < want && ahead + bin_mass[mine] >= want) chosen[2] = key;     // (one of them, or none: all are in)
                }
                __syncthreads();
                hi = chosen[2];
            }
        }
        cut = hi;
        if (!by_mass && f.p < 1.0f) {                            // the mass up to the cut
            u64 mass = 0;
            each([&](u64 key) {
                if (key <= cut) mass += weight_units(key_value<DT>(key), ref, f.rate, bits);
            });
            total = (double)talk.sum(mass) * to_row + (from ? through_mass[from - 1] : 0.0);
        }
    }
    if (mode == DRAW_MANY && border == kBuckets) {               // (what lies beyond the buckets is not counted)
        const u64 key = last_key<DT>(least_ordered_of_bucket(kBuckets - 1, f, top, most));
        cut = key < cut ? key : cut;
    }
    auto kept = [&](float z, int v) { return rank_key<DT>(z, v) <= cut; };

    // ---- what is left of each part
    __syncthreads();
    if (mode == DRAW_MANY) {
#pragma unroll 1
        for (int b = w; b < nb; b += kDrawWaves) {
            u64 v[kBuckets / 64], sum = 0;
            const int n = border - shift[b];
#pragma unroll
            for (int i = 0; i < kBuckets / 64; ++i) {
                const int j = 64 * i + lane;
                v[i] = j < n ? p.mass[((long long)r * nb + b) * kBuckets + j] : 0;
            }
#pragma unroll
            for (int i = 0; i < kBuckets / 64; ++i) sum += v[i];
            sum = wave_sum(sum);
            if (lane == 0) part_mass[b] = sum;
        }
        __syncthreads();
    }
    if (mode == DRAW_FEW || (mode == DRAW_MANY && border < kBuckets)) {
        each([&](u64 key) {
            if (key > cut) return;
            const int b = (key_token(key) + row.skew) / kPartTokens;
            atomicAdd(&part_mass[b], weight_units(key_value<DT>(key), part_max[b], f.rate, kPartBits));
        });
        __syncthreads();
    }
    // ---- a refused draft is left out; the part that the draw falls in: the first whose running mass exceeds it, else the last that has any
    bool accepted = false;
    if (w == 0) {
        constexpr int EACH = (kMaxTokenParts + 63) / 64;
        const int per = (nb + 63) / 64;
        const bool in = draft >= 0 && draft < p.V && draft_logit > -__builtin_inff() && kept(draft_logit, draft);
        const int draft_part = in ? (draft + row.skew) / kPartTokens : 0;
        const u64 draft_units = in ? weight_units(draft_logit, part_max[draft_part], f.rate, kPartBits) : 0;
        u64 units[EACH];
        double sum = 0.0, through;
        auto add_up = [&] {
            sum = 0.0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += i < per && lane * per + i < nb ? (double)units[i] * factor[lane * per + i] : 0.0;
            through = lane_sums_through(sum);
            return of_lane(through, 63);
        };
#pragma unroll
        for (int i = 0; i < EACH; ++i) units[i] = i < per && lane * per + i < nb ? part_mass[lane * per + i] : 0;
        double whole = add_up();
        if (p.draft) {
            const double of_draft = (double)draft_units * factor[draft_part] / whole;
            if (lane == 0 && p.p) p.p[row_at] = (float)of_draft;
            accepted = !last_row && (double)u_accept < of_draft;
            if (!last_row && draft_units) {
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (i < per && lane * per + i == draft_part) units[i] -= draft_units;
                whole = add_up();
            }
        }
        const double target = u_at > 0.0f ? (double)u_at * whole : 0.0;
        const unsigned long long mass = __builtin_amdgcn_ballot_w64(sum > 0.0), reach = __builtin_amdgcn_ballot_w64(sum > 0.0 && through > target);
        const int owner = mass ? draw_lane(reach, mass) : -1;
        if (lane == 0) drawn_part = -1, drawn_total = whole, drawn_banned = !last_row ? draft : -1;
        if (lane == owner) {
            double ahead = through - sum;
            int part = -1;
            u64 of_part = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (i >= per || !units[i] || !(factor[lane * per + i] > 0.0) || (part >= 0 && ahead + (double)of_part * factor[part] > target)) continue;
                if (part >= 0) ahead += (double)of_part * factor[part];
                part = lane * per + i;
                of_part = units[i];
            }
            const double left = (target - ahead) / factor[part];
            u64 at = left > 0.0 ? (left < 0x1p62 ? (u64)left : 1ull << 62) : 0;
            if (at >= of_part) at = of_part - 1;
            drawn_part = part;
            chosen[0] = at;
        }
    }
    __syncthreads();
    const int part = drawn_part;
    if (part < 0) {                                              // (all mass was the draft's)
        finish(-1, accepted);
        return;
    }
    // ---- the token: eight places a thread, in order
    const int banned = drawn_banned;
    const u64 ahead = chosen[0];
    constexpr int LAST = kPartTokens / kDrawThreads / N;         // loads
    u32x4 raw[LAST];
    float x[LAST][N];
    const int at0 = part * kPartTokens + tid * (kPartTokens / kDrawThreads);
    u64 units[kPartTokens / kDrawThreads], sum = 0;
#pragma unroll
    for (int i = 0; i < LAST; ++i) raw[i] = row.request(at0 / N + i);
#pragma unroll
    for (int i = 0; i < LAST; ++i) row.values(at0 / N + i, raw[i], x[i], [](float z) { return logit_value(z); });
#pragma unroll
    for (int i = 0; i < kPartTokens / kDrawThreads; ++i) {
        const int v = at0 + i - row.skew;
        const float z = x[i / N][i % N];
        units[i] = 0;
        if (kept(z, v) && v != banned) units[i] = weight_units(z, part_max[part], f.rate, kPartBits);
        sum += units[i];
    }
    const u64 through = talk.sum_through(sum);
    if (through > ahead && through - sum <= ahead) {
        u64 at = through - sum;
#pragma unroll
        for (int i = 0; i < kPartTokens / kDrawThreads; ++i) {
            if (at <= ahead && at + units[i] > ahead) {
                drawn_token = at0 + i - row.skew;
                if (p.p && !p.draft) p.p[row_at] = (float)((double)units[i] * factor[part] / drawn_total);
            }
            at += units[i];
        }
    }
    __syncthreads();
    finish(drawn_token, accepted);
}

}  // namespace quasar
