// C entry points of the paged key/value cache: checks on the host, launches.
#include "../../include/quasar.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>

#include "pages.hpp"
#include "paged_attention.hpp"
#include "prompt_attention.hpp"

using namespace quasar;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int compute_units() {
    static std::atomic<int> cached[64];
    int dev = 0, v = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    v = cached[dev].load();
    if (v == 0) {
        if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) v = 256;
        cached[dev] = v;
    }
    return v;
}

// The opt-in to more dynamic LDS than the default, once for each kernel and device.
template <auto Kernel> bool large_lds() {
    static std::atomic<unsigned long long> done{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load() & bit)) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return false;
    if (dev < 64) done.fetch_or(bit);
    return true;
}

int launched() { return hipGetLastError() == hipSuccess ? QUASAR_OK : QUASAR_ERR_HIP; }

int kv_type(int dtype) { return dtype == QUASAR_BF16 ? KV_BF16 : dtype == QUASAR_E4M3 ? KV_E4M3 : -1; }
int block_shift_of(int64_t page_len) {
    for (int i = 0; i <= 5; ++i)
        if (page_len == (int64_t)kKvBlock << i) return i;
    return -1;
}
constexpr int64_t kMaxPages = 1 << 20;

// What the calls have in common of a cache's shape.
int check_books(int64_t table_ld, int64_t n_seqs, int64_t max_pages, int64_t n_pages, int64_t page_len) {
    if (n_seqs < 1 || n_seqs > kMaxSeqs || max_pages < 1 || table_ld < max_pages || table_ld > (int64_t(1) << 40)) return QUASAR_ERR_SHAPE;
    if (n_pages < 1 || n_pages > kMaxPages || block_shift_of(page_len) < 0 || max_pages > kMaxPositions / page_len) return QUASAR_ERR_SHAPE;
    return QUASAR_OK;
}
int check_heads(int64_t Hq, int64_t Hkv) {
    return Hkv < 1 || Hkv > 1024 || Hq < Hkv || Hq % Hkv || Hq > 4096 ? QUASAR_ERR_SHAPE : QUASAR_OK;
}

struct CacheArgs {
    int64_t T, Hq, Hkv;
    const void *pages;
    int64_t n_pages, page_len;
    int kv_dtype;
    const float *k_scale, *v_scale;
    const int32_t *table;
    int64_t table_ld, n_seqs, max_pages;
    const int32_t *lengths, *row_start;
};
int check_cache(const CacheArgs &a, PagedParams &p) {
    if (!a.pages || !a.table || !a.lengths || !a.row_start) return QUASAR_ERR_NULL;
    if (kv_type(a.kv_dtype) < 0) return QUASAR_ERR_DTYPE;
    if (a.T < 1 || a.T > kMaxPositions || check_heads(a.Hq, a.Hkv)) return QUASAR_ERR_SHAPE;
    if (const int e = check_books(a.table_ld, a.n_seqs, a.max_pages, a.n_pages, a.page_len)) return e;
    if (kv_type(a.kv_dtype) == KV_BF16 && (a.k_scale || a.v_scale)) return QUASAR_ERR_DTYPE;
    if (!aligned(a.pages, 16) || !aligned(a.table, 4) || !aligned(a.lengths, 4) || !aligned(a.row_start, 4) || !aligned(a.k_scale, 4) ||
        !aligned(a.v_scale, 4))
        return QUASAR_ERR_ALIGN;
    p.pages = static_cast<unsigned char *>(const_cast<void *>(a.pages));
    p.table = a.table; p.lengths = a.lengths; p.row_start = a.row_start;
    p.k_scale = a.k_scale; p.v_scale = a.v_scale;
    p.table_ld = a.table_ld;
    p.T = (int)a.T; p.n_seqs = (int)a.n_seqs; p.n_pages = (int)a.n_pages; p.columns = (int)a.max_pages;
    p.Hkv = (int)a.Hkv; p.Hq = (int)a.Hq; p.G = (int)(a.Hq / a.Hkv);
    p.block_shift = block_shift_of(a.page_len);
    p.max_new = kMaxPositions;
    return QUASAR_OK;
}
// New rows a sequence, on average, from which the append goes block by block: 40 sequences of up to 90 rows of 32 / 8 heads in 8-bit pages
// 22.4 us row by row and 24 to 31 by blocks, 11 of up to 1531 88 and 57.
constexpr int kBlockRows = 64;
constexpr float kScaleLog2 = 1.4426950408889634f / 11.313708498984761f;      // log2(e) / sqrt(128)

// ---- what the attention calls share of a launch: workgroups of a kv head, and the room for what they leave of shared sequences or tiles
struct FlatShape {
    int64_t tiles;            // of rows, at most (prompts)
    int workers;              // 0: nothing is shared
    size_t part_o, part_ml, pieces;
    size_t bytes() const { return part_o + part_ml + pieces; }
    void room(int64_t wanted, int64_t parts_each /* 16-byte-a-lane parts of a slot */, int64_t stats_each /* bytes */, int64_t Hkv) {
        workers = (int)(wanted < 1 ? 1 : wanted > kMaxWorkers ? kMaxWorkers : wanted);
        const size_t slots = (size_t)Hkv * 2 * workers;
        part_o = slots * parts_each * 64 * 16;
        part_ml = slots * stats_each;
        pieces = (size_t)workers * 16;
    }
};

// ---- attention of a step.  Up to 32 rows of a sequence and kv head take the 16 x 16 products, more the kernel of prompts, whose tiles have 64
// or 128 rows: 16 sequences of 8 tokens over up to 4000 positions, 32 / 8 heads (32 rows), 44.5 us in tiles of 16 and 61 in tiles of 32; 8
// of 16 tokens over 8000 (64 rows) 65.7 and 48.5.
struct StepShape {
    int NQT;                  // 16-row tiles; 0: the kernel of prompts with PW
    int PW;
    FlatShape flat;
};
bool step_shape(int64_t max_new, int64_t Hq, int64_t Hkv, int64_t n_seqs, StepShape &a) {
    if (max_new < 1 || max_new > 32 || check_heads(Hq, Hkv)) return false;
    const int64_t R = max_new * (Hq / Hkv), cus = compute_units();
    if (R > 1024) return false;
    a = StepShape{};
    a.NQT = R <= 16 ? 1 : R <= 32 ? 2 : 0;
    if (a.NQT) {
        a.flat.room(cus / Hkv, a.NQT * 8, a.NQT * 16 * 8, Hkv);
        return true;
    }
    a.PW = R <= 64 ? 2 : 1;
    const int rw = kPromptWaves / a.PW;
    a.flat.tiles = n_seqs * ((R + 32 * rw - 1) / (32 * rw));
    if (a.flat.tiles <= kMaxFlatTiles) a.flat.room(2 * cus / Hkv, rw * 16, rw * 64 * 8, Hkv);
    return true;
}

template <auto Kernel, class Params>
int launch_attention(unsigned int workgroups_x, unsigned int workgroups_y, int lds, hipStream_t st, const Params &p) {
    if (!large_lds<Kernel>()) return QUASAR_ERR_HIP;
    hipLaunchKernelGGL(Kernel, dim3(workgroups_x, workgroups_y), dim3(kPromptWaves * 64), lds, st, p);
    return launched();
}
template <int KV>
int launch_step(const PagedAttnParams &p, int NQT, hipStream_t st) {
    const int lds = kPagedWaves * NQT * (8 * 64 * 16 + 16 * 2 * 4) + (kPagedWaves + 4 * (p.c.n_seqs + 1)) * 4;
    const int e = NQT == 1 ? launch_attention<paged_attention_kernel<KV, 1>>(p.workers, p.c.Hkv, lds, st, p)
                           : launch_attention<paged_attention_kernel<KV, 2>>(p.workers, p.c.Hkv, lds, st, p);
    if (e || p.workers == 1) return e;                                       // (one worker finishes every sequence)
    hipLaunchKernelGGL(paged_merge_kernel, dim3((unsigned int)(2 * compute_units())), dim3(512), 0, st, p, NQT);
    return launched();
}

// ---- attention of prompts: tiles of 128 rows, shared where they would leave compute units idle, being fewer than the two workgroups that each
// unit holds.  (4 x 700 rows behind 3000 positions 112.8 us, shared 111.2; 2 x 2048 behind 2000, two rounds of tiles, 133.2 and 161.7; one of 3000
// rows 86.3 and 130.5: the join moves 16 KB for 32 rows of each part.)
FlatShape prompt_shape(int64_t T, int64_t Hq, int64_t Hkv, int64_t n_seqs) {
    FlatShape a{};
    a.tiles = T * (Hq / Hkv) / (32 * kPromptWaves) + n_seqs;                 // (at most a ragged one a sequence)
    const int64_t per = 2 * (int64_t)compute_units() / Hkv;
    if (a.tiles <= kMaxFlatTiles && a.tiles < per) a.room(per, kPromptWaves * 16, kPromptWaves * 64 * 8, Hkv);
    return a;
}
// Where sharing is possible, the kernel shares tiles if the longest has more steps than a worker's share and this many: what starts of further
// tiles and the join cost, more with more tiles.  Both ways, us, bf16, 32 / 8 heads, over a table of 262144 positions: 61 rows 17.6 shared and 11.8
// whole, behind 400 positions (8 steps where a share is 4) 20.0 and 21.4, behind 900 21.5 and 31.2; 256 rows 27.4 and 15.9, behind 500 (12
// and 4) 27.1 and 26.9; 512 rows 33.0 and 21.0, behind 600 (18 and 4) 34.8 and 34.1, behind 1000 (24 and 6) 38.8 and 41.5; 1900 rows (30 and
// 15) 73.0 and 58.0, behind 2000 (61 and 45) 117.2 and 116.5; 2048 rows of 8 / 1 heads (32 and 5) 47.1 and 52.5.
int whole_more(int64_t T, int64_t G) {
    const int64_t tiles = (T * G + 32 * kPromptWaves - 1) / (32 * kPromptWaves);
    return (int)(tiles < 16 ? tiles : 16);
}
template <int KV>
int launch_prompt(const PromptParams &p, int64_t tiles, int PW, hipStream_t st) {
    const int lds = 2 * kPromptStepBytes + (kMaxSeqs + kPromptWaves + 8) * 4;
    if (!p.workers) return launch_attention<prompt_attention_kernel<KV, false, 1>>((unsigned int)(tiles * p.c.Hkv), 1, lds, st, p);
    const unsigned int n = (unsigned int)(p.workers * p.c.Hkv);
    const int e = PW == 1 ? launch_attention<prompt_attention_kernel<KV, true, 1>>(n, 1, lds + kMaxFlatTiles * 4, st, p)
                          : launch_attention<prompt_attention_kernel<KV, true, 2>>(n, 1, lds + kMaxFlatTiles * 4, st, p);
    if (e || p.workers == 1) return e;
    hipLaunchKernelGGL(prompt_merge_kernel, dim3((unsigned int)(4 * compute_units())), dim3(256), 0, st, p, kPromptWaves / PW);
    return launched();
}

// The workspace's parts, in the parameters of either kernel.
template <class Params> void lay_out(Params &p, const FlatShape &a, void *workspace) {
    p.workers = a.workers;
    p.part_o = static_cast<f32x4 *>(workspace);
    p.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + a.part_o);
    p.pieces = reinterpret_cast<int *>(static_cast<unsigned char *>(workspace) + a.part_o + a.part_ml);
}

BooksParams books(int32_t *table, int64_t table_ld, int64_t n_seqs, int64_t max_pages, int32_t *lengths, int32_t *refs, int64_t n_pages, int64_t page_len) {
    BooksParams b{};
    b.table = table; b.lengths = lengths; b.refs = refs;
    b.table_ld = table_ld;
    b.n_seqs = (int)n_seqs; b.columns = (int)max_pages; b.n_pages = (int)n_pages;
    b.block_shift = block_shift_of(page_len);
    return b;
}
struct PagesRoom { size_t copies, lists; };      // bytes of the copy list (a header and an item a page or sequence) and of each list of pages
PagesRoom pages_room(int64_t n_seqs, int64_t n_pages) {
    return {16 + 16 * (size_t)(n_seqs > n_pages ? n_seqs : n_pages), 4 * (size_t)((n_pages + 3) & ~int64_t(3))};
}
int launch_copies(const BooksParams &b, const CopyList *copies, const int32_t *to, void *pool, int64_t n_layers, int64_t Hkv, int kv, hipStream_t st) {
    const int block_bytes = 2 * (kv == KV_E4M3 ? kv_block_bytes<KV_E4M3> : kv_block_bytes<KV_BF16>);
    hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned int)(8 * compute_units())), dim3(256), 0, st, b, copies, to, static_cast<unsigned char *>(pool),
                       (int)n_layers, (int)Hkv, block_bytes);
    return launched();
}

}  // namespace

extern "C" {

size_t quasar_paged_cache_bytes(int64_t n_layers, int64_t n_kv_heads, int64_t n_pages, int64_t page_len, int kv_dtype) {
    if (n_layers < 1 || n_layers > 4096 || n_kv_heads < 1 || n_kv_heads > 1024 || n_pages < 1 || n_pages > kMaxPages) return 0;
    if (block_shift_of(page_len) < 0 || kv_type(kv_dtype) < 0) return 0;
    return (size_t)n_layers * (size_t)n_pages * (size_t)n_kv_heads * (size_t)page_len * 2 * kHeadDim * (kv_type(kv_dtype) == KV_BF16 ? 2 : 1);
}

int quasar_paged_prepare(const uint16_t *qkv, int64_t T, int64_t ld, int64_t n_q_heads, int64_t n_kv_heads, const int32_t *row_start,
                         int64_t n_seqs, const uint16_t *q_gamma, const uint16_t *k_gamma, float eps, float rope_theta, uint16_t *q_out,
                         int64_t ldq, void *pages, int64_t n_pages, int64_t page_len, int kv_dtype, const float *k_scale, const float *v_scale,
                         const int32_t *table, int64_t table_ld, int64_t max_pages, const int32_t *lengths, void *hip_stream) {
    if (!qkv || !q_gamma || !k_gamma || !q_out) return QUASAR_ERR_NULL;
    PrepareParams p{};
    const CacheArgs a{T, n_q_heads, n_kv_heads, pages, n_pages, page_len, kv_dtype, k_scale, v_scale, table, table_ld, n_seqs, max_pages, lengths, row_start};
    if (const int e = check_cache(a, p.c)) return e;
    if (ld < (n_q_heads + 2 * n_kv_heads) * kHeadDim || ldq < n_q_heads * kHeadDim || ld % 8 || ldq % 8) return QUASAR_ERR_SHAPE;
    if (!(eps >= 0.f && eps < 1.f) || !(rope_theta > 1.f) || !(rope_theta < 1e30f)) return QUASAR_ERR_SHAPE;
    if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(q_gamma, 16) || !aligned(k_gamma, 16)) return QUASAR_ERR_ALIGN;
    p.qkv = qkv; p.q_gamma = q_gamma; p.k_gamma = k_gamma; p.q_out = q_out;
    p.ld = ld; p.ldq = ldq; p.eps = eps;
    p.log2_theta = std::log2((double)rope_theta);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int64_t heads = n_q_heads + 2 * n_kv_heads;
    if (T >= kBlockRows * n_seqs) {
        // as many heads a workgroup as keep four workgroups a compute unit, eight at most: 512 rows of 32 / 8 heads 8.3 us with one (eight: 14.7),
        // 11 prompts of up to 1531 rows in 8-bit pages 57 with eight (four: 60)
        const int64_t blocks = T / kKvBlock + 2 * n_seqs;                    // (two ragged ones a sequence)
        int64_t parts = (T / kKvBlock * heads) / (4 * compute_units());
        parts = parts < 1 ? 1 : parts > 8 ? 8 : parts;
        p.parts = (int)parts;
        const dim3 grid((unsigned int)blocks, (unsigned int)((heads + parts - 1) / parts));
        if (kv_type(kv_dtype) == KV_BF16) hipLaunchKernelGGL(paged_prepare_block_kernel<KV_BF16>, grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL(paged_prepare_block_kernel<KV_E4M3>, grid, dim3(256), 0, st, p);
        return launched();
    }
    const int64_t quads = (heads + 3) / 4;
    int64_t parts = 4096 / T;
    parts = parts < 1 ? 1 : parts > quads ? quads : parts;
    p.parts = (int)parts;
    const dim3 grid((unsigned int)((T * parts + 3) / 4));
    if (kv_type(kv_dtype) == KV_BF16) hipLaunchKernelGGL(paged_prepare_kernel<KV_BF16>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(paged_prepare_kernel<KV_E4M3>, grid, dim3(256), 0, st, p);
    return launched();
}

size_t quasar_paged_attention_workspace_bytes(int64_t max_new, int64_t n_q_heads, int64_t n_kv_heads) {
    StepShape a{};
    return step_shape(max_new, n_q_heads, n_kv_heads, 1, a) ? a.flat.bytes() : 0;
}

int quasar_paged_attention(const uint16_t *q, int64_t T, int64_t ldq, int64_t n_q_heads, int64_t n_kv_heads, const int32_t *row_start,
                           int64_t n_seqs, int64_t max_new, const void *pages, int64_t n_pages, int64_t page_len, int kv_dtype,
                           const float *k_scale, const float *v_scale, const int32_t *table, int64_t table_ld, int64_t max_pages,
                           const int32_t *lengths, uint16_t *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!q || !out) return QUASAR_ERR_NULL;
    PagedParams c{};
    const CacheArgs a{T, n_q_heads, n_kv_heads, pages, n_pages, page_len, kv_dtype, k_scale, v_scale, table, table_ld, n_seqs, max_pages, lengths, row_start};
    if (const int e = check_cache(a, c)) return e;
    const int kv = kv_type(kv_dtype);
    StepShape shape{};
    if (!step_shape(max_new, n_q_heads, n_kv_heads, n_seqs, shape)) return QUASAR_ERR_SHAPE;
    if (ldq < n_q_heads * kHeadDim || ldo < n_q_heads * kHeadDim || ldq % 8 || ldo % 4) return QUASAR_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(out, 8)) return QUASAR_ERR_ALIGN;
    if (!workspace || workspace_bytes < quasar_paged_attention_workspace_bytes(max_new, n_q_heads, n_kv_heads)) return QUASAR_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUASAR_ERR_ALIGN;
    c.max_new = (int)max_new;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (shape.NQT) {
        PagedAttnParams p{};
        p.c = c;
        p.q = q; p.out = out; p.ldq = ldq; p.ldo = ldo;
        p.scale_log2 = kScaleLog2;
        lay_out(p, shape.flat, workspace);
        return kv == KV_BF16 ? launch_step<KV_BF16>(p, shape.NQT, st) : launch_step<KV_E4M3>(p, shape.NQT, st);
    }
    PromptParams p{};
    p.c = c;
    p.q = q; p.out = out; p.ldq = ldq; p.ldo = ldo;
    p.scale_log2 = kScaleLog2;
    p.whole_more = -(1 << 30);                                                   // (a step's tiles are shared always: minus more than any share)
    if (shape.flat.workers) lay_out(p, shape.flat, workspace);
    return kv == KV_BF16 ? launch_prompt<KV_BF16>(p, shape.flat.tiles, shape.PW, st) : launch_prompt<KV_E4M3>(p, shape.flat.tiles, shape.PW, st);
}

size_t quasar_prompt_attention_workspace_bytes(int64_t T, int64_t n_q_heads, int64_t n_kv_heads, int64_t n_seqs) {
    if (T < 1 || T > kMaxPositions || check_heads(n_q_heads, n_kv_heads) || n_seqs < 1 || n_seqs > kMaxSeqs) return 0;
    return prompt_shape(T, n_q_heads, n_kv_heads, n_seqs).bytes();
}

int quasar_prompt_attention(const uint16_t *q, int64_t T, int64_t ldq, int64_t n_q_heads, int64_t n_kv_heads, const int32_t *row_start,
                            int64_t n_seqs, const void *pages, int64_t n_pages, int64_t page_len, int kv_dtype, const float *k_scale,
                            const float *v_scale, const int32_t *table, int64_t table_ld, int64_t max_pages, const int32_t *lengths,
                            uint16_t *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!q || !out) return QUASAR_ERR_NULL;
    PromptParams p{};
    const CacheArgs a{T, n_q_heads, n_kv_heads, pages, n_pages, page_len, kv_dtype, k_scale, v_scale, table, table_ld, n_seqs, max_pages, lengths, row_start};
    if (const int e = check_cache(a, p.c)) return e;
    if (T * (n_q_heads / n_kv_heads) > (1 << 26)) return QUASAR_ERR_SHAPE;       // (the tiles of all sequences are counted in 32 bits)
    if (ldq < n_q_heads * kHeadDim || ldo < n_q_heads * kHeadDim || ldq % 8 || ldo % 4) return QUASAR_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(out, 8) || !aligned(workspace, 16)) return QUASAR_ERR_ALIGN;
    p.q = q; p.out = out; p.ldq = ldq; p.ldo = ldo;
    p.scale_log2 = kScaleLog2;
    const FlatShape shape = prompt_shape(T, n_q_heads, n_kv_heads, n_seqs);
    p.whole_more = whole_more(T, n_q_heads / n_kv_heads);
    // (a table so short that tiles stay whole whatever the lengths are: launched without the join)
    const bool may_share = max_pages * page_len > (int64_t)kPromptStep * (kFlatLeast + p.whole_more);
    if (workspace && shape.workers && workspace_bytes >= shape.bytes() && may_share) lay_out(p, shape, workspace);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return kv_type(kv_dtype) == KV_BF16 ? launch_prompt<KV_BF16>(p, shape.tiles, 1, st) : launch_prompt<KV_E4M3>(p, shape.tiles, 1, st);
}

size_t quasar_pages_workspace_bytes(int64_t n_seqs, int64_t n_pages) {
    if (n_seqs < 1 || n_seqs > kMaxSeqs || n_pages < 1 || n_pages > kMaxPages) return 0;
    const PagesRoom r = pages_room(n_seqs, n_pages);
    return r.copies + 2 * r.lists;
}

int quasar_pages_reserve(int32_t *table, int64_t table_ld, int64_t n_seqs, int64_t max_pages, const int32_t *lengths, const int32_t *n_new,
                         int32_t *refs, int64_t n_pages, int64_t page_len, int32_t *out_status, void *pool, int64_t n_layers,
                         int64_t n_kv_heads, int kv_dtype, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!table || !lengths || !n_new || !refs || !out_status || !pool) return QUASAR_ERR_NULL;
    if (kv_type(kv_dtype) < 0) return QUASAR_ERR_DTYPE;
    if (const int e = check_books(table_ld, n_seqs, max_pages, n_pages, page_len)) return e;
    if (!quasar_paged_cache_bytes(n_layers, n_kv_heads, n_pages, page_len, kv_dtype)) return QUASAR_ERR_SHAPE;
    if (!aligned(table, 4) || !aligned(lengths, 4) || !aligned(n_new, 4) || !aligned(refs, 4) || !aligned(out_status, 4) || !aligned(pool, 16)) return QUASAR_ERR_ALIGN;
    if (!workspace || workspace_bytes < quasar_pages_workspace_bytes(n_seqs, n_pages)) return QUASAR_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUASAR_ERR_ALIGN;
    const BooksParams b = books(table, table_ld, n_seqs, max_pages, const_cast<int32_t *>(lengths), refs, n_pages, page_len);
    CopyList *copies = static_cast<CopyList *>(workspace);
    int *free_list = reinterpret_cast<int *>(static_cast<unsigned char *>(workspace) + pages_room(n_seqs, n_pages).copies);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(1024), 0, st, b, n_new, out_status, free_list, copies);
    if (const int e = launched()) return e;
    return launch_copies(b, copies, nullptr, pool, n_layers, n_kv_heads, kv_type(kv_dtype), st);
}

int quasar_pages_fork(int32_t *table, int64_t table_ld, int64_t n_seqs, int64_t max_pages, int32_t *lengths, const int32_t *parent,
                      const int32_t *keep, int32_t *refs, int64_t n_pages, int64_t page_len, void *hip_stream) {
    if (!table || !lengths || !parent || !refs) return QUASAR_ERR_NULL;
    if (const int e = check_books(table_ld, n_seqs, max_pages, n_pages, page_len)) return e;
    if (!aligned(table, 4) || !aligned(lengths, 4) || !aligned(parent, 4) || !aligned(keep, 4) || !aligned(refs, 4)) return QUASAR_ERR_ALIGN;
    const BooksParams b = books(table, table_ld, n_seqs, max_pages, lengths, refs, n_pages, page_len);
    if (!large_lds<pages_fork_kernel>()) return QUASAR_ERR_HIP;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(pages_fork_kernel, dim3((unsigned int)((max_pages + kForkColumns - 1) / kForkColumns)), dim3(256),
                       (unsigned int)(n_seqs * kForkColumns * 4), st, b, parent, keep);
    if (const int e = launched()) return e;
    hipLaunchKernelGGL(pages_fork_lengths_kernel, dim3(1), dim3(1024), 0, st, b, parent, keep);
    return launched();
}

int quasar_pages_compact(int32_t *table, int64_t table_ld, int64_t n_seqs, int64_t max_pages, int32_t *refs, int64_t n_pages,
                         int64_t page_len, int32_t *out_to, void *pool, int64_t n_layers, int64_t n_kv_heads, int kv_dtype,
                         void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!table || !refs || !out_to || !pool) return QUASAR_ERR_NULL;
    if (kv_type(kv_dtype) < 0) return QUASAR_ERR_DTYPE;
    if (const int e = check_books(table_ld, n_seqs, max_pages, n_pages, page_len)) return e;
    if (!quasar_paged_cache_bytes(n_layers, n_kv_heads, n_pages, page_len, kv_dtype)) return QUASAR_ERR_SHAPE;
    if (!aligned(table, 4) || !aligned(refs, 4) || !aligned(out_to, 4) || !aligned(pool, 16)) return QUASAR_ERR_ALIGN;
    if (!workspace || workspace_bytes < quasar_pages_workspace_bytes(n_seqs, n_pages)) return QUASAR_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUASAR_ERR_ALIGN;
    const BooksParams b = books(table, table_ld, n_seqs, max_pages, nullptr, refs, n_pages, page_len);
    const PagesRoom room = pages_room(n_seqs, n_pages);
    CopyList *copies = static_cast<CopyList *>(workspace);
    int *holes = reinterpret_cast<int *>(static_cast<unsigned char *>(workspace) + room.copies), *moved = holes + room.lists / 4;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(1024), 0, st, b, out_to, holes, moved, copies);
    if (const int e = launched()) return e;
    return launch_copies(b, copies, out_to, pool, n_layers, n_kv_heads, kv_type(kv_dtype), st);
}

}  // extern "C"
