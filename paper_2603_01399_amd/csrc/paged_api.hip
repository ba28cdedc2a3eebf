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
    return QUASAR_OK;
}
// New rows a sequence, on average, from which the append goes block by block: 40 sequences of up to 90 rows of 32 / 8 heads in 8-bit pages
// 22.4 us row by row and 24 to 31 by blocks, 11 of up to 1531 88 and 57.
constexpr int kBlockRows = 64;
constexpr int kFlatRounds = 1, kFlatPositions = 1024;
constexpr float kScaleLog2 = 1.4426950408889634f / 11.313708498984761f;      // log2(e) / sqrt(128)

// ---- attention of a step: workers of a kv head, query tiles and groups of rows.  Up to 16 rows of a sequence and kv head take the 16 x 16
// products; more take the 32 x 32 ones, but bf16 pages up to 32 rows: 16 sequences of 8 tokens over up to 4000 positions, 32 / 8 heads
// 45.2 us narrow and 61 wide, 8-bit pages 36.4 and 30.4; 8 of 16 tokens over 8000 in bf16 65.7 (four narrow tiles) and 55.8.
struct StepShape { int NQT, groups, workers; bool wide; size_t part_o, part_ml, pieces; };
bool step_shape(int64_t max_new, int64_t Hq, int64_t Hkv, int kv, StepShape &a) {
    if (max_new < 1 || max_new > 32 || check_heads(Hq, Hkv)) return false;
    const int64_t R = max_new * (Hq / Hkv);
    if (R > 1024) return false;
    a.NQT = R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : 8;
    a.wide = a.NQT > 2 || (a.NQT == 2 && kv == KV_E4M3);
    a.groups = (int)((R + 16 * a.NQT - 1) / (16 * a.NQT));
    const int64_t per = (a.wide ? 2 : 1) * (int64_t)compute_units() / (Hkv * a.groups);      // as many workgroups as are on the GPU at once
    a.workers = (int)(per < 1 ? 1 : per > kMaxWorkers ? kMaxWorkers : per);
    const size_t slots = (size_t)a.groups * Hkv * 2 * a.workers * a.NQT;
    a.part_o = slots * 8 * 64 * 16;
    a.part_ml = slots * 16 * 2 * 4;
    a.pieces = (size_t)a.groups * a.workers * 16;
    return true;
}

template <auto Kernel>
int launch_step(const PagedAttnParams &p, const StepShape &a, int lds, hipStream_t st) {
    if (!large_lds<Kernel>()) return QUASAR_ERR_HIP;
    hipLaunchKernelGGL(Kernel, dim3((unsigned int)a.workers, (unsigned int)p.c.Hkv, (unsigned int)a.groups), dim3(kPagedWaves * 64),
                       lds + (kPagedWaves + p.c.n_seqs + 1) * 4, st, p);
    if (const int e = launched()) return e;
    if (a.workers == 1) return QUASAR_OK;                                    // (every sequence is finished by its one worker)
    hipLaunchKernelGGL(paged_merge_kernel, dim3((unsigned int)(2 * compute_units()), (unsigned int)a.groups), dim3(512), 0, st, p, a.NQT);
    return launched();
}
template <int KV>
int launch_step(PagedAttnParams &p, const StepShape &a, hipStream_t st) {
    p.group_rows = 16 * a.NQT;
    constexpr auto narrow = [](int nqt) { return kPagedWaves * nqt * (8 * 64 * 16 + 16 * 2 * 4); };
    constexpr auto wide = [](int rw) { return rw * (kPagedWaves / rw - 1) * (16 * 64 * 16 + 64 * 8); };
    if (a.NQT == 1) return launch_step<paged_attention_kernel<KV, 1>>(p, a, narrow(1), st);
    if (a.NQT == 4) return launch_step<paged_attention_wide_kernel<KV, 2>>(p, a, wide(2), st);
    if (a.NQT == 8) return launch_step<paged_attention_wide_kernel<KV, 4>>(p, a, wide(4), st);
    if constexpr (KV == KV_BF16) return launch_step<paged_attention_kernel<KV, 2>>(p, a, narrow(2), st);
    else return launch_step<paged_attention_wide_kernel<KV, 1>>(p, a, wide(1), st);
}

// ---- attention of prompts: workgroups of a kv head where tiles are shared
struct PromptShape { int64_t tiles; int workers; size_t part_o, part_ml, pieces; };
PromptShape prompt_shape(int64_t T, int64_t Hq, int64_t Hkv, int64_t n_seqs) {
    PromptShape a{};
    a.tiles = T * (Hq / Hkv) / (32 * kPromptWaves) + n_seqs;                 // (at most a ragged one a sequence)
    const int64_t per = 2 * (int64_t)compute_units() / Hkv;
    if (a.tiles > kMaxFlatTiles || a.tiles >= kFlatRounds * per) return a;
    a.workers = (int)(per < 1 ? 1 : per > kMaxWorkers ? kMaxWorkers : per);
    const size_t parts = (size_t)Hkv * 2 * a.workers * kPromptWaves;
    a.part_o = parts * 16 * 64 * 16;
    a.part_ml = parts * 64 * 8;
    a.pieces = (size_t)a.workers * 16;
    return a;
}

template <int KV>
int launch_prompt(const PromptParams &p, const PromptShape &a, hipStream_t st) {
    const int lds = 2 * kPromptStepBytes + (kMaxSeqs + kPromptWaves + 4) * 4;
    if (!p.workers) {
        constexpr auto kern = prompt_attention_kernel<KV, false>;
        if (!large_lds<kern>()) return QUASAR_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3((unsigned int)(a.tiles * p.c.Hkv)), dim3(kPromptWaves * 64), lds, st, p);
        return launched();
    }
    constexpr auto kern = prompt_attention_kernel<KV, true>;
    if (!large_lds<kern>()) return QUASAR_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3((unsigned int)(p.workers * p.c.Hkv)), dim3(kPromptWaves * 64), lds + kMaxFlatTiles * 4, st, p);
    if (const int e = launched()) return e;
    hipLaunchKernelGGL(prompt_merge_kernel, dim3((unsigned int)(4 * compute_units())), dim3(256), 0, st, p);
    return launched();
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
    StepShape a{}, b{};
    if (!step_shape(max_new, n_q_heads, n_kv_heads, KV_BF16, a) || !step_shape(max_new, n_q_heads, n_kv_heads, KV_E4M3, b)) return 0;
    const size_t x = a.part_o + a.part_ml + a.pieces, y = b.part_o + b.part_ml + b.pieces;
    return x > y ? x : y;
}

int quasar_paged_attention(const uint16_t *q, int64_t T, int64_t ldq, int64_t n_q_heads, int64_t n_kv_heads, const int32_t *row_start,
                           int64_t n_seqs, int64_t max_new, const void *pages, int64_t n_pages, int64_t page_len, int kv_dtype,
                           const float *k_scale, const float *v_scale, const int32_t *table, int64_t table_ld, int64_t max_pages,
                           const int32_t *lengths, uint16_t *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!q || !out) return QUASAR_ERR_NULL;
    PagedAttnParams p{};
    const CacheArgs a{T, n_q_heads, n_kv_heads, pages, n_pages, page_len, kv_dtype, k_scale, v_scale, table, table_ld, n_seqs, max_pages, lengths, row_start};
    if (const int e = check_cache(a, p.c)) return e;
    StepShape shape{};
    if (!step_shape(max_new, n_q_heads, n_kv_heads, kv_type(kv_dtype), shape)) return QUASAR_ERR_SHAPE;
    if (ldq < n_q_heads * kHeadDim || ldo < n_q_heads * kHeadDim || ldq % 8 || ldo % 4) return QUASAR_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(out, 8)) return QUASAR_ERR_ALIGN;
    if (!workspace || workspace_bytes < quasar_paged_attention_workspace_bytes(max_new, n_q_heads, n_kv_heads)) return QUASAR_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUASAR_ERR_ALIGN;
    p.q = q; p.out = out; p.ldq = ldq; p.ldo = ldo;
    p.part_o = static_cast<f32x4 *>(workspace);
    p.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + shape.part_o);
    p.pieces = reinterpret_cast<int *>(static_cast<unsigned char *>(workspace) + shape.part_o + shape.part_ml);
    p.workers = shape.workers; p.max_new = (int)max_new;
    p.scale_log2 = kScaleLog2;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return kv_type(kv_dtype) == KV_BF16 ? launch_step<KV_BF16>(p, shape, st) : launch_step<KV_E4M3>(p, shape, st);
}

size_t quasar_prompt_attention_workspace_bytes(int64_t T, int64_t n_q_heads, int64_t n_kv_heads, int64_t n_seqs) {
    if (T < 1 || T > kMaxPositions || check_heads(n_q_heads, n_kv_heads) || n_seqs < 1 || n_seqs > kMaxSeqs) return 0;
    const PromptShape a = prompt_shape(T, n_q_heads, n_kv_heads, n_seqs);
    return a.part_o + a.part_ml + a.pieces;
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
    const PromptShape shape = prompt_shape(T, n_q_heads, n_kv_heads, n_seqs);
    if (workspace && shape.workers && workspace_bytes >= shape.part_o + shape.part_ml + shape.pieces && max_pages * page_len > kFlatPositions) {
        p.workers = shape.workers;
        p.part_o = static_cast<f32x4 *>(workspace);
        p.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + shape.part_o);
        p.pieces = reinterpret_cast<int *>(static_cast<unsigned char *>(workspace) + shape.part_o + shape.part_ml);
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return kv_type(kv_dtype) == KV_BF16 ? launch_prompt<KV_BF16>(p, shape, st) : launch_prompt<KV_E4M3>(p, shape, st);
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
