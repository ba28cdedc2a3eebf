// The books of a paged cache and the copies they ask for (gfx950): reference counts of the pages, page table and lengths of the
// sequences, all in device memory, so that a step that ends with a length only the device knows goes on without the host.
//
// Every rule here names its result page by page (lowest free page first, in the order of sequences and columns), so that results do not
// depend on the order in which waves arrive; atomics only add integers.  What is read from the books is bounded before it is an index.
#pragma once

#include "paged.hpp"

namespace quasar {

struct BooksParams {
    int32_t *table, *lengths, *refs;
    long long table_ld;
    int n_seqs, columns, n_pages;
    int block_shift;
};
struct CopyItem { int src, dst, blocks, unused; };
struct CopyList { int count, unused[3]; CopyItem items[1]; };   // in the workspace

__device__ __forceinline__ bool is_page(const BooksParams &b, int id) { return page_exists(id, b.n_pages); }

// Exclusive prefix sum over the 1024 threads of a workgroup; `total` for all.  wave_sums: [16] of LDS.
__device__ __forceinline__ int exclusive_scan_1024(int v, int *wave_sums, int &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int sum = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int up = __shfl_up(sum, off, 64);
        if (lane >= off) sum += up;
    }
    __syncthreads();                                             // (wave_sums may still be read from the last scan)
    if (lane == 63) wave_sums[w] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        before += i < w ? wave_sums[i] : 0;
        total += wave_sums[i];
    }
    return before + sum - v;
}

// ---------------------------------------------------------------------------------------------
// Room for new positions.  One workgroup, a thread a sequence; sequences that want more than four pages are walked by whole waves.
// free_list: [n_pages] of the workspace.  4.5 us for 48 sequences: six trips to memory one after another, each a barrier; the call, with the
// launch of the copies behind it (2.1 us when there are none), 12 to 13.  Over 32768 pages of which the last are free 38: 0.8 us a turn of 1024.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void pages_reserve_kernel(const BooksParams b, const int32_t *n_new, int32_t *status, int *free_list,
                                                             CopyList *copies) {
    __shared__ int wave_sums[16], last_page[kMaxSeqs], wanted_of[kMaxSeqs], first_of[kMaxSeqs], need_of[kMaxSeqs];
    __shared__ int n_copies;
    const int s = threadIdx.x, lane = s & 63, w = s >> 6;
    const int page_shift = b.block_shift + 5, page_mask = (1 << page_shift) - 1;
    if (s == 0) n_copies = 0;
    int len = 0, n = 0, first = 0, need = 0, last = -1;
    if (s < b.n_seqs) {
        len = b.lengths[s];
        n = n_new[s];
    }
    bool asks = n > 0 && len >= 0 && len <= kMaxPositions && n <= kMaxPositions;
    if (asks) {
        first = len >> page_shift;
        need = (len + n + page_mask) >> page_shift;
        asks = need <= b.columns;
    }
    int32_t *row = b.table + s * b.table_ld;
    bool copied = false;
    if (asks && (len & page_mask)) {
        last = row[first];
        if (!is_page(b, last)) last = -1;
    }
    last_page[s] = last;
    __syncthreads();
    if (last >= 0) {
        const int held = b.refs[last];
        if (held > 1) {                                          // earlier writers of the page take copies first: the last holder keeps it
            int earlier = 0;
            for (int i = 0; i < s; ++i) earlier += last_page[i] == last;
            copied = held - earlier > 1;
        }
    }
    const bool by_wave = asks && need - first > 4;
    int wanted = copied;
    if (asks && !by_wave)
        for (int col = first; col < need; ++col) wanted += row[col] < 0;
    wanted_of[s] = by_wave ? wanted : -1;                        // (-1: counted)
    first_of[s] = first;
    need_of[s] = need;
    const bool any_by_wave = __syncthreads_or(by_wave);
    if (any_by_wave) {
        for (int i = w; i < b.n_seqs; i += 16) {
            if (wanted_of[i] < 0) continue;
            const int32_t *r = b.table + i * b.table_ld;
            int count = 0;
            for (int col = first_of[i]; col < need_of[i]; col += 64) {
                const bool empty = col + lane < need_of[i] && r[col + lane] < 0;
                count += __popcll(__builtin_amdgcn_ballot_w64(empty));
            }
            if (lane == 0) wanted_of[i] += count;
        }
        __syncthreads();
        if (by_wave) wanted = wanted_of[s];
    }
    int total;
    const int before = exclusive_scan_1024(wanted, wave_sums, total);
    // the lowest free pages, as many as are wanted
    int n_free = 0;
    for (int p0 = 0; p0 < b.n_pages && n_free < total; p0 += 1024) {
        const int id = p0 + s;
        const bool is_free = id < b.n_pages && b.refs[id] == 0;
        int got;
        const int rank = n_free + exclusive_scan_1024(is_free, wave_sums, got);
        if (is_free && rank < total) free_list[rank] = id;
        n_free += got;
    }
    __syncthreads();
    // the first sequence that finds too few, and those behind it, are left as they are
    const bool ok = asks && before + wanted <= n_free;
    if (s < b.n_seqs) status[s] = ok || n <= 0;
    int rank = before;
    if (ok && copied) {
        const int to = free_list[rank++];
        row[first] = to;
        b.refs[to] = 1;
        atomicSub(&b.refs[last], 1);
        copies->items[atomicAdd(&n_copies, 1)] = CopyItem{last, to, ((len & page_mask) + kKvBlock - 1) / kKvBlock, 0};
    }
    if (ok && !by_wave)
        for (int col = first; col < need; ++col)
            if (row[col] < 0) {
                const int to = free_list[rank++];
                row[col] = to;
                b.refs[to] = 1;
            }
    if (any_by_wave) {
        __syncthreads();
        wanted_of[s] = ok && by_wave ? rank : -1;
        __syncthreads();
        for (int i = w; i < b.n_seqs; i += 16) {
            int at = wanted_of[i];
            if (at < 0) continue;
            int32_t *r = b.table + i * b.table_ld;
            for (int col = first_of[i]; col < need_of[i]; col += 64) {
                const bool empty = col + lane < need_of[i] && r[col + lane] < 0;
                const unsigned long long mask = __builtin_amdgcn_ballot_w64(empty);
                if (empty) {
                    const int to = free_list[at + __popcll(mask & ((1ull << lane) - 1))];
                    r[col + lane] = to;
                    b.refs[to] = 1;
                }
                at += __popcll(mask);
            }
        }
    }
    __syncthreads();
    if (s == 0) copies->count = n_copies;
}

// ---------------------------------------------------------------------------------------------
// Fork, reorder, cut and free: row s takes the pages of row parent[s], as far as its new length reaches.  A workgroup takes 16 columns
// of all rows through LDS, since any row may be another's parent.
// ---------------------------------------------------------------------------------------------
constexpr int kForkColumns = 16;

__device__ __forceinline__ int forked_length(const BooksParams &b, const int32_t *parent, const int32_t *keep, int s, int &from) {
    from = parent[s];
    if ((unsigned int)from >= (unsigned int)b.n_seqs) from = -1;
    int len = from < 0 ? 0 : b.lengths[from];
    if (keep) len = min(len, keep[s]);
    return max(len, 0);
}

__global__ __launch_bounds__(256) void pages_fork_kernel(const BooksParams b, const int32_t *parent, const int32_t *keep) {
    extern __shared__ int old[];                                 // [n_seqs][kForkColumns]
    const int c0 = blockIdx.x * kForkColumns, cols = min(kForkColumns, b.columns - c0);
    const int page_shift = b.block_shift + 5, page_mask = (1 << page_shift) - 1;
    for (int i = threadIdx.x; i < b.n_seqs * kForkColumns; i += 256) {
        const int s = i / kForkColumns, col = i % kForkColumns;
        old[i] = col < cols ? b.table[s * b.table_ld + c0 + col] : -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < b.n_seqs * kForkColumns; i += 256) {
        const int s = i / kForkColumns, col = i % kForkColumns;
        if (col >= cols) continue;
        int from;
        const int len = forked_length(b, parent, keep, s, from);
        const int held = (int)(((long long)len + page_mask) >> page_shift);
        const int now = c0 + col < held ? old[from * kForkColumns + col] : -1;
        const int was = old[i];
        if (now == was) continue;
        b.table[s * b.table_ld + c0 + col] = now;
        if (is_page(b, now)) atomicAdd(&b.refs[now], 1);
        if (is_page(b, was)) atomicSub(&b.refs[was], 1);
    }
}

__global__ __launch_bounds__(1024) void pages_fork_lengths_kernel(const BooksParams b, const int32_t *parent, const int32_t *keep) {
    const int s = threadIdx.x;
    int from, len = 0;
    if (s < b.n_seqs) len = forked_length(b, parent, keep, s, from);
    __syncthreads();
    if (s < b.n_seqs) b.lengths[s] = len;
}

// ---------------------------------------------------------------------------------------------
// Compaction: with n pages in use, the i-th of those at n and beyond goes to the i-th free page below n.  One workgroup finds the
// pairs; tables and pages follow in a launch that fills the card.  holes, moved: [n_pages] of the workspace each.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void pages_compact_kernel(const BooksParams b, int32_t *to, int *holes, int *moved, CopyList *copies) {
    __shared__ int wave_sums[16];
    const int tid = threadIdx.x;
    int mine = 0, n_live;
    for (int id = tid; id < b.n_pages; id += 1024) mine += b.refs[id] > 0;
    exclusive_scan_1024(mine, wave_sums, n_live);
    int n_holes = 0, n_moved = 0;
    for (int p0 = 0; p0 < b.n_pages; p0 += 1024) {
        const int id = p0 + tid;
        const bool in = id < b.n_pages, live = in && b.refs[id] > 0;
        const bool hole = in && !live && id < n_live, moves = live && id >= n_live;
        int got;
        const int rank = exclusive_scan_1024((hole ? 1 : 0) + (moves ? 1 << 16 : 0), wave_sums, got);
        if (in) to[id] = id;
        if (hole) holes[n_holes + (rank & 0xFFFF)] = id;
        if (moves) moved[n_moved + (rank >> 16)] = id;
        n_holes += got & 0xFFFF;
        n_moved += got >> 16;
    }
    __syncthreads();                                             // (as many holes as moves: both are the pages in use less those below n_live)
    for (int i = tid; i < n_moved; i += 1024) {
        const int src = moved[i], dst = holes[i];
        to[src] = dst;
        b.refs[dst] = b.refs[src];
        b.refs[src] = 0;
        copies->items[i] = CopyItem{src, dst, 1 << b.block_shift, 0};
    }
    if (tid == 0) copies->count = n_moved;
}

// ---------------------------------------------------------------------------------------------
// Copies the listed pages of every layer, and (compaction) renames the pages in the table.  A task is a kv head of a page of a
// layer, contiguous; tasks go round the workgroups.  Bound by memory: 512 pages of 4 layers (1.07 GB moved) 207 us, 5.2 TB/s, as a plain copy;
// 56 last pages of 36 layers 170.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pages_copy_kernel(const BooksParams b, const CopyList *copies, const int32_t *to, unsigned char *pool,
                                                         int n_layers, int Hkv, int block_bytes /* keys and values of 32 positions of a head */) {
    if (to)
        for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)b.n_seqs * b.columns; i += (long long)gridDim.x * 256) {
            int32_t *entry = b.table + (i / b.columns) * b.table_ld + i % b.columns;
            const int id = *entry;
            if (is_page(b, id) && to[id] != id) *entry = to[id];
        }
    const long long head_bytes = (long long)block_bytes << b.block_shift, page_bytes = head_bytes * Hkv;
    const long long tasks = (long long)copies->count * n_layers * Hkv;
    for (long long t = blockIdx.x; t < tasks; t += gridDim.x) {
        const int h = (int)(t % Hkv), layer = (int)(t / Hkv % n_layers);
        const CopyItem item = copies->items[t / Hkv / n_layers];
        const long long layer_at = layer * page_bytes * b.n_pages + h * head_bytes;
        const u32x4 *src = reinterpret_cast<const u32x4 *>(pool + layer_at + item.src * page_bytes);
        u32x4 *dst = reinterpret_cast<u32x4 *>(pool + layer_at + item.dst * page_bytes);
        const int n = item.blocks * (block_bytes / 16);          // (a multiple of 512)
        for (int i = threadIdx.x; i < n; i += 512) {
            const u32x4 v0 = __builtin_nontemporal_load(src + i), v1 = __builtin_nontemporal_load(src + i + 256);
            __builtin_nontemporal_store(v0, dst + i);
            __builtin_nontemporal_store(v1, dst + i + 256);
        }
    }
}

}  // namespace quasar
