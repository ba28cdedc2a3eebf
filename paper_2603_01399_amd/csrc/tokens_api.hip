// C entry points that draw and verify tokens from a batch's logits: checks on the host, launches.
#include "../../include/quasar.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <type_traits>

#include "tokens.hpp"

using namespace quasar;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
int launched() { return hipGetLastError() == hipSuccess ? QUASAR_OK : QUASAR_ERR_HIP; }

constexpr int64_t kMaxVocabulary = int64_t(1) << kIndexBits, kMaxTokenRows = int64_t(1) << 20;
// Rows whose parts are in the workspace at a time: more than fill the GPU several times over.
constexpr int64_t kRowsAtOnce = 512;

struct TokenRoom {
    int64_t nb, rows;
    size_t mass, count, chunk_max, part_max, rows_out, done;
    TokenRoom(int64_t T, int64_t V, bool drafts) {
        nb = (V + 7 + kPartTokens - 1) / kPartTokens;            // (a row may begin seven places behind a 16-byte border)
        rows = T < kRowsAtOnce ? T : kRowsAtOnce;
        mass = (size_t)(rows * nb) * kBuckets * 8;
        count = (size_t)(rows * nb) * kBuckets * 4;
        chunk_max = (size_t)(rows * nb) * part_chunks<0> * 4;            // (fp32's chunks are the smaller ones)
        part_max = ((size_t)(rows * nb) * 4 + 15) & ~(size_t)15;
        rows_out = drafts ? ((size_t)T * 4 + 15) & ~(size_t)15 : 0;
        done = drafts ? kMaxSeqs * 4 : 0;
    }
    size_t bytes() const { return mass + count + chunk_max + part_max + 2 * rows_out + done; }
};
bool token_shape(int64_t T, int64_t V) { return T >= 1 && T <= kMaxTokenRows && V >= 1 && V <= kMaxVocabulary; }

int check_tokens(TokenParams &p, int dtype, int64_t T, int64_t V, int64_t ld, const void *workspace, size_t workspace_bytes, const TokenRoom &room) {
    if (dtype != QUASAR_F32 && dtype != QUASAR_BF16) return QUASAR_ERR_DTYPE;
    if (!token_shape(T, V) || (ld < V && ld != 0) || ld > (int64_t(1) << 40)) return QUASAR_ERR_SHAPE;
    if (!aligned(p.logits, dtype == QUASAR_BF16 ? 2 : 4) || !aligned(p.temperature, 4) || !aligned(p.top_k, 4) || !aligned(p.top_p, 4) || !aligned(p.min_p, 4) ||
        !aligned(p.u, 4) || !aligned(p.u_accept, 4) || !aligned(p.p, 4) || !aligned(p.draft, 4) || !aligned(p.row_start, 4))
        return QUASAR_ERR_ALIGN;
    if (!workspace || workspace_bytes < room.bytes()) return QUASAR_ERR_WORKSPACE;
    return aligned(workspace, 16) ? QUASAR_OK : QUASAR_ERR_ALIGN;
}

// The opt-in to more dynamic LDS than the default, once for each kernel and device (done: a bit a device).
bool large_lds(const void *kernel, std::atomic<unsigned long long> &done) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load() & bit)) return true;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (kMaxTokenParts * part_chunks<0> + kChunkTurn) * (int)sizeof(unsigned short)) != hipSuccess) return false;
    if (dev < 64) done.fetch_or(bit);
    return true;
}

template <int DT>
int launch_tokens(TokenParams p, const TokenRoom &room, int64_t T, hipStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const unsigned int chunks = ((unsigned int)room.nb * part_chunks<DT> + kChunkTurn) * sizeof(unsigned short);
    if (!large_lds(reinterpret_cast<const void *>(token_draw_kernel<DT>), done)) return QUASAR_ERR_HIP;
    for (int64_t row0 = 0; row0 < T; row0 += room.rows) {
        const unsigned int rows = (unsigned int)(T - row0 < room.rows ? T - row0 : room.rows);
        p.row0 = (int)row0;
        hipLaunchKernelGGL(token_parts_kernel<DT>, dim3((unsigned int)room.nb, rows), dim3(kPartThreads), 0, st, p);
        if (const int e = launched()) return e;
        hipLaunchKernelGGL(token_draw_kernel<DT>, dim3(rows), dim3(kDrawThreads), chunks, st, p);
        if (const int e = launched()) return e;
    }
    return QUASAR_OK;
}

int run_tokens(TokenParams &p, int dtype, const TokenRoom &room, int64_t T, void *workspace, hipStream_t st) {
    unsigned char *at = static_cast<unsigned char *>(workspace);
    auto take = [&](size_t bytes) {
        unsigned char *here = at;
        at += bytes;
        return here;
    };
    p.mass = reinterpret_cast<u64 *>(take(room.mass));
    p.count = reinterpret_cast<unsigned int *>(take(room.count));
    p.chunk_max = reinterpret_cast<float *>(take(room.chunk_max));
    p.part_max = reinterpret_cast<float *>(take(room.part_max));
    if (room.rows_out) {
        p.token = reinterpret_cast<int32_t *>(take(room.rows_out));
        p.accepted = reinterpret_cast<int32_t *>(take(room.rows_out));
        p.done = reinterpret_cast<int32_t *>(take(room.done));
    }
    p.nb = (int)room.nb;
    return dtype == QUASAR_BF16 ? launch_tokens<1>(p, room, T, st) : launch_tokens<0>(p, room, T, st);
}

}  // namespace

extern "C" {

size_t quasar_sample_tokens_workspace_bytes(int64_t T, int64_t V) { return token_shape(T, V) ? TokenRoom(T, V, false).bytes() : 0; }
size_t quasar_verify_tokens_workspace_bytes(int64_t T, int64_t V) { return token_shape(T, V) ? TokenRoom(T, V, true).bytes() : 0; }

int quasar_sample_tokens(const void *logits, int logits_dtype, int64_t T, int64_t V, int64_t ld, const float *temperature, const int32_t *top_k,
                         const float *top_p, const float *min_p, const float *u, int32_t *out_token, float *out_p, void *workspace,
                         size_t workspace_bytes, void *hip_stream) {
    if (!logits || !u || !out_token) return QUASAR_ERR_NULL;
    TokenParams p{};
    p.logits = logits; p.ld = ld;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
    p.u = u; p.token = out_token; p.p = out_p;
    const TokenRoom room(token_shape(T, V) ? T : 1, token_shape(T, V) ? V : 1, false);
    if (const int e = check_tokens(p, logits_dtype, T, V, ld, workspace, workspace_bytes, room)) return e;
    if (!aligned(out_token, 4)) return QUASAR_ERR_ALIGN;
    p.V = (int)V; p.T = (int)T;
    return run_tokens(p, logits_dtype, room, T, workspace, static_cast<hipStream_t>(hip_stream));
}

int quasar_verify_tokens(const void *logits, int logits_dtype, int64_t T, int64_t V, int64_t ld, const int32_t *row_start, int64_t n_seqs,
                         const int32_t *draft_ids, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                         const float *u_accept, const float *u_sample, int32_t *out_accept_len, int32_t *out_token, float *out_p_draft,
                         void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!logits || !row_start || !draft_ids || !u_accept || !u_sample || !out_accept_len || !out_token) return QUASAR_ERR_NULL;
    TokenParams p{};
    p.logits = logits; p.ld = ld;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
    p.row_start = row_start; p.draft = draft_ids; p.u_accept = u_accept; p.u = u_sample; p.p = out_p_draft;
    const TokenRoom room(token_shape(T, V) ? T : 1, token_shape(T, V) ? V : 1, true);
    if (n_seqs < 1 || n_seqs > kMaxSeqs) return QUASAR_ERR_SHAPE;
    if (const int e = check_tokens(p, logits_dtype, T, V, ld, workspace, workspace_bytes, room)) return e;
    if (!aligned(out_accept_len, 4) || !aligned(out_token, 4)) return QUASAR_ERR_ALIGN;
    p.V = (int)V; p.T = (int)T; p.n_seqs = (int)n_seqs;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    p.out_accept_len = out_accept_len; p.out_token = out_token;
    return run_tokens(p, logits_dtype, room, T, workspace, st);
}

}  // extern "C"
