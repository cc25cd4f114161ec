// C entry points of the beam-search operators (include/pdec.h): argument
// checks and launches.  Nothing here allocates, synchronises or throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "operators.h"
#include "../../include/pdec.h"

using namespace pdec;

namespace {

pd_status fail(pd_status st, const char* msg) { return fail_with(st, msg); }

pd_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return PD_OK;
  char msg[160];
  std::snprintf(msg, sizeof msg, "%s launch: %s", what, hipGetErrorString(e));
  return fail(PD_E_DEVICE, msg);
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

constexpr long long kMaxRows = 1LL << 22;        // workgroups of the largest launch
constexpr long long kMaxBeams = 1LL << 20;       // of the selection, whose workgroups are larger
constexpr long long kMaxPositions = 1LL << 30;   // tokens a table row can name

// The shape of a cache (its buffers aside).
pd_status check_shape(const pd_cache* c) {
  if (c == nullptr) return fail(PD_E_ARG, "null cache");
  if (c->dtype != PD_F32 && c->dtype != PD_BF16 && c->dtype != PD_INT4)
    return fail(PD_E_ARG, "cache dtype must be PD_F32, PD_BF16 or PD_INT4");
  if (c->layers < 1 || c->pages < 1 || c->kv_heads < 1) return fail(PD_E_ARG, "layers, pages and kv_heads must be >= 1");
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
    return fail(PD_E_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  if (c->head_dim != 16 && c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return fail(PD_E_UNSUPPORTED, "head_dim must be 16, 32, 64 or 128");
  if (c->layers > 4096 || c->kv_heads > 1024 || c->pages > (1 << 24))
    return fail(PD_E_SHAPE, "at most 4096 layers, 1024 kv_heads and 2^24 pages");
  return PD_OK;
}

CacheView view(const pd_cache* c) {
  CacheView v;
  v.type = c->dtype;
  v.layers = c->layers;
  v.pages = c->pages;
  v.ps = c->page_size;
  v.kv_heads = c->kv_heads;
  v.dh = c->head_dim;
  v.groups = c->head_dim > 32 ? c->head_dim / 32 : 1;
  v.k = static_cast<char*>(c->k);
  v.v = static_cast<char*>(c->v);
  v.ks = static_cast<char*>(c->k_scale);
  v.vs = static_cast<char*>(c->v_scale);
  return v;
}

pd_status check_cache(const pd_cache* c) {
  const pd_status st = check_shape(c);
  if (st != PD_OK) return st;
  if (c->k == nullptr || c->v == nullptr || !aligned(c->k, 16) || !aligned(c->v, 16))
    return fail(PD_E_ARG, "k and v must be non-null and 16-byte aligned");
  if (c->dtype == PD_INT4 && (c->k_scale == nullptr || c->v_scale == nullptr || !aligned(c->k_scale, 16) ||
                              !aligned(c->v_scale, 16)))
    return fail(PD_E_ARG, "a cache in 4 bits needs k_scale and v_scale, 16-byte aligned");
  return PD_OK;
}

pd_status check_table(const pd_cache* c, const int32_t* table, int32_t table_ld, const int32_t* lens, int32_t n_seqs) {
  if (table == nullptr || lens == nullptr) return fail(PD_E_ARG, "null table or lens");
  if (n_seqs < 1 || table_ld < 1) return fail(PD_E_ARG, "n_seqs and table_ld must be >= 1");
  if (n_seqs > kMaxRows) return fail(PD_E_SHAPE, "more than 2^22 sequences");
  if (static_cast<long long>(table_ld) * c->page_size > kMaxPositions)
    return fail(PD_E_SHAPE, "table_ld * page_size exceeds 2^30");
  return PD_OK;
}

pd_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need > 0 && (ws == nullptr || !aligned(ws, 256))) return fail(PD_E_WORKSPACE, "workspace is null or not 256-byte aligned");
  if (have < need) {
    char msg[96];
    std::snprintf(msg, sizeof msg, "workspace too small: need %zu bytes", need);
    return fail(PD_E_WORKSPACE, msg);
  }
  return PD_OK;
}

pd_status check_select(int32_t dtype, int32_t B, int32_t beam, int32_t vocab) {
  if (dtype != PD_F32 && dtype != PD_BF16) return fail(PD_E_ARG, "logits must be PD_F32 or PD_BF16");
  if (B < 1 || beam < 1 || vocab < 1) return fail(PD_E_ARG, "B, beam and vocab must be >= 1");
  if (beam > kMaxBeam) return fail(PD_E_SHAPE, "at most 64 beams");
  if (vocab > (1 << 24) || static_cast<long long>(B) * beam > kMaxBeams)
    return fail(PD_E_SHAPE, "vocab exceeds 2^24 or B * beam exceeds 2^20");
  return PD_OK;
}

pd_status check_heads(const pd_cache* c, int32_t heads, int32_t n_seqs, int32_t group, int32_t max_len) {
  if (heads < 1 || heads % c->kv_heads != 0) return fail(PD_E_ARG, "heads must be a multiple of kv_heads");
  if (heads / c->kv_heads > kMaxQueriesPerKv) return fail(PD_E_UNSUPPORTED, "at most 16 query heads per key/value head");
  if (n_seqs < 1 || group < 1 || n_seqs % group != 0) return fail(PD_E_ARG, "n_seqs must be a positive multiple of group");
  if (max_len < 1) return fail(PD_E_ARG, "max_len must be >= 1");
  if (max_len > kMaxPositions) return fail(PD_E_SHAPE, "max_len exceeds 2^30");
  if (static_cast<long long>(n_seqs) * heads > kMaxRows) return fail(PD_E_SHAPE, "n_seqs * heads exceeds 2^22");
  return PD_OK;
}

}  // namespace

extern "C" {

pd_status pd_beam_select_bytes(int32_t dtype, int32_t B, int32_t beam, int32_t vocab, size_t* bytes) {
  if (bytes == nullptr) return fail(PD_E_ARG, "null argument");
  const pd_status st = check_select(dtype, B, beam, vocab);
  if (st != PD_OK) return st;
  *bytes = select_workspace(dtype, B, beam, vocab);
  return PD_OK;
}

pd_status pd_beam_select(const void* logits, int32_t dtype, int64_t ld, int32_t B, int32_t beam, int32_t vocab,
                         const float* scores, const int32_t* lens, const int32_t* done, const int32_t* max_len,
                         int32_t eos_id, int32_t pad_id, float alpha, float* out_scores, int32_t* out_parent,
                         int32_t* out_token, int32_t* out_len, int32_t* out_done, int32_t* out_src,
                         int32_t* out_flags, void* workspace, size_t workspace_bytes, void* stream) {
  if (logits == nullptr || scores == nullptr || lens == nullptr || done == nullptr || out_scores == nullptr ||
      out_parent == nullptr || out_token == nullptr || out_len == nullptr || out_done == nullptr ||
      out_src == nullptr || out_flags == nullptr)
    return fail(PD_E_ARG, "null argument");
  pd_status st = check_select(dtype, B, beam, vocab);
  if (st != PD_OK) return st;
  if (ld < vocab || ld > (1LL << 40)) return fail(PD_E_ARG, "ld must be in [vocab, 2^40]");
  if (!aligned(logits, dtype == PD_BF16 ? 2 : 4)) return fail(PD_E_ARG, "logits are misaligned");
  if (!(alpha >= 0.f) || !std::isfinite(alpha)) return fail(PD_E_ARG, "alpha must be finite and >= 0");
  if ((st = check_workspace(workspace, workspace_bytes, select_workspace(dtype, B, beam, vocab))) != PD_OK) return st;
  const SelectArgs a{logits, dtype, ld, B, beam, vocab, scores, lens, done, max_len, eos_id, pad_id, alpha,
                     out_scores, out_parent, out_token, out_len, out_done, out_src, out_flags,
                     static_cast<char*>(workspace)};
  return launched(launch_beam_select(a, static_cast<hipStream_t>(stream)), "beam selection");
}

pd_status pd_cache_bytes(const pd_cache* cache, size_t* kv_bytes, size_t* scale_bytes) {
  if (kv_bytes == nullptr || scale_bytes == nullptr) return fail(PD_E_ARG, "null argument");
  const pd_status st = check_shape(cache);
  if (st != PD_OK) return st;
  const CacheView v = view(cache);
  const size_t n = static_cast<size_t>(v.layers) * v.pages;
  *kv_bytes = n * v.kv_page_bytes();
  *scale_bytes = n * v.scale_page_bytes();
  return PD_OK;
}

pd_status pd_cache_attend_bytes(const pd_cache* cache, int32_t heads, int32_t n_seqs, int32_t group, int32_t max_len,
                                size_t* bytes) {
  if (bytes == nullptr) return fail(PD_E_ARG, "null argument");
  pd_status st = check_shape(cache);
  if (st != PD_OK) return st;
  if ((st = check_heads(cache, heads, n_seqs, group, max_len)) != PD_OK) return st;
  *bytes = attend_workspace(view(cache), n_seqs, heads, group, max_len);
  return PD_OK;
}

pd_status pd_cache_attend(const pd_cache* cache, int32_t layer, const void* q, int32_t q_dtype, int64_t q_ld,
                          int32_t heads, const void* new_k, const void* new_v, int32_t new_dtype, int64_t new_ld,
                          const int32_t* table, int32_t table_ld, const int32_t* lens, int32_t n_seqs, int32_t group,
                          int32_t max_len, float scale, void* out, int32_t out_dtype, int64_t out_ld, void* workspace,
                          size_t workspace_bytes, void* stream) {
  pd_status st = check_cache(cache);
  if (st != PD_OK) return st;
  if (layer < 0 || layer >= cache->layers) return fail(PD_E_ARG, "layer out of range");
  if (q == nullptr || out == nullptr) return fail(PD_E_ARG, "null q or out");
  if ((q_dtype != PD_F32 && q_dtype != PD_BF16) || (out_dtype != PD_F32 && out_dtype != PD_BF16))
    return fail(PD_E_ARG, "q and out must be PD_F32 or PD_BF16");
  if ((st = check_heads(cache, heads, n_seqs, group, max_len)) != PD_OK) return st;
  if ((st = check_table(cache, table, table_ld, lens, n_seqs)) != PD_OK) return st;
  const int64_t row = static_cast<int64_t>(heads) * cache->head_dim;
  const int64_t kv_row = static_cast<int64_t>(cache->kv_heads) * cache->head_dim;
  if (q_ld < row || out_ld < row || q_ld > kMaxPositions || out_ld > kMaxPositions)
    return fail(PD_E_ARG, "q_ld and out_ld must be in [heads * head_dim, 2^30]");
  if (q_ld % 8 != 0 || out_ld % 8 != 0 || !aligned(q, 16) || !aligned(out, 16))
    return fail(PD_E_ARG, "rows of q and out must be 16-byte aligned (ld a multiple of 8)");
  if ((new_k == nullptr) != (new_v == nullptr)) return fail(PD_E_ARG, "new_k and new_v go together");
  if (new_k != nullptr) {
    if (new_dtype != PD_F32 && new_dtype != PD_BF16) return fail(PD_E_ARG, "new_k and new_v must be PD_F32 or PD_BF16");
    if (new_ld < kv_row || new_ld > kMaxPositions) return fail(PD_E_ARG, "new_ld must be in [kv_heads * head_dim, 2^30]");
    if (new_ld % 8 != 0 || !aligned(new_k, 16) || !aligned(new_v, 16))
      return fail(PD_E_ARG, "rows of new_k and new_v must be 16-byte aligned (ld a multiple of 8)");
  }
  if (!std::isfinite(scale)) return fail(PD_E_ARG, "scale must be finite");
  const CacheView v = view(cache);
  if ((st = check_workspace(workspace, workspace_bytes, attend_workspace(v, n_seqs, heads, group, max_len))) != PD_OK)
    return st;
  const AttendArgs a{v, layer, q, q_dtype == PD_BF16, q_ld, heads, new_k, new_v, new_dtype == PD_BF16, new_ld, table,
                     table_ld, lens, n_seqs, group, max_len, scale, out, out_dtype == PD_BF16, out_ld,
                     static_cast<char*>(workspace)};
  return launched(launch_cache_attend(a, static_cast<hipStream_t>(stream)), "cache attention");
}

pd_status pd_cache_read(const pd_cache* cache, int32_t layer, const int32_t* table, int32_t table_ld,
                        const int32_t* lens, int32_t n_seqs, const int32_t* first, int32_t count, float* out_k,
                        float* out_v, void* stream) {
  pd_status st = check_cache(cache);
  if (st != PD_OK) return st;
  if (layer < 0 || layer >= cache->layers) return fail(PD_E_ARG, "layer out of range");
  if ((st = check_table(cache, table, table_ld, lens, n_seqs)) != PD_OK) return st;
  if (first == nullptr || out_k == nullptr || out_v == nullptr) return fail(PD_E_ARG, "null argument");
  if (count < 1) return fail(PD_E_ARG, "count must be >= 1");
  if (static_cast<long long>(n_seqs) * count > (1LL << 40)) return fail(PD_E_SHAPE, "n_seqs * count exceeds 2^40");
  const ReadArgs a{view(cache), layer, table, table_ld, lens, n_seqs, first, count, out_k, out_v};
  return launched(launch_cache_read(a, static_cast<hipStream_t>(stream)), "cache read");
}

pd_status pd_pages_bytes(const pd_cache* cache, int32_t n_seqs, size_t* bytes) {
  if (bytes == nullptr) return fail(PD_E_ARG, "null argument");
  const pd_status st = check_shape(cache);
  if (st != PD_OK) return st;
  if (n_seqs < 1) return fail(PD_E_ARG, "n_seqs must be >= 1");
  if (n_seqs > kMaxRows) return fail(PD_E_SHAPE, "more than 2^22 sequences");
  *bytes = pages_workspace(view(cache), n_seqs);
  return PD_OK;
}

pd_status pd_pages_fork(const pd_cache* cache, const int32_t* table, int32_t table_ld, const int32_t* lens,
                        int32_t n_seqs, const int32_t* parents, int32_t n_out, int32_t grow, int32_t* out_table,
                        int32_t* out_lens, int32_t* out_refs, int32_t* out_status, void* workspace,
                        size_t workspace_bytes, void* stream) {
  pd_status st = check_cache(cache);
  if (st != PD_OK) return st;
  if ((st = check_table(cache, table, table_ld, lens, n_seqs)) != PD_OK) return st;
  if (parents == nullptr || out_table == nullptr || out_lens == nullptr || out_refs == nullptr || out_status == nullptr)
    return fail(PD_E_ARG, "null argument");
  if (n_out < 1) return fail(PD_E_ARG, "n_out must be >= 1");
  if (n_out > kMaxRows) return fail(PD_E_SHAPE, "more than 2^22 sequences");
  const size_t row = sizeof(int32_t) * static_cast<size_t>(table_ld);
  if (overlap(table, row * n_seqs, out_table, row * n_out) ||
      overlap(lens, sizeof(int32_t) * static_cast<size_t>(n_seqs), out_lens, sizeof(int32_t) * static_cast<size_t>(n_out)))
    return fail(PD_E_ARG, "the new table and lengths must not overlap the old ones");
  const CacheView v = view(cache);
  if ((st = check_workspace(workspace, workspace_bytes, pages_workspace(v, n_out))) != PD_OK) return st;
  const PagesArgs a{v, table, table_ld, lens, n_seqs, parents, n_out, grow != 0, out_table, out_lens, out_refs,
                    out_status, static_cast<char*>(workspace)};
  return launched(launch_pages_fork(a, static_cast<hipStream_t>(stream)), "page fork");
}

pd_status pd_pages_compact(const pd_cache* cache, const int32_t* table, int32_t table_ld, const int32_t* lens,
                           int32_t n_seqs, int32_t* out_table, int32_t* out_remap, int32_t* out_status,
                           void* workspace, size_t workspace_bytes, void* stream) {
  pd_status st = check_cache(cache);
  if (st != PD_OK) return st;
  if ((st = check_table(cache, table, table_ld, lens, n_seqs)) != PD_OK) return st;
  if (out_table == nullptr || out_remap == nullptr || out_status == nullptr) return fail(PD_E_ARG, "null argument");
  const size_t bytes = sizeof(int32_t) * static_cast<size_t>(table_ld) * n_seqs;
  if (table != out_table && overlap(table, bytes, out_table, bytes))
    return fail(PD_E_ARG, "out_table must be the table itself or not overlap it");
  const CacheView v = view(cache);
  if ((st = check_workspace(workspace, workspace_bytes, pages_workspace(v, n_seqs))) != PD_OK) return st;
  const PagesArgs a{v, table, table_ld, lens, n_seqs, nullptr, 0, 0, out_table, nullptr, out_remap, out_status,
                    static_cast<char*>(workspace)};
  return launched(launch_pages_compact(a, static_cast<hipStream_t>(stream)), "page compaction");
}

}  // extern "C"
