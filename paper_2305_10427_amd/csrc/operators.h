// Internal launch interface of the beam-search operators: selection over beams
// and vocabulary, attention over a paged cache, operations on the cache's pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace pdec {

enum CacheType { CT_F32 = DT_F32, CT_BF16 = DT_BF16, CT_INT4 = 2 };

constexpr int kMaxBeam = 64;         // beams of one sentence (one candidate list per lane of a wave)
constexpr int kMaxQueriesPerKv = 16; // query heads that share a key/value head

// A pool of pages for the keys and values of `layers` layers.  Page id p of
// layer l is the p-th page of that layer in each array:
//   k [layers][pages][kv_heads][page_size][dh]       v [layers][pages][kv_heads][dh][page_size]
// in the storage type; in 4 bits the last axis is packed, eight values to a
// 32-bit word with value e at bit 4 (e / 2 + 4 (e & 1)), so that one AND leaves
// two neighbours of a word in the two halves of a register; ks, vs
// [layers][pages][kv_heads][page_size][groups][2] hold the (step, least value)
// in bfloat16 of each group of min(dh, 32) dimensions of a token's head vector.
struct CacheView {
  int type, layers, pages, ps, kv_heads, dh, groups;
  char *k, *v, *ks, *vs;
  __host__ __device__ size_t kv_page_bytes() const {      // of k (or v), one layer
    const size_t n = static_cast<size_t>(kv_heads) * ps * dh;
    return type == CT_F32 ? 4 * n : type == CT_BF16 ? 2 * n : n / 2;
  }
  __host__ __device__ size_t scale_page_bytes() const {   // of ks (or vs), one layer
    return type == CT_INT4 ? static_cast<size_t>(kv_heads) * ps * groups * 4 : 0;
  }
};

struct SelectArgs {
  const void* logits;      // [B beam][ld], rows of vocab values
  int dtype;
  long long ld;
  int B, beam, vocab;
  const float* scores;     // [B][beam]
  const int* lens;
  const int* done;
  const int* max_len;      // [B] or nullptr
  int eos_id, pad_id;
  float alpha;
  float* out_scores;
  int *out_parent, *out_token, *out_len, *out_done, *out_src, *out_flags;
  char* ws;
};
size_t select_workspace(int dtype, int B, int beam, int vocab);
size_t select_workspace_most(int rows, int beam);      // of any launch of up to so many rows
hipError_t launch_beam_select(const SelectArgs& a, hipStream_t s);

struct AttendArgs {
  CacheView c;
  int layer;
  const void* q;           // [n_seqs][q_ld], heads x dh values a row
  int q_bf16;
  long long q_ld;
  int heads;
  const void* new_k;       // [n_seqs][new_ld], kv_heads x dh values a row (nullptr: nothing is appended)
  const void* new_v;
  int new_bf16;
  long long new_ld;
  const int* table;        // [n_seqs][table_ld]
  int table_ld;
  const int* lens;
  int n_seqs, group, max_len;
  float scale;
  void* out;               // [n_seqs][out_ld], heads x dh values a row
  int out_bf16;
  long long out_ld;
  char* ws;
};
size_t attend_workspace(const CacheView& c, int n_seqs, int heads, int group, int max_len);
size_t attend_workspace_most(const CacheView& c);      // of any launch on such a cache
hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s);

struct ReadArgs {
  CacheView c;
  int layer;
  const int* table;
  int table_ld;
  const int* lens;
  int n_seqs;
  const int* first;        // [n_seqs] first position read of each sequence
  int count;
  float *out_k, *out_v;    // [n_seqs][count][kv_heads][dh]
};
hipError_t launch_cache_read(const ReadArgs& a, hipStream_t s);

struct PagesArgs {
  CacheView c;
  const int* table;        // [n_in][table_ld]
  int table_ld;
  const int* lens;         // [n_in]
  int n_in;
  const int* parents;      // [n_out] (fork)
  int n_out;
  int grow;
  int* out_table;          // [n_out][table_ld]
  int* out_lens;           // [n_out] (fork)
  int* refs;               // [pages]: references (fork), the new id of each page (compact)
  int* status;             // [2]
  char* ws;
};
size_t pages_workspace(const CacheView& c, int n_out);
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s);

// State of a beam decode (device arrays of R = B * beam rows unless noted).
struct BeamArgs {
  int B, beam, steps_max;
  float* scores;
  int *lens, *done, *parent, *token, *src;
  int* cache_lens;             // lengths of the first page table
  int *row_sent, *row_pos, *row_tok;
  int *k, *flags, *step_flags, *finished;   // [B]
  int2* hist;                  // [steps_max][R] (parent, token)
  int* step;                   // device scalar: steps done
  int* seq;                    // the context's control-step counter and host word, as CtrlArgs'
  int seq0;
  int* host_rows;
  int pad_id, bos_id, eos_id, flag_converged, flag_eos;
  int *out_ids, *out_len, *out_k, *out_flags;
  float* out_scores;
  int out_ld;
};
hipError_t launch_beam_init(const BeamArgs& a, hipStream_t s);
hipError_t launch_beam_step(const BeamArgs& a, hipStream_t s);
hipError_t launch_beam_out(const BeamArgs& a, hipStream_t s);

}  // namespace pdec
