// Beam search's selection over beams and vocabulary.
//
// For the live beam k of a sentence with score s, length n and logits x_v:
//   lse = log sum_v exp(x_v),  c_v = s + (x_v - lse),  key_v = c_v / (n + 1)^alpha;
// a finished beam has one candidate, itself: c = s, key = s / n^alpha.  The
// `beam` candidates of largest key survive.  Within a beam the order of the
// keys is that of the logits, so a row's best `beam` logits are found first
// (k_select_rows, with the row's log-sum-exp) and a sentence's rows are merged
// by key (k_select_merge).  Keys are compared in double: neighbouring keys of
// different rows differ by the rounding of their log-sum-exps.
#include "common.h"
#include "operators.h"

namespace pdec {

namespace {

constexpr int kRowThreads = 256;

// Scratch of a launch: each row's best logits with their words (best first;
// word -1: none), its log-sum-exp, and whether it held a NaN or +inf.
struct SelectWs {
  float* val;
  int* word;
  double* lse;
  int* bad;
};

SelectWs carve(char* ws, int rows, int beam) {
  SelectWs w;
  w.lse = reinterpret_cast<double*>(ws);
  w.val = reinterpret_cast<float*>(w.lse + rows);
  w.word = reinterpret_cast<int*>(w.val + static_cast<size_t>(rows) * beam);
  w.bad = w.word + static_cast<size_t>(rows) * beam;
  return w;
}

__device__ __forceinline__ bool row_live(const SelectArgs& a, int row) {
  return a.done[row] == 0 && isfinite(a.scores[row]);
}

// NaN and +inf are left out like -inf (and reported); -0 counts as 0.
__device__ __forceinline__ float usable(float x, int& bad) {
  if (x != x || x == INFINITY) {
    bad = 1;
    return -INFINITY;
  }
  return x + 0.f;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_select_rows(SelectArgs a, SelectWs w) {
  const int row = blockIdx.x, t = threadIdx.x;
  if (!row_live(a, row)) return;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld;
  __shared__ float s_v[kRowThreads];
  __shared__ int s_i[kRowThreads];
  __shared__ double s_d[kRowThreads];
  int bad = 0;
  float last = INFINITY, top = -INFINITY;
  int last_i = -1;
  for (int r = 0; r < a.beam; ++r) {
    float bv = -INFINITY;
    int bi = -1;
    for (int i = t; i < a.vocab; i += kRowThreads) {
      const float v = usable(Elt<T>::load(x, i), bad);
      if ((v < last || (v == last && i > last_i)) && v > bv) { bv = v; bi = i; }
    }
    s_v[t] = bv;
    s_i[t] = bi;
    __syncthreads();
    for (int o = kRowThreads / 2; o > 0; o >>= 1) {
      if (t < o) {
        const float v = s_v[t + o];
        const int i = s_i[t + o];
        if (v > s_v[t] || (v == s_v[t] && i >= 0 && (s_i[t] < 0 || i < s_i[t]))) { s_v[t] = v; s_i[t] = i; }
      }
      __syncthreads();
    }
    last = s_v[0];
    last_i = s_i[0];
    if (r == 0) top = last;
    __syncthreads();
    if (t == 0) {
      w.val[static_cast<size_t>(row) * a.beam + r] = last;
      w.word[static_cast<size_t>(row) * a.beam + r] = last_i;
    }
    if (last_i < 0) last = -INFINITY, last_i = a.vocab;   // nothing is left
  }
  double sum = 0.0;
  for (int i = t; i < a.vocab; i += kRowThreads) {
    const float v = usable(Elt<T>::load(x, i), bad);
    if (v > -INFINITY) sum += exp(static_cast<double>(v) - static_cast<double>(top));
  }
  s_d[t] = sum;
  s_i[t] = bad;
  __syncthreads();
  for (int o = kRowThreads / 2; o > 0; o >>= 1) {
    if (t < o) { s_d[t] += s_d[t + o]; s_i[t] |= s_i[t + o]; }
    __syncthreads();
  }
  if (t == 0) {
    w.lse[row] = static_cast<double>(top) + log(s_d[0]);
    w.bad[row] = s_i[0];
  }
}

constexpr int kMergeThreads = 256;

__global__ __launch_bounds__(kMergeThreads) void k_select_merge(SelectArgs a, SelectWs w) {
  const int b = blockIdx.x, t = threadIdx.x, K = a.beam;
  __shared__ double s_key[kMaxBeam * kMaxBeam];
  __shared__ int s_bad;
  if (t == 0) s_bad = 0;
  __syncthreads();
  auto cum_of = [&](int k, int r) -> double {   // the candidate's score, -inf if there is none
    const int row = b * K + k;
    if (!isfinite(a.scores[row])) return -INFINITY;
    if (a.done[row] != 0) return r == 0 ? static_cast<double>(a.scores[row]) : -INFINITY;
    const size_t at = static_cast<size_t>(row) * K + r;
    if (w.word[at] < 0) return -INFINITY;
    return static_cast<double>(a.scores[row]) + (static_cast<double>(w.val[at]) - w.lse[row]);
  };
  for (int c = t; c < K * K; c += kMergeThreads) {
    const int k = c / K, row = b * K + k;
    const int n = a.lens[row] + (a.done[row] != 0 ? 0 : 1);
    s_key[c] = cum_of(k, c - k * K) / pow(static_cast<double>(n > 1 ? n : 1), static_cast<double>(a.alpha));
    if (c == k * K && row_live(a, row) && w.bad[row]) s_bad = 1;
  }
  __syncthreads();
  // every candidate counts those before it: (key, beam, rank in the beam)
  float o_score = -INFINITY;
  int o_par = -1, o_tok = a.pad_id, o_len = 0, o_done = 1;
  __shared__ int s_at[kMaxBeam];
  if (t < K) s_at[t] = -1;
  __syncthreads();
  for (int c = t; c < K * K; c += kMergeThreads) {
    const double key = s_key[c];
    if (!(key > -INFINITY)) continue;
    int rank = 0;
    for (int o = 0; o < K * K; ++o) rank += s_key[o] > key || (s_key[o] == key && o < c);
    if (rank < K) s_at[rank] = c;
  }
  __syncthreads();
  if (t < K && s_at[t] >= 0) {
    const int c = s_at[t], k = c / K, r = c - k * K, row = b * K + k;
    const bool fin = a.done[row] != 0;
    o_score = static_cast<float>(cum_of(k, r));
    o_par = k;
    o_tok = fin ? a.pad_id : w.word[static_cast<size_t>(row) * K + r];
    o_len = a.lens[row] + (fin ? 0 : 1);
    o_done = fin || o_tok == a.eos_id || (a.max_len != nullptr && o_len >= a.max_len[b]) ? 1 : 0;
  }
  __syncthreads();   // the outputs may be the inputs' own arrays
  if (t < K) {
    const int o = b * K + t;
    a.out_scores[o] = o_score;
    a.out_parent[o] = o_par;
    a.out_token[o] = o_tok;
    a.out_len[o] = o_len;
    a.out_done[o] = o_done;
    a.out_src[o] = o_done ? -1 : b * K + o_par;
  }
  if (t == 0) a.out_flags[b] = s_bad ? 8 : 0;
}

}  // namespace

size_t select_workspace(int B, int beam, int vocab) {
  const size_t rows = static_cast<size_t>(B) * beam;
  return rows * (8 + 4) + rows * beam * 8;
}

hipError_t launch_beam_select(const SelectArgs& a, hipStream_t s) {
  const int rows = a.B * a.beam;
  const SelectWs w = carve(a.ws, rows, a.beam);
  if (a.dtype == DT_BF16) hipLaunchKernelGGL(k_select_rows<bf16_t>, dim3(rows), dim3(kRowThreads), 0, s, a, w);
  else hipLaunchKernelGGL(k_select_rows<float>, dim3(rows), dim3(kRowThreads), 0, s, a, w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_select_merge, dim3(a.B), dim3(kMergeThreads), 0, s, a, w);
  return hipGetLastError();
}

}  // namespace pdec
