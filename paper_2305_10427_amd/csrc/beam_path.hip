// Control kernels of beam decoding (pd_decode_beam): the state before the first
// step, the book-keeping after a step's selection, and the hypotheses read back
// from the steps' (parent, token) records.
#include "common.h"
#include "operators.h"

namespace pdec {

namespace {

constexpr int kCtrlThreads = 1024;

__global__ __launch_bounds__(256) void k_beam_init(BeamArgs a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < a.B * a.beam) {
    const bool first = r % a.beam == 0;           // one live hypothesis a sentence: the empty one
    a.scores[r] = first ? 0.f : -INFINITY;
    a.lens[r] = 0;
    a.done[r] = 0;
    a.src[r] = first ? r : -1;
    a.cache_lens[r] = 0;
    a.row_sent[r] = r / a.beam;
    a.row_pos[r] = 0;
    a.row_tok[r] = a.bos_id;
  }
  if (r < a.B) {
    a.k[r] = 0;
    a.flags[r] = 0;
  }
  if (r == 0) {
    *a.step = 0;
    *a.seq = a.seq0;
    __hip_atomic_store(a.host_rows, host_word(a.B * a.beam, false, a.seq0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  }
}

// After a selection: records the survivors, lays out the next step's rows and
// publishes how many hypotheses are still growing.  One workgroup: the next
// step waits for all of it anyway.
__global__ __launch_bounds__(kCtrlThreads) void k_beam_step(BeamArgs a) {
  const int t = threadIdx.x, R = a.B * a.beam;
  const int step = *a.step;
  __shared__ int s_live;
  if (t == 0) s_live = 0;
  __syncthreads();
  int live = 0;
  for (int r = t; r < R; r += kCtrlThreads) {
    const int tok = a.token[r];
    if (step < a.steps_max) a.hist[static_cast<size_t>(step) * R + r] = make_int2(a.parent[r], tok);
    a.row_tok[r] = tok;
    a.row_pos[r] = min(step + 1, a.steps_max - 1);     // a row that goes on is within the positional table
    live += a.done[r] == 0;
  }
  for (int b = t; b < a.B; b += kCtrlThreads) {
    a.flags[b] |= a.step_flags[b];
    // a forward counts for a sentence that had a hypothesis to extend
    if (a.finished[b] == 0 || step == 0) a.k[b] = step + 1;
    int left = 0;
    for (int i = 0; i < a.beam; ++i) left += a.done[b * a.beam + i] == 0;
    a.finished[b] = left == 0;
  }
  if (live != 0) atomicAdd(&s_live, live);
  __syncthreads();
  if (t == 0) {
    const int seq = (*a.seq + 1) & kSeqMask;
    *a.step = step + 1;
    *a.seq = seq;
    __hip_atomic_store(a.host_rows, host_word(s_live, false, seq), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  }
}

// The hypotheses: a workgroup per sentence, a lane per hypothesis walking back
// through the steps' records, which are brought to LDS in pieces.
constexpr int kTraceRecords = 4096;

__global__ __launch_bounds__(256) void k_beam_out(BeamArgs a) {
  const int b = blockIdx.x, t = threadIdx.x, K = a.beam, R = a.B * K;
  __shared__ int2 s_hist[kTraceRecords];
  const int steps = min(*a.step, a.steps_max);
  const int piece = kTraceRecords / K;
  const int row = b * K + t;
  int at = t, len = 0;
  if (t < K) {
    len = a.lens[row];
    a.out_len[row] = len;
    a.out_scores[row] = a.scores[row];
  }
  for (int i = t; i < K * a.out_ld; i += 256) a.out_ids[static_cast<size_t>(b) * K * a.out_ld + i] = a.pad_id;
  int last = a.pad_id;
  for (int hi = steps; hi > 0; hi -= piece) {
    const int lo = max(0, hi - piece);
    __syncthreads();
    for (int i = t; i < (hi - lo) * K; i += 256) {
      const int s = i / K;
      s_hist[i] = a.hist[static_cast<size_t>(lo + s) * R + b * K + (i - s * K)];
    }
    __syncthreads();
    if (t < K && len > 0) {
      for (int s = hi - 1; s >= lo && at >= 0; --s) {
        const int2 h = s_hist[(s - lo) * K + at];
        if (s < len) a.out_ids[static_cast<size_t>(row) * a.out_ld + s] = h.y;
        if (s == len - 1) last = h.y;
        at = h.x;
      }
    }
  }
  if (t == 0) {
    a.out_k[b] = a.k[b];
    a.out_flags[b] = a.flags[b] | a.flag_converged | (len > 0 && last == a.eos_id ? a.flag_eos : 0);
  }
}

}  // namespace

hipError_t launch_beam_init(const BeamArgs& a, hipStream_t s) {
  const int n = a.B * a.beam;
  hipLaunchKernelGGL(k_beam_init, dim3((n + 255) / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_beam_step(const BeamArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_beam_step, dim3(1), dim3(kCtrlThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_beam_out(const BeamArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_beam_out, dim3(a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace pdec
