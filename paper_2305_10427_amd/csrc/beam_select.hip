// Beam search's selection over beams and vocabulary.
//
// For the live beam k of a sentence with score s, length n and logits x_v:
//   lse = log sum_v exp(x_v),  c_v = s + (x_v - lse),  key_v = c_v / (n + 1)^alpha;
// a finished beam has one candidate, itself: c = s, key = s / n^alpha.  The
// `beam` candidates of largest key survive.  Within a beam the order of the
// keys is that of the logits, so a row's best `beam` logits are found first,
// together with its log-sum-exp, in one pass over the row (k_select_rows, a
// row in parts, a wave each), and a sentence's rows are merged by key
// (k_select_merge).  Keys are compared in double: neighbouring keys of
// different rows differ by the rounding of their log-sum-exps.
//
// A logit and its word are one 64-bit number: the logit's order-preserving bits
// above the complement of the word, so that a larger number is a better
// candidate and equal logits go to the lower word, in whatever order a row is
// read.  A wave keeps the bar (the beam-th best number so far) and collects
// what is above it in LDS; the maximum of each lane's 16 bytes, which the
// running softmax needs anyway, tells whether a chunk holds anything.
#include "common.h"
#include "operators.h"

namespace pdec {

namespace {

constexpr int kRowWaves = 4;
constexpr int kBufKeys = 2 * kMaxBeam;       // a full list and one number of every lane
constexpr uint64_t kNothing = 0x007fffffffffffffull;   // -inf with every word below: what lies above is a candidate

typedef unsigned long long u64;

// Scratch of a launch: the best numbers of each part of each row (0: none), and
// the part's largest logit, sum of exp(x - largest) and whether it held a NaN or +inf.
struct PartStat {
  double sum;
  float max;
  int bad;
};
struct SelectWs {
  u64* keys;         // [rows][parts][beam]
  PartStat* stat;    // [rows][parts]
};

__device__ __forceinline__ bool row_live(const SelectArgs& a, int row) {
  return a.done[row] == 0 && isfinite(a.scores[row]);
}

// NaN and +inf are left out like -inf (and reported); -0 counts as 0.
__device__ __forceinline__ float usable(float x, int& bad) {
  const bool no = !(x < INFINITY);
  bad |= no ? 1 : 0;
  return no ? -INFINITY : x + 0.f;
}

__device__ __forceinline__ u64 key_of(float x, int word) {
  return static_cast<u64>(float_key(x)) << 32 | (0xffffffffu - static_cast<uint32_t>(word));
}
__device__ __forceinline__ float key_logit(u64 key) {
  const uint32_t u = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_word(u64 key) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key)); }

// A wave's list of its best numbers.  All lanes call every member together.
struct WaveBest {
  u64* buf;          // [kBufKeys] in LDS, this wave's
  int want;          // numbers kept
  int n;             // numbers in buf
  u64 bar;           // only numbers above it are taken
  __device__ __forceinline__ void init(u64* lds, int k) {
    buf = lds;
    want = k;
    n = 0;
    bar = kNothing;
  }
  // Keeps the `want` best of buf, best first, by counting for each number those
  // above it (all are different).
  __device__ __forceinline__ void sort(int lane) {
    wave_lds_sync();
    u64 mine[kBufKeys / kWave];
    int rank[kBufKeys / kWave];
#pragma unroll
    for (int i = 0; i < kBufKeys / kWave; ++i) {
      mine[i] = lane + kWave * i < n ? buf[lane + kWave * i] : 0;
      rank[i] = 0;
    }
    for (int j = 0; j < n; ++j) {
      const u64 o = buf[j];
#pragma unroll
      for (int i = 0; i < kBufKeys / kWave; ++i) rank[i] += o > mine[i] ? 1 : 0;
    }
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < kBufKeys / kWave; ++i)
      if (mine[i] != 0 && rank[i] < want) buf[rank[i]] = mine[i];
    n = n < want ? n : want;
    wave_lds_sync();
    if (n == want) {
      const u64 last = buf[want - 1];
      if (last > bar) bar = last;
    }
  }
  // Raises the bar by the lanes' largest numbers: where `want` lanes hold one
  // above a bound, the want-th best is above it too.  Bits 63 .. 48 are searched.
  __device__ __forceinline__ void raise(uint32_t top) {
    uint32_t lo = static_cast<uint32_t>(bar >> 32);
    if (__popcll(__ballot(top > lo)) < want) return;
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t c = t | 1u << bit;
      if (__popcll(__ballot(top >= c)) >= want) t = c;
    }
    if (t > lo) bar = (static_cast<u64>(t) << 32) - 1;   // every number of a logit at or above t is above it
  }
  __device__ __forceinline__ void offer(u64 key, bool there, int lane) {
    const u64 vote = __ballot(there && key > bar);
    if (vote == 0) return;
    if (n + __popcll(vote) > kBufKeys) {
      sort(lane);
      return offer_once(key, there, lane);
    }
    push(key, vote, lane);
  }
  __device__ __forceinline__ void offer_once(u64 key, bool there, int lane) { push(key, __ballot(there && key > bar), lane); }
  __device__ __forceinline__ void push(u64 key, u64 vote, int lane) {
    if (vote >> lane & 1) buf[n + __popcll(vote & ((1ull << lane) - 1))] = key;
    n += __popcll(vote);
  }
};

// Running maximum and sum of exp(x - max) of a lane.
struct LaneSum {
  float max;
  double sum;
};

// exp(d) for d <= 0 to about 2^-23: the product with log2 e in two parts.
__device__ __forceinline__ float exp_neg(float d) {
  constexpr float hi = 1.442695022f, lo = 1.925963033e-8f;
  return __builtin_amdgcn_exp2f(fmaf(d, hi, d * lo));
}

// N consecutive logits of a lane (words word0 ...; none below zero are there).
template <int N>
__device__ __forceinline__ void take_chunk(const float* x, int word0, bool there, WaveBest& best, LaneSum& ls, int lane) {
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < N; ++e) top = fmaxf(top, x[e]);
  const float m = fmaxf(ls.max, top);
  if (m > -INFINITY) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) sum += exp_neg(x[e] - m);
    const float f = exp_neg(ls.max - m);
    ls.sum = fma(ls.sum, static_cast<double>(f), static_cast<double>(sum));
    ls.max = m;
  }
  const uint32_t top_bits = there ? float_key(top) : 0u;
  if (__ballot(top_bits >= static_cast<uint32_t>(best.bar >> 32)) == 0) return;
  best.raise(top_bits);
#pragma unroll
  for (int e = 0; e < N; ++e) best.offer(key_of(x[e], word0 + e), there, lane);
}

// Parts of a row: vectors of 16 bytes from the row's first aligned one on.
// kVecs of them a lane and step, all requested before the first is used.
constexpr int kVecs = 4;

template <typename T>
__global__ __launch_bounds__(kRowWaves * kWave) void k_select_rows(SelectArgs a, SelectWs w, int parts, int steps) {
  constexpr int E = Vec16<T>::N;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int unit = blockIdx.x * kRowWaves + wave;
  if (unit >= a.B * a.beam * parts) return;
  const int row = unit / parts, part = unit - row * parts;
  if (!row_live(a, row)) return;
  __shared__ u64 s_buf[kRowWaves][kBufKeys];
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld;
  const int V = a.vocab;
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(x) / sizeof(T) % E);
  const int head = min(V, off == 0 ? 0 : E - off);
  const int vecs = (V - head) / E;
  const T* body = x + head;

  WaveBest best;
  best.init(s_buf[wave], a.beam);
  LaneSum ls{-INFINITY, 0.0};
  int bad = 0;
  const int v0 = part * steps * (kVecs * kWave);
  const int v1 = min(vecs, v0 + steps * (kVecs * kWave));
  if (v0 < v1) {
    uint4 cur[kVecs];
    auto load = [&](int v, uint4* q) {     // past the end: the row's last vector again
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        q[i] = *reinterpret_cast<const uint4*>(body + static_cast<size_t>(min(v + i * kWave + lane, v1 - 1)) * E);
    };
    load(v0, cur);
    for (int v = v0; v < v1; v += kVecs * kWave) {
      uint4 next[kVecs];
      load(min(v + kVecs * kWave, v1 - 1), next);
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int at = v + i * kWave + lane;
        float f[E];
        const uint32_t u[4] = {cur[i].x, cur[i].y, cur[i].z, cur[i].w};
        const bool there = at < v1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float r = sizeof(T) == 4 ? __uint_as_float(u[e & 3])
                                         : __uint_as_float(e & 1 ? u[e / 2 & 3] & 0xffff0000u : u[e / 2 & 3] << 16);
          const float y = usable(r, bad);
          f[e] = there ? y : -INFINITY;
        }
        take_chunk<E>(f, head + at * E, there, best, ls, lane);
      }
#pragma unroll
      for (int i = 0; i < kVecs; ++i) cur[i] = next[i];
    }
  }
  if (part == 0) {   // the words before the first aligned vector and behind the last
    const int tail = head + vecs * E;
    const int word = lane < head ? lane : tail + (lane - head);
    const bool there = word < V && (lane < head || lane - head < V - tail);
    const float f = there ? usable(Elt<T>::load(x, word), bad) : -INFINITY;
    take_chunk<1>(&f, word, there, best, ls, lane);
  }
  best.sort(lane);
  const float m = wave_max(ls.max);
  double s = ls.max > -INFINITY ? ls.sum * static_cast<double>(exp_neg(ls.max - m)) : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  const u64 any = __ballot(bad != 0);
  const size_t out = static_cast<size_t>(unit);
  for (int i = lane; i < a.beam; i += kWave) w.keys[out * a.beam + i] = i < best.n ? best.buf[i] : 0;
  if (lane == 0) w.stat[out] = PartStat{s, m, any != 0 ? 1 : 0};
}

constexpr int kMergeWaves = 4;
constexpr int kMergeThreads = kMergeWaves * kWave;

__global__ __launch_bounds__(kMergeThreads) void k_select_merge(SelectArgs a, SelectWs w, int parts) {
  const int b = blockIdx.x, K = a.beam;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __shared__ u64 s_buf[kMergeWaves][kBufKeys];
  __shared__ u64 s_key[kMaxBeam][kMaxBeam];      // a beam's best numbers, best first (0: none; finished: one, the score)
  __shared__ int s_n[kMaxBeam];                  // how many
  __shared__ double s_lse[kMaxBeam];             // log-sum-exp
  __shared__ double s_div[kMaxBeam];             // length^alpha
  __shared__ int s_at[kMaxBeam];
  __shared__ int s_bad;
  if (threadIdx.x == 0) s_bad = 0;
  if (threadIdx.x < K) s_at[threadIdx.x] = -1;
  __syncthreads();
  for (int k = wave; k < K; k += kMergeWaves) {  // a wave per beam
    const int row = b * K + k;
    const float score = a.scores[row];
    const bool fin = a.done[row] != 0;
    int n = 0;
    double lse = 0.0;
    if (!isfinite(score)) {
      n = 0;
    } else if (fin) {
      n = 1;
    } else {
      const size_t p0 = static_cast<size_t>(row) * parts;
      float m = -INFINITY;
      int bad = 0;
      for (int p = lane; p < parts; p += kWave) {
        m = fmaxf(m, w.stat[p0 + p].max);
        bad |= w.stat[p0 + p].bad;
      }
      m = wave_max(m);
      double s = 0.0;
      for (int p = lane; p < parts; p += kWave) {
        const PartStat st = w.stat[p0 + p];
        if (st.max > -INFINITY) s += st.sum * exp(static_cast<double>(st.max) - static_cast<double>(m));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
      lse = static_cast<double>(m) + log(s);
      if (__ballot(bad != 0) != 0 && lane == 0) s_bad = 1;
      WaveBest best;
      best.init(s_buf[wave], K);
      for (int i0 = 0; i0 < parts * K; i0 += kWave) {
        const int i = i0 + lane;
        const u64 key = i < parts * K ? w.keys[p0 * K + i] : 0;
        if (__ballot(key > best.bar) == 0) continue;
        best.raise(static_cast<uint32_t>(key >> 32));
        best.offer(key, key != 0, lane);
      }
      best.sort(lane);
      n = best.n;
      for (int i = lane; i < n; i += kWave) s_key[k][i] = best.buf[i];
    }
    if (lane == 0) {
      const int len = a.lens[row] + (fin ? 0 : 1);
      s_n[k] = n;
      s_lse[k] = lse;
      s_div[k] = pow(static_cast<double>(len > 1 ? len : 1), static_cast<double>(a.alpha));
    }
  }
  __syncthreads();
  auto cum_of = [&](int k, int r) -> double {
    const int row = b * K + k;
    const double score = a.scores[row];
    return a.done[row] != 0 ? score : score + (static_cast<double>(key_logit(s_key[k][r])) - s_lse[k]);
  };
  // every candidate counts those before it: (key, beam, rank in the beam).  A
  // beam's candidates are in order, so those of another beam are found by halving.
  for (int c = threadIdx.x; c < K * K; c += kMergeThreads) {
    const int r = c / K, k = c - r * K;
    if (r >= s_n[k]) continue;
    const double key = cum_of(k, r) / s_div[k];
    int rank = r;
    for (int o = 0; o < K && rank < K; ++o) {
      if (o == k) continue;
      int lo = 0, hi = s_n[o];           // the first of beam o that comes after the candidate
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const double other = cum_of(o, mid) / s_div[o];
        if (other > key || (other == key && o < k)) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank < K) s_at[rank] = c;
  }
  __syncthreads();
  float o_score = -INFINITY;
  int o_par = -1, o_tok = a.pad_id, o_len = 0, o_done = 1;
  const int t = threadIdx.x;
  if (t < K && s_at[t] >= 0) {
    const int c = s_at[t], r = c / K, k = c - r * K, row = b * K + k;
    const bool fin = a.done[row] != 0;
    o_score = static_cast<float>(cum_of(k, r));
    o_par = k;
    o_tok = fin ? a.pad_id : key_word(s_key[k][r]);
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

// Parts of a row and the steps of a part: kWantWaves waves in all where the
// rows are long enough, each of at least one step (4 KB).
constexpr int kWantWaves = 4096;
struct Split {
  int parts, steps;
};
Split split_rows(int dtype, int rows, int vocab) {
  const int per_step = kVecs * kWave * (dtype == DT_BF16 ? 8 : 4);
  const int all = (vocab + per_step - 1) / per_step;
  int parts = (kWantWaves + rows - 1) / rows;
  if (parts > all) parts = all;
  Split s;
  s.steps = (all + parts - 1) / parts;
  s.parts = (all + s.steps - 1) / s.steps;
  return s;
}

}  // namespace

size_t select_workspace(int dtype, int B, int beam, int vocab) {
  const int rows = B * beam;
  const size_t units = static_cast<size_t>(rows) * split_rows(dtype, rows, vocab).parts;
  return units * (static_cast<size_t>(beam) * sizeof(u64) + sizeof(PartStat));
}

hipError_t launch_beam_select(const SelectArgs& a, hipStream_t s) {
  const int rows = a.B * a.beam;
  const Split sp = split_rows(a.dtype, rows, a.vocab);
  const size_t units = static_cast<size_t>(rows) * sp.parts;
  SelectWs w;
  w.stat = reinterpret_cast<PartStat*>(a.ws);
  w.keys = reinterpret_cast<u64*>(w.stat + units);
  const dim3 grid(static_cast<unsigned>((units + kRowWaves - 1) / kRowWaves)), block(kRowWaves * kWave);
  if (a.dtype == DT_BF16) hipLaunchKernelGGL(k_select_rows<bf16_t>, grid, block, 0, s, a, w, sp.parts, sp.steps);
  else hipLaunchKernelGGL(k_select_rows<float>, grid, block, 0, s, a, w, sp.parts, sp.steps);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_select_merge, dim3(a.B), dim3(kMergeThreads), 0, s, a, w, sp.parts);
  return hipGetLastError();
}

}  // namespace pdec
