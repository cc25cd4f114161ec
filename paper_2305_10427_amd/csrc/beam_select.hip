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
// what is above it in LDS; the maximum of each lane's step, which the running
// softmax needs anyway, tells whether a step holds anything.
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
  // The least logit that can be above the bar.
  __device__ __forceinline__ float floor() const { return key_logit(bar); }
  // A number of every lane (0: none).
  __device__ __forceinline__ void offer(u64 key, int lane) {
    u64 vote = __ballot(key > bar);
    if (n + __popcll(vote) > kBufKeys) {
      sort(lane);
      vote = __ballot(key > bar);
    }
    if (vote >> lane & 1) buf[n + __popcll(vote & ((1ull << lane) - 1))] = key;
    n += __popcll(vote);
  }
};

// Sum of the wave's values, in the order of wave_sum.
template <int CTRL> __device__ __forceinline__ double dpp_d(double v) {
  const u64 u = static_cast<u64>(__double_as_longlong(v));
  const uint32_t lo = dpp_u<CTRL>(static_cast<uint32_t>(u)), hi = dpp_u<CTRL>(static_cast<uint32_t>(u >> 32));
  return __longlong_as_double(static_cast<long long>(static_cast<u64>(hi) << 32 | lo));
}
__device__ __forceinline__ double wave_sum_d(double v) {
  v += dpp_d<kDppXor1>(v);
  v += dpp_d<kDppXor2>(v);
  v += dpp_d<kDppHalfMirror>(v);
  v += dpp_d<kDppMirror>(v);
  auto at = [&](int l) {
    const u64 u = static_cast<u64>(__double_as_longlong(v));
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(u), l), hi = __builtin_amdgcn_readlane(static_cast<int>(u >> 32), l);
    return __longlong_as_double(static_cast<long long>(static_cast<u64>(hi) << 32 | lo));
  };
  return (at(0) + at(16)) + (at(32) + at(48));
}

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

// A step's exponentials are summed in float, in kSums sums: at most 9 roundings.
constexpr int kSums = 4;

// One step of a lane: NV vectors of E logits of the row, whose words start at
// word0 and lie `apart` apart (those that do not exist: -inf).  A NaN or +inf makes the sum NaN,
// which is seen afterwards: then those logits are left out and the step is
// repeated, so that the usual step pays nothing for them.
template <typename T, int NV, int E>
__device__ __forceinline__ void take_step(const T* row, float* x, int word0, int apart, WaveBest& best, LaneSum& ls, int& bad, int lane) {
  float top, sum, m;
  auto reduce = [&]() {
    top = x[0];
#pragma unroll
    for (int i = 1; i < NV * E; ++i) top = fmaxf(top, x[i]);
    m = fmaxf(ls.max, top);
    float part[kSums] = {};
#pragma unroll
    for (int i = 0; i < NV * E; ++i) part[i % kSums] += exp_neg(x[i] - m);
    sum = (part[0] + part[1]) + (part[2] + part[3]);
  };
  reduce();
  if (!(sum < INFINITY)) {             // something is not finite, or nothing is there yet (-inf - -inf)
#pragma unroll
    for (int i = 0; i < NV * E; ++i) x[i] = usable(x[i], bad);
    reduce();
  }
  if (m > -INFINITY) {
    ls.sum = fma(ls.sum, static_cast<double>(exp_neg(ls.max - m)), static_cast<double>(sum));
    ls.max = m;
  }
  const uint32_t top_bits = float_key(top + 0.f);
  if (__ballot(top_bits > static_cast<uint32_t>(best.bar >> 32)) == 0 &&
      __ballot(top_bits == static_cast<uint32_t>(best.bar >> 32)) == 0)
    return;
  best.raise(top_bits);
  // which of the lane's logits are not below the bar; those few are read again
  // rather than picked out of the registers, which would take all of them
  // through the list's code one by one
  const float floor = fmaxf(best.floor(), -3.4028235e38f);
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < NV * E; ++i) mask |= x[i] >= floor ? 1u << i : 0u;
  while (__ballot(mask != 0) != 0) {
    u64 key = 0;
    if (mask != 0) {
      const int i = __ffs(static_cast<int>(mask)) - 1, word = word0 + i / E * apart + i % E;
      key = key_of(Elt<T>::load(row, word) + 0.f, word);
      mask &= mask - 1;
    }
    best.offer(key, lane);
  }
}

// Parts of a row: vectors of 16 bytes from the row's first aligned one on.
// kVecs of them a lane and step, all requested before the first is used.
constexpr int kVecs = 4;

// Part `unit % parts` of row `unit / parts`, by one wave; buf: its list in LDS.
template <typename T>
__device__ __forceinline__ void row_part(const SelectArgs& a, const SelectWs& w, int parts, int steps, int unit, u64* buf,
                                         int lane) {
  constexpr int E = Vec16<T>::N;
  const int row = unit / parts, part = unit - row * parts;
  if (!row_live(a, row)) return;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld;
  const int V = a.vocab;
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(x) / sizeof(T) % E);
  const int head = min(V, off == 0 ? 0 : E - off);
  const int vecs = (V - head) / E;
  const T* body = x + head;

  WaveBest best;
  best.init(buf, a.beam);
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
      float f[kVecs * E];
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const uint32_t u[4] = {cur[i].x, cur[i].y, cur[i].z, cur[i].w};
#pragma unroll
        for (int e = 0; e < E; ++e)
          f[i * E + e] = sizeof(T) == 4 ? __uint_as_float(u[e & 3])
                                        : __uint_as_float(e & 1 ? u[e / 2 & 3] & 0xffff0000u : u[e / 2 & 3] << 16);
      }
      if (v + kVecs * kWave > v1) {
#pragma unroll
        for (int i = 0; i < kVecs * E; ++i) f[i] = v + i / E * kWave + lane < v1 ? f[i] : -INFINITY;
      }
      take_step<T, kVecs, E>(x, f, head + (v + lane) * E, kWave * E, best, ls, bad, lane);
#pragma unroll
      for (int i = 0; i < kVecs; ++i) cur[i] = next[i];
    }
  }
  if (part == 0 && vecs * E < V) {   // the words before the first aligned vector and behind the last
    const int tail = head + vecs * E;
    const int word = lane < head ? lane : tail + (lane - head);
    const bool there = lane < head || lane - head < V - tail;
    float f = there ? Elt<T>::load(x, word) : -INFINITY;
    take_step<T, 1, 1>(x, &f, word, 0, best, ls, bad, lane);
  }
  best.sort(lane);
  const float m = wave_max(ls.max);
  const double s = wave_sum_d(ls.max > -INFINITY ? ls.sum * static_cast<double>(exp_neg(ls.max - m)) : 0.0);
  const u64 any = __ballot(bad != 0);
  const size_t out = static_cast<size_t>(unit);
  for (int i = lane; i < a.beam; i += kWave) w.keys[out * a.beam + i] = i < best.n ? best.buf[i] : 0;
  if (lane == 0) w.stat[out] = PartStat{s, m, any != 0 ? 1 : 0};
}

// The rows, in one pass over the logits: bound by memory and by the launch's start
// and end (a wave sorts its list).  64 x 5 rows of 58,101 float32 words, four fifths
// of them live (59.5 MB): 17.5 us, 3.4 TB/s; 128 rows of 250,027 bfloat16 words (58
// MB): 20.7 us, 2.8 TB/s; a copy of 1 GB reaches 5.2.
template <typename T>
__global__ __launch_bounds__(kRowWaves * kWave) void k_select_rows(SelectArgs a, SelectWs w, int parts, int steps) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int unit = blockIdx.x * kRowWaves + wave;
  __shared__ u64 s_buf[kRowWaves][kBufKeys];
  if (unit < a.B * a.beam * parts) row_part<T>(a, w, parts, steps, unit, s_buf[wave], lane);
}

// Order-preserving bits of a double (no NaN; -0 counts as 0).
__device__ __forceinline__ u64 double_key(double d) {
  const u64 u = static_cast<u64>(__double_as_longlong(d + 0.0));
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// Up to KM beams.
template <int KM> struct MergeLds {
  u64 key[KM][KM];                  // a beam's best numbers, best first
  u64 by[KM][KM];                   // double_key of what they are ranked by
  double lse[KM];
  float score[KM];
  int n[KM];                  // a beam's candidates
  int len[KM];                // their length
  int fin[KM];
  int at_beam[KM], at_rank[KM];
  int bad;
};

// The survivors of sentence b, from its rows' part lists.  A wave per beam merges
// the parts; then the first wave merges the beams, a lane each with its best
// candidate that is left, the largest key and of those the lowest lane first, from
// keys that the waves have made for all candidates (of 16 beams: 14.1 us a call,
// 16.3 with the keys made as they come up).  A chain of latencies: 6 us.
//
// The parts' numbers are read 64 at a time, kBatch of those before any is used: as
// they lie where they all fit, else (BY_RANK) rank by rank, until a rank has nothing
// above the bar, nor then have later ones.  5 rows of 250,027 words 13.4 us a call by
// rank, 15.0 in order; 16 rows 21.9 and 35.6.
//
// Up to kFewBeams beams take a workgroup of as many waves and lists of that length:
// 64 x 5 rows of 58,101 words 23.2 us a call against 23.9 in workgroups for 64
// beams, one sentence of them 10.8 against 11.3.
constexpr int kFewBeams = 8, kMergeBatch = 6;

template <int KM, int kBatch, bool BY_RANK>
__device__ __forceinline__ void merge_sentence(const SelectArgs& a, const SelectWs& w, int parts, int b, MergeLds<KM>& sm,
                                               u64* buf, int lane, int wave, int waves) {
  const int K = a.beam;
  if (threadIdx.x == 0) sm.bad = 0;
  __syncthreads();
  for (int k = wave; k < K; k += waves) {
    const int row = b * K + k;
    const float score = a.scores[row];
    const bool fin = a.done[row] != 0;
    const int len = a.lens[row] + (fin ? 0 : 1);
    const size_t p0 = static_cast<size_t>(row) * parts;
    u64 key[kBatch];
    const int groups = (parts + kWave - 1) / kWave;
    auto load = [&](int q0) {         // by rank: reads q0 .. of (rank, 64 parts)
      int r = BY_RANK ? q0 / groups : 0, g = BY_RANK ? q0 - r * groups : 0;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int at = BY_RANK ? (g * kWave + lane) * K + r : i * kWave + lane;
        const bool in = BY_RANK ? g * kWave + lane < parts && r < K : at < parts * K;
        const u64 x = w.keys[p0 * K + (in ? at : 0)];
        key[i] = in ? x : 0;
        if (BY_RANK && ++g == groups) g = 0, ++r;
      }
    };
    load(0);
    PartStat mine = w.stat[p0 + min(lane, parts - 1)];
    double div = 1.0;                 // length^alpha, while the loads are under way
    if (a.alpha == 1.f) div = static_cast<double>(max(len, 1));
    else if (a.alpha != 0.f) div = pow(static_cast<double>(max(len, 1)), static_cast<double>(a.alpha));
    int n = 0;
    double lse = 0.0;
    if (!isfinite(score)) {
      n = 0;
    } else if (fin) {
      n = 1;
      if (lane == 0) sm.by[k][0] = double_key(static_cast<double>(score) / div);
    } else {
      if (lane >= parts) mine = PartStat{0.0, -INFINITY, 0};
      for (int p = lane + kWave; p < parts; p += kWave) {
        const PartStat st = w.stat[p0 + p];
        const float m = fmaxf(mine.max, st.max);
        if (m > -INFINITY)
          mine.sum = mine.sum * static_cast<double>(exp_neg(mine.max - m)) + st.sum * static_cast<double>(exp_neg(st.max - m));
        mine.max = m;
        mine.bad |= st.bad;
      }
      const float m = wave_max(mine.max);
      const double s = wave_sum_d(mine.max > -INFINITY ? mine.sum * static_cast<double>(exp_neg(mine.max - m)) : 0.0);
      lse = static_cast<double>(m) + log(s);
      if (__ballot(mine.bad != 0) != 0 && lane == 0) sm.bad = 1;
      WaveBest best;
      best.init(buf, K);
      int idle = 0;                   // reads in turn that held nothing
      for (int q0 = 0;;) {
        u64 top = key[0];
#pragma unroll
        for (int i = 1; i < kBatch; ++i) top = key[i] > top ? key[i] : top;
        best.raise(static_cast<uint32_t>(top >> 32));
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const bool any = __ballot(key[i] > best.bar) != 0;
          if (any) best.offer(key[i], lane);
          idle = any ? 0 : idle + 1;
        }
        q0 += kBatch;
        if (!BY_RANK || q0 >= K * groups || idle >= groups) break;
        load(q0);
      }
      best.sort(lane);
      n = best.n;
      for (int i = lane; i < n; i += kWave) {
        const u64 x = best.buf[i];
        sm.key[k][i] = x;
        sm.by[k][i] = double_key((static_cast<double>(score) + (static_cast<double>(key_logit(x)) - lse)) / div);
      }
    }
    if (lane == 0) {
      sm.n[k] = n;
      sm.lse[k] = lse;
      sm.score[k] = score;
      sm.len[k] = len;
      sm.fin[k] = fin ? 1 : 0;
    }
  }
  __syncthreads();
  auto cum_of = [&](int k, int r) -> double {
    const double score = sm.score[k];
    return sm.fin[k] ? score : score + (static_cast<double>(key_logit(sm.key[k][r])) - sm.lse[k]);
  };
  if (wave == 0) {
    const int k = lane < K ? lane : 0;
    int r = 0;
    u64 head = lane < K && sm.n[k] > 0 ? sm.by[k][0] : 0;
    for (int j = 0; j < K; ++j) {
      const uint32_t hi = static_cast<uint32_t>(head >> 32), hi_max = wave_max_u32(hi);
      u64 vote = __ballot(hi == hi_max);
      if (__popcll(vote) > 1) {
        const uint32_t lo = hi == hi_max ? static_cast<uint32_t>(head) : 0u, lo_max = wave_max_u32(lo);
        vote = __ballot(hi == hi_max && lo == lo_max);
      }
      const int win = __ffsll(static_cast<long long>(vote)) - 1;
      if (lane == win) {
        sm.at_beam[j] = head == 0 ? -1 : lane;
        sm.at_rank[j] = r;
        ++r;
        head = head != 0 && r < sm.n[k] ? sm.by[k][r] : 0;
      }
    }
  }
  __syncthreads();   // the outputs may be the inputs' own arrays: everything has been read
  const int t = threadIdx.x;
  if (t < K) {
    const int k = sm.at_beam[t], r = sm.at_rank[t], o = b * K + t;
    const bool there = k >= 0;
    const bool fin = there && sm.fin[k] != 0;
    const int tok = !there || fin ? a.pad_id : key_word(sm.key[k][r]);
    const int len = there ? sm.len[k] : 0;
    const int done = !there || fin || tok == a.eos_id || (a.max_len != nullptr && len >= a.max_len[b]) ? 1 : 0;
    // a sum of lowest values stays finite, so that a hypothesis never turns into none
    a.out_scores[o] = there ? fmaxf(static_cast<float>(cum_of(k, r)), -3.4028235e38f) : -INFINITY;
    a.out_parent[o] = k;
    a.out_token[o] = tok;
    a.out_len[o] = len;
    a.out_done[o] = done;
    a.out_src[o] = done ? -1 : b * K + k;
  }
  if (t == 0) a.out_flags[b] = sm.bad ? 8 : 0;
}

template <int KM, int MW, bool BY_RANK>
__global__ __launch_bounds__(MW * kWave) void k_select_merge(SelectArgs a, SelectWs w, int parts) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __shared__ u64 s_buf[MW][kBufKeys];
  __shared__ MergeLds<KM> sm;
  merge_sentence<KM, kMergeBatch, BY_RANK>(a, w, parts, blockIdx.x, sm, s_buf[wave], lane, wave, MW);
}

// Both stages of a sentence of at most kSmallWaves parts of one step, a wave each:
// one launch.  Against two (us a call): 4 rows of 1,000 words 7.6 / 8.7, 64 x 4 rows
// 8.2 / 9.7, 1,024 x 4 rows 11.5 / 16.3, 64 x 5 rows of 2,999 words 11.0 / 11.2; with
// more than a step a wave the two are faster: 1,024 x 5 rows of 10,007 words 63.9 /
// 49.0.
constexpr int kSmallWaves = 16;

template <typename T>
__global__ __launch_bounds__(kSmallWaves * kWave) void k_select_small(SelectArgs a, SelectWs w, int parts, int steps) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  __shared__ u64 s_buf[kSmallWaves][kBufKeys];
  __shared__ MergeLds<kSmallWaves> sm;
  row_part<T>(a, w, parts, steps, blockIdx.x * a.beam * parts + wave, s_buf[wave], lane);
  __threadfence_block();
  __syncthreads();
  merge_sentence<kSmallWaves, kSmallWaves * kSmallWaves / kWave, false>(a, w, parts, blockIdx.x, sm, s_buf[wave], lane, wave, a.beam * parts);
}

// Parts of a row and the steps of a part: kWantWaves waves in all where the
// rows are long enough, each of at least one step (4 KB).  Half as many are slower
// for 320 rows of 58,101 words, twice as many no faster.
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

template <int KM, int MW, bool BY_RANK>
hipError_t launch_merge(const SelectArgs& a, const SelectWs& w, int parts, hipStream_t s) {
  hipLaunchKernelGGL((k_select_merge<KM, MW, BY_RANK>), dim3(a.B), dim3(MW * kWave), 0, s, a, w, parts);
  return hipGetLastError();
}

}  // namespace

size_t select_workspace(int dtype, int B, int beam, int vocab) {
  const int rows = B * beam;
  const size_t units = static_cast<size_t>(rows) * split_rows(dtype, rows, vocab).parts;
  return units * (static_cast<size_t>(beam) * sizeof(u64) + sizeof(PartStat));
}

// parts <= (kWantWaves + rows - 1) / rows, so rows * parts < kWantWaves + rows.
size_t select_workspace_most(int rows, int beam) {
  return (static_cast<size_t>(rows) + kWantWaves) * (static_cast<size_t>(beam) * sizeof(u64) + sizeof(PartStat));
}

hipError_t launch_beam_select(const SelectArgs& a, hipStream_t s) {
  const int rows = a.B * a.beam;
  const Split sp = split_rows(a.dtype, rows, a.vocab);
  const size_t units = static_cast<size_t>(rows) * sp.parts;
  SelectWs w;
  w.stat = reinterpret_cast<PartStat*>(a.ws);
  w.keys = reinterpret_cast<u64*>(w.stat + units);
  if (a.beam * sp.parts <= kSmallWaves && sp.steps == 1) {
    const dim3 grid(a.B), block(a.beam * sp.parts * kWave);
    if (a.dtype == DT_BF16) hipLaunchKernelGGL(k_select_small<bf16_t>, grid, block, 0, s, a, w, sp.parts, sp.steps);
    else hipLaunchKernelGGL(k_select_small<float>, grid, block, 0, s, a, w, sp.parts, sp.steps);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>((units + kRowWaves - 1) / kRowWaves)), block(kRowWaves * kWave);
  if (a.dtype == DT_BF16) hipLaunchKernelGGL(k_select_rows<bf16_t>, grid, block, 0, s, a, w, sp.parts, sp.steps);
  else hipLaunchKernelGGL(k_select_rows<float>, grid, block, 0, s, a, w, sp.parts, sp.steps);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool by_rank = a.beam * sp.parts > kMergeBatch * kWave;
  if (a.beam <= kFewBeams) return by_rank ? launch_merge<kFewBeams, kFewBeams, true>(a, w, sp.parts, s) : launch_merge<kFewBeams, kFewBeams, false>(a, w, sp.parts, s);
  return by_rank ? launch_merge<kMaxBeam, 16, true>(a, w, sp.parts, s) : launch_merge<kMaxBeam, 16, false>(a, w, sp.parts, s);
}

}  // namespace pdec
