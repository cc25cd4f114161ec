// Operations on the pages of a paged cache: the table follows a set of parents
// (fork), and the pages in use move to the front of the pool (compact).
//
// Fork.  Sequence s of the new table takes the pages of its parent; with grow
// it also gets the slot of its next token, position n (the parent's length):
//   n on a page border         a free page;
//   otherwise                  the parent's last page, if every reference to it
//                              in the new table is a sequence that grows and s
//                              is the first of them; else a free page with
//                              the last page's contents copied.
// A page nothing refers to afterwards is free.  The free pages with the lowest
// ids are taken in the order of s, so the result does not depend on timing:
// atomics only count (integer sums and minima).
// A page is copied from only if it stays referenced, and copied to only if it
// is not, so the copies of one call touch disjoint pages.
#include "common.h"
#include "operators.h"

namespace pdec {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;

// Scratch: per page the number of growing sequences that end in it and the
// first of them; the list of page copies; the number of copies.
struct PagesWs {
  int* writers;
  int* first;
  int2* copies;
  int* n_copies;
};

PagesWs carve(char* ws, int pages, int n_out) {
  PagesWs w;
  w.copies = reinterpret_cast<int2*>(ws);
  w.writers = reinterpret_cast<int*>(w.copies + (pages > n_out ? pages : n_out));
  w.first = w.writers + pages;
  w.n_copies = w.first + pages;
  return w;
}

// Exclusive prefix sum of v over the workgroup; total: the sum.  s: one int
// per wave.  Every thread must call it.
__device__ __forceinline__ int block_scan(int v, int* s, int& total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) s[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    before += i < wave ? s[i] : 0;
    total += s[i];
  }
  return before + x - v;
}

__device__ __forceinline__ int pages_of(int len, int ps) { return (len + ps - 1) / ps; }

// A length within what the table's row names.
__device__ __forceinline__ int clamped(const PagesArgs& a, int n) {
  const long long most = static_cast<long long>(a.table_ld) * a.c.ps;
  return n < 0 ? 0 : n > most ? static_cast<int>(most) : n;
}

// The parent of output s (-1: none) and its length, both within their ranges.
__device__ __forceinline__ int parent_of(const PagesArgs& a, int s, int& len) {
  const int p = a.parents[s];
  len = 0;
  if (p < 0 || p >= a.n_in) return -1;
  len = clamped(a, a.lens[p]);
  return p;
}

// A plan is one workgroup's work: a page gets its number by a prefix sum over the
// pool.  What bounds it is latency, so pools and tables that fit (most do: 8192
// pages, 2048 sequences) are counted in LDS, with the loads of kBatch entries
// under way at a time; larger ones in global memory.  64 x 5 sequences over 1,746
// pages: 8.2 us in LDS (a fork 23.6 us a call, 46.2 with the counts in global
// memory; a compaction of 1,699 pages 45.3 and 59.7).  Of 13,688 pages and 2,500
// sequences, in global memory, a fork takes 79 us and a compaction 83, of 12,621 pages
// and 320 sequences 71 and 90 (small pages: the plan's time).
constexpr int kLdsPages = 8192, kLdsSeqs = 2048;
constexpr int kBatch = 4;

template <bool LDS> __device__ __forceinline__ int counted(const int* p) {   // a value that atomics have made
  return LDS ? *p : __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <bool LDS>
__global__ __launch_bounds__(kPlanThreads) void k_fork_plan(PagesArgs a, PagesWs w) {
  const int t = threadIdx.x, P = a.c.pages, ps = a.c.ps, ld = a.table_ld;
  __shared__ int s_scan[kPlanWaves];
  __shared__ int s_full;
  __shared__ int s_refs[LDS ? kLdsPages : 1], s_writers[LDS ? kLdsPages : 1], s_first[LDS ? kLdsPages : 1];
  __shared__ int2 s_seq[LDS ? kLdsSeqs : 1], s_need[LDS ? kLdsSeqs : 1];
  int* refs = LDS ? s_refs : a.refs;
  int* writers = LDS ? s_writers : w.writers;
  int* first = LDS ? s_first : w.first;
  int2* need_list = LDS ? s_need : w.copies;          // (page to copy or -1, sequence)
  auto sync = [&]() {
    if constexpr (!LDS) __threadfence();
    __syncthreads();
  };
  // no references yet; each sequence's parent (-1: none) and its length
  if constexpr (LDS) {
    for (int s = t; s < a.n_out; s += kPlanThreads) {
      int len;
      const int p = parent_of(a, s, len);
      s_seq[s] = make_int2(p, len);
    }
  }
  for (int p = t; p < P; p += kPlanThreads) {
    refs[p] = 0;
    writers[p] = 0;
    first[p] = 0x7fffffff;
  }
  if (t == 0) s_full = 0;
  sync();
  auto seq = [&](int s, int& len) -> int {
    if constexpr (LDS) {
      len = s_seq[s].y;
      return s_seq[s].x;
    }
    return parent_of(a, s, len);
  };
  // the parents' pages, counted
  const long long entries = static_cast<long long>(a.n_out) * ld;
  for (long long i0 = t; i0 < entries; i0 += kBatch * kPlanThreads) {
    int id[kBatch], s[kBatch], j[kBatch], len[kBatch], p[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const long long i = i0 + k * kPlanThreads;
      const bool in = i < entries;
      if constexpr (LDS) s[k] = in ? static_cast<int>(i) / ld : 0;
      else s[k] = in ? static_cast<int>(i / ld) : 0;
      j[k] = static_cast<int>(i - static_cast<long long>(s[k]) * ld);
      p[k] = seq(s[k], len[k]);
      const bool there = in && p[k] >= 0 && j[k] < pages_of(len[k], ps);
      id[k] = there ? a.table[static_cast<size_t>(p[k]) * ld + j[k]] : -1;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const long long i = i0 + k * kPlanThreads;
      if (i >= entries) continue;
      if (id[k] < 0 || id[k] >= P) id[k] = -1;
      a.out_table[i] = id[k];
      if (id[k] >= 0) atomicAdd(&refs[id[k]], 1);
      if (j[k] == 0) a.out_lens[s[k]] = len[k] + (p[k] >= 0 && a.grow ? 1 : 0);
      if (id[k] >= 0 && a.grow && len[k] % ps != 0 && j[k] == len[k] / ps) {
        atomicAdd(&writers[id[k]], 1);
        atomicMin(&first[id[k]], s[k]);
      }
      if (j[k] == 0 && p[k] >= 0 && a.grow && len[k] == ld * ps) atomicAdd(&s_full, 1);   // no place for a page
    }
  }
  sync();
  // sequences that need a page, in order
  int n_need = 0;
  for (int s0 = 0; a.grow && s0 < a.n_out; s0 += kPlanThreads) {
    const int s = s0 + t;
    int need = 0, from = -1;
    if (s < a.n_out) {
      int len;
      const int p = seq(s, len);
      if (p >= 0 && len < ld * ps) {
        if (len % ps == 0) {
          need = 1;
        } else {
          int id = a.table[static_cast<size_t>(p) * ld + len / ps];
          if (id < 0 || id >= P) id = -1;
          if (id < 0) need = 1;
          else if (counted<LDS>(&refs[id]) != counted<LDS>(&writers[id]) || counted<LDS>(&first[id]) != s) {
            need = 1;
            from = id;
          }
        }
      }
    }
    int total;
    const int k = n_need + block_scan(need, s_scan, total);
    if (need) need_list[k] = make_int2(from, s);
    n_need += total;
  }
  sync();
  // the lowest free pages, one for each
  int n_free = 0;
  for (int p0 = 0; n_free < n_need && p0 < P; p0 += kPlanThreads) {
    const int p = p0 + t;
    const int is = p < P && counted<LDS>(&refs[p]) == 0;
    int total;
    const int k = n_free + block_scan(is, s_scan, total);
    if (is && k < n_need) first[k] = p;              // first[] has served, and k < P
    n_free += total;
  }
  sync();
  const int missing = (n_need > n_free ? n_need - n_free : 0) + s_full;
  if (missing > 0) {
    // refused as a whole: every sequence comes out empty
    for (long long i = t; i < entries; i += kPlanThreads) a.out_table[i] = -1;
    for (int s = t; s < a.n_out; s += kPlanThreads) a.out_lens[s] = 0;
    for (int p = t; p < P; p += kPlanThreads) refs[p] = 0;
    n_need = 0;
  }
  for (int k = t; k < n_need; k += kPlanThreads) {
    const int2 c = need_list[k];
    const int id = first[k];
    int len;
    seq(c.y, len);
    a.out_table[static_cast<size_t>(c.y) * ld + len / ps] = id;
    refs[id] = 1;
    if (c.x >= 0) atomicAdd(&refs[c.x], -1);
    w.copies[k] = make_int2(c.x, id);
  }
  sync();
  int used = 0, sum = 0;
  for (int p = t; p < P; p += kPlanThreads) {
    const int r = counted<LDS>(&refs[p]);
    used += r > 0;
    if constexpr (LDS) a.refs[p] = r;
  }
  block_scan(used, s_scan, sum);
  if (t == 0) {
    a.status[0] = missing;
    a.status[1] = sum;
    *w.n_copies = n_need;
  }
}

// The copies of a plan: whole pages of every layer, 16 bytes a lane.  Bound by
// memory: 98 MB read and written in 20 us (4.9 TB/s; a copy of 1 GB reaches 5.2).
// Several words requested ahead, or rows of a page a workgroup, measured the
// same or slower (20.7 and 23.6 us).
__global__ __launch_bounds__(256) void k_copy_pages(CacheView c, PagesWs w) {
  const int n = *w.n_copies;
  const size_t kv = c.kv_page_bytes() / 16, sc = c.scale_page_bytes() / 16;
  const size_t per_layer = 2 * (kv + sc);
  const size_t total = per_layer * c.layers * n;
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < total; i += gridDim.x * 256ull) {
    const size_t m = i / (per_layer * c.layers), r = i - m * per_layer * c.layers;
    const int2 cp = w.copies[m];
    if (cp.x < 0) continue;
    const size_t l = r / per_layer;
    size_t o = r - l * per_layer;
    char* base;
    size_t words;
    if (o < kv) { base = c.k; words = kv; }
    else if (o < 2 * kv) { base = c.v; o -= kv; words = kv; }
    else if (o < 2 * kv + sc) { base = c.ks; o -= 2 * kv; words = sc; }
    else { base = c.vs; o -= 2 * kv + sc; words = sc; }
    uint4* at = reinterpret_cast<uint4*>(base);
    at[(l * c.pages + cp.y) * words + o] = at[(l * c.pages + cp.x) * words + o];
  }
}

template <bool LDS>
__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(PagesArgs a, PagesWs w) {
  const int t = threadIdx.x, P = a.c.pages, ps = a.c.ps, ld = a.table_ld;
  __shared__ int s_scan[kPlanWaves];
  __shared__ int s_used[LDS ? kLdsPages : 1], s_remap[LDS ? kLdsPages : 1];
  __shared__ int2 s_move[LDS ? kLdsPages : 1];
  int* in_use = LDS ? s_used : w.writers;
  int* remap = LDS ? s_remap : a.refs;
  int2* move = LDS ? s_move : w.copies;
  auto sync = [&]() {
    if constexpr (!LDS) __threadfence();
    __syncthreads();
  };
  for (int p = t; p < P; p += kPlanThreads) in_use[p] = 0;
  sync();
  // f(entry, page or -1) of every entry, kBatch of them under way at a time
  const long long entries = static_cast<long long>(a.n_in) * ld;
  auto each_entry = [&](auto f) {
    for (long long i0 = t; i0 < entries; i0 += kBatch * kPlanThreads) {
      int id[kBatch], n[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const long long i = min(i0 + k * kPlanThreads, entries - 1);
        id[k] = a.table[i];
        n[k] = clamped(a, a.lens[i / ld]);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const long long i = i0 + k * kPlanThreads;
        if (i >= entries) continue;
        const bool there = i % ld < pages_of(n[k], ps) && id[k] >= 0 && id[k] < P;
        f(i, there ? id[k] : -1);
      }
    }
  };
  each_entry([&](long long, int id) {
    if (id >= 0) atomicOr(&in_use[id], 1);
  });
  sync();
  int used = 0;
  {
    int mine = 0;
    for (int p = t; p < P; p += kPlanThreads) mine += counted<LDS>(&in_use[p]);
    block_scan(mine, s_scan, used);
  }
  // the i-th lowest page in use from `used` on goes to the i-th lowest free one below it
  int moves = 0, holes = 0;
  for (int p0 = 0; p0 < P; p0 += kPlanThreads) {
    const int p = p0 + t;
    const int u = p < P ? counted<LDS>(&in_use[p]) : 0;
    const int src = u && p >= used, hole = p < used && !u;
    int total;
    const int k = moves + block_scan(src, s_scan, total);
    moves += total;
    const int h = holes + block_scan(hole, s_scan, total);
    holes += total;
    if (src) move[k].x = p;
    if (hole) move[h].y = p;
    if (p < P && !src) remap[p] = u ? p : -1;
  }
  sync();
  for (int k = t; k < moves; k += kPlanThreads) {
    const int2 m = move[k];
    remap[m.x] = m.y;
    if constexpr (LDS) w.copies[k] = m;
  }
  sync();
  each_entry([&](long long i, int id) { a.out_table[i] = id < 0 ? -1 : remap[id]; });
  if constexpr (LDS)
    for (int p = t; p < P; p += kPlanThreads) a.refs[p] = remap[p];
  if (t == 0) {
    a.status[0] = moves;
    a.status[1] = used;
    *w.n_copies = moves;
  }
}

hipError_t copy_pages(const PagesArgs& a, const PagesWs& w, hipStream_t s) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_copy_pages, dim3(2048), dim3(256), 0, s, a.c, w);
  return hipGetLastError();
}

}  // namespace

size_t pages_workspace(const CacheView& c, int n_out) {
  const size_t most = c.pages > n_out ? c.pages : n_out;
  return most * 8 + static_cast<size_t>(c.pages) * 8 + 16;
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s) {
  const PagesWs w = carve(a.ws, a.c.pages, a.n_out);
  if (a.c.pages <= kLdsPages && a.n_out <= kLdsSeqs && static_cast<long long>(a.n_out) * a.table_ld < (1LL << 30))
    hipLaunchKernelGGL(k_fork_plan<true>, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  else
    hipLaunchKernelGGL(k_fork_plan<false>, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  return copy_pages(a, w, s);
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const PagesWs w = carve(a.ws, a.c.pages, a.n_in);
  if (a.c.pages <= kLdsPages) hipLaunchKernelGGL(k_compact_plan<true>, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  else hipLaunchKernelGGL(k_compact_plan<false>, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  return copy_pages(a, w, s);
}

}  // namespace pdec
