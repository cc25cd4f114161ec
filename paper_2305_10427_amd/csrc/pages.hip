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

// The parent of output s (-1: none) and its length, both within their ranges.
__device__ __forceinline__ int parent_of(const PagesArgs& a, int s, int& len) {
  const int p = a.parents[s];
  len = 0;
  if (p < 0 || p >= a.n_in) return -1;
  const long long most = static_cast<long long>(a.table_ld) * a.c.ps;
  const int n = a.lens[p];
  len = n < 0 ? 0 : n > most ? static_cast<int>(most) : n;
  return p;
}

__global__ __launch_bounds__(kPlanThreads) void k_fork_plan(PagesArgs a, PagesWs w) {
  const int t = threadIdx.x, P = a.c.pages, ps = a.c.ps, ld = a.table_ld;
  __shared__ int s_scan[kPlanWaves];
  __shared__ int s_full;
  // no references yet
  for (int p = t; p < P; p += kPlanThreads) {
    a.refs[p] = 0;
    w.writers[p] = 0;
    w.first[p] = 0x7fffffff;
  }
  if (t == 0) s_full = 0;
  __threadfence();
  __syncthreads();
  // the parents' pages, counted
  for (long long i = t; i < static_cast<long long>(a.n_out) * ld; i += kPlanThreads) {
    const int s = static_cast<int>(i / ld), j = static_cast<int>(i - static_cast<long long>(s) * ld);
    int len;
    const int p = parent_of(a, s, len);
    int id = -1;
    if (p >= 0 && j < pages_of(len, ps)) id = a.table[static_cast<size_t>(p) * ld + j];
    if (id < 0 || id >= P) id = -1;
    if (id >= 0) atomicAdd(&a.refs[id], 1);
    a.out_table[i] = id;
    if (j == 0) a.out_lens[s] = len + (p >= 0 && a.grow ? 1 : 0);
    if (id >= 0 && a.grow && len % ps != 0 && j == len / ps) {
      atomicAdd(&w.writers[id], 1);
      atomicMin(&w.first[id], s);
    }
    if (j == 0 && p >= 0 && a.grow && len == ld * ps) atomicAdd(&s_full, 1);   // the table row has no place for a page
  }
  __threadfence();
  __syncthreads();
  // sequences that need a page, in order
  int n_need = 0;
  for (int s0 = 0; a.grow && s0 < a.n_out; s0 += kPlanThreads) {
    const int s = s0 + t;
    int need = 0, from = -1, j = 0;
    if (s < a.n_out) {
      int len;
      const int p = parent_of(a, s, len);
      if (p >= 0 && len < ld * ps) {
        j = len / ps;
        if (len % ps == 0) {
          need = 1;
        } else {
          const int id = a.out_table[static_cast<size_t>(s) * ld + j];
          if (id < 0) need = 1;
          else if (__hip_atomic_load(&a.refs[id], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) !=
                       __hip_atomic_load(&w.writers[id], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ||
                   __hip_atomic_load(&w.first[id], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != s) {
            need = 1;
            from = id;
          }
        }
      }
    }
    int total;
    const int k = n_need + block_scan(need, s_scan, total);
    if (need) w.copies[k] = make_int2(from, s);      // the target follows below
    n_need += total;
  }
  __threadfence();
  __syncthreads();
  // the lowest free pages, one for each
  int n_free = 0;
  for (int p0 = 0; n_free < n_need && p0 < P; p0 += kPlanThreads) {
    const int p = p0 + t;
    const int is = p < P && __hip_atomic_load(&a.refs[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0;
    int total;
    const int k = n_free + block_scan(is, s_scan, total);
    if (is && k < n_need) w.first[k] = p;            // first[] has served; n_need <= P is checked below
    n_free += total;
  }
  __threadfence();
  __syncthreads();
  const int missing = (n_need > n_free ? n_need - n_free : 0) + s_full;
  if (missing > 0) {
    // refused as a whole: every sequence comes out empty
    for (long long i = t; i < static_cast<long long>(a.n_out) * ld; i += kPlanThreads) a.out_table[i] = -1;
    for (int s = t; s < a.n_out; s += kPlanThreads) a.out_lens[s] = 0;
    for (int p = t; p < P; p += kPlanThreads) a.refs[p] = 0;
    n_need = 0;
  }
  for (int k = t; k < n_need; k += kPlanThreads) {
    const int2 c = w.copies[k];
    const int id = w.first[k];
    int len;
    parent_of(a, c.y, len);
    a.out_table[static_cast<size_t>(c.y) * ld + len / ps] = id;
    a.refs[id] = 1;
    if (c.x >= 0) atomicAdd(&a.refs[c.x], -1);
    w.copies[k] = make_int2(c.x, id);
  }
  __threadfence();
  __syncthreads();
  int used = 0, sum = 0;
  for (int p = t; p < P; p += kPlanThreads)
    used += __hip_atomic_load(&a.refs[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 0;
  block_scan(used, s_scan, sum);
  if (t == 0) {
    a.status[0] = missing;
    a.status[1] = sum;
    *w.n_copies = n_need;
  }
}

// The copies of a plan: whole pages of every layer, 16 bytes a lane.
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

__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(PagesArgs a, PagesWs w) {
  const int t = threadIdx.x, P = a.c.pages, ps = a.c.ps, ld = a.table_ld;
  __shared__ int s_scan[kPlanWaves];
  for (int p = t; p < P; p += kPlanThreads) w.writers[p] = 0;
  __threadfence();
  __syncthreads();
  auto entry = [&](long long i) -> int {
    const int s = static_cast<int>(i / ld), j = static_cast<int>(i - static_cast<long long>(s) * ld);
    const int n = a.lens[s];
    if (n <= 0 || j >= pages_of(n, ps)) return -1;
    const int id = a.table[i];
    return id < 0 || id >= P ? -1 : id;
  };
  const long long entries = static_cast<long long>(a.n_in) * ld;
  for (long long i = t; i < entries; i += kPlanThreads) {
    const int id = entry(i);
    if (id >= 0) atomicOr(&w.writers[id], 1);
  }
  __threadfence();
  __syncthreads();
  auto in_use = [&](int p) {
    return p < P ? __hip_atomic_load(&w.writers[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  };
  int used = 0;
  {
    int mine = 0;
    for (int p = t; p < P; p += kPlanThreads) mine += in_use(p);
    block_scan(mine, s_scan, used);
  }
  // the i-th lowest page in use from `used` on goes to the i-th lowest free one below it
  int moves = 0, holes = 0;
  for (int p0 = 0; p0 < P; p0 += kPlanThreads) {
    const int p = p0 + t;
    const int u = in_use(p);
    const int src = u && p >= used, hole = p < used && !u;
    int total;
    const int k = moves + block_scan(src, s_scan, total);
    moves += total;
    const int h = holes + block_scan(hole, s_scan, total);
    holes += total;
    if (src) w.copies[k].x = p;
    if (hole) w.copies[h].y = p;
    if (p < P && !src) a.refs[p] = u ? p : -1;
  }
  __threadfence();
  __syncthreads();
  for (int k = t; k < moves; k += kPlanThreads) a.refs[w.copies[k].x] = w.copies[k].y;
  __threadfence();
  __syncthreads();
  for (long long i = t; i < entries; i += kPlanThreads) {
    const int id = entry(i);
    a.out_table[i] = id < 0 ? -1 : a.refs[id];
  }
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
  hipLaunchKernelGGL(k_fork_plan, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  return copy_pages(a, w, s);
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  const PagesWs w = carve(a.ws, a.c.pages, a.n_in);
  hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(kPlanThreads), 0, s, a, w);
  return copy_pages(a, w, s);
}

}  // namespace pdec
