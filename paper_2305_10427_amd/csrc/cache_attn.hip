// Attention of single tokens over a paged cache, the append of a token, and
// the reading back of a cache's values.
//
//   o[s,h] = sum_j p_j v_j,  p = softmax_j(scale q[s,h] . k_j),  j < len[s]
// with k_j, v_j the key and value of head h / (heads / kv_heads) in slot
// j mod page_size of page table[s][j / page_size].  Keys of pages that do not
// exist (an id outside the pool) are left out; a row without keys is zero.
#include "common.h"
#include "operators.h"

namespace pdec {

namespace {

__device__ __forceinline__ int nibble_shift(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// Number of keys of sequence s: within max_len and the table's row.
__device__ __forceinline__ int keys_of(const int* lens, int s, int max_len, int table_ld, int ps) {
  const long long most = static_cast<long long>(table_ld) * ps;
  int n = lens[s];
  n = n < max_len ? n : max_len;
  return n < 0 ? 0 : n > most ? static_cast<int>(most) : n;
}

__device__ __forceinline__ int page_at(const int* table, int table_ld, int s, int j, int pages) {
  const int id = table[static_cast<size_t>(s) * table_ld + j];
  return id >= 0 && id < pages ? id : -1;
}

__device__ __forceinline__ float load_any(const void* p, int bf16, size_t i) {
  return bf16 ? Elt<bf16_t>::load(static_cast<const bf16_t*>(p), i) : Elt<float>::load(static_cast<const float*>(p), i);
}

// Index (in page-head blocks) of head h of page id of a layer.
__device__ __forceinline__ size_t head_block(const CacheView& c, int layer, int id, int h) {
  return (static_cast<size_t>(layer) * c.pages + id) * c.kv_heads + h;
}

// Value of dimension d of slot t: K (is_v 0) or V (1) of head block hb.
__device__ __forceinline__ float cache_value(const CacheView& c, size_t hb, int t, int d, int is_v) {
  const char* base = is_v ? c.v : c.k;
  const size_t i = (hb * c.ps * c.dh) + (is_v ? static_cast<size_t>(d) * c.ps + t : static_cast<size_t>(t) * c.dh + d);
  if (c.type == CT_F32) return reinterpret_cast<const float*>(base)[i];
  if (c.type == CT_BF16) return bf16_to_f32(reinterpret_cast<const bf16_t*>(base)[i]);
  const uint32_t w = reinterpret_cast<const uint32_t*>(base)[i >> 3];
  const uint32_t par = reinterpret_cast<const uint32_t*>(is_v ? c.vs : c.ks)[(hb * c.ps + t) * c.groups + d / 32];
  const float code = static_cast<float>((w >> nibble_shift(static_cast<int>(i & 7))) & 15u);
  return code * __uint_as_float(par << 16) + __uint_as_float(par & 0xffff0000u);
}

// The largest bfloat16 up to x (x itself if it is not finite).
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t u = __float_as_uint(x), low = u & 0xffffu;
  return __uint_as_float(u - low + (low != 0 && x < 0.f ? 0x10000u : 0u));
}

// Step and least value of a group with the extremes lo, hi: the least value is
// rounded down and the step up to bfloat16, so that the fifteen steps reach hi.
// The test of the step is an exact product, on halves so that nothing
// overflows.  A group with a value that is not finite becomes NaN as a whole.
__device__ __forceinline__ void group_params(float lo, float hi, bool finite, float& step, float& least) {
  least = bf16_down(lo);
  const float half = hi * 0.5f - least * 0.5f;
  step = bf16_down(half * (2.f / 15.f));
  if (step * 7.5f < half) step = __uint_as_float(__float_as_uint(step) + 0x10000u);
  if (!finite) step = 0.f, least = NAN;
}
__device__ __forceinline__ uint32_t group_code(float x, float step, float least) {
  if (!(step > 0.f)) return 0u;
  const float c = rintf((x - least) / step);
  return static_cast<uint32_t>(fminf(fmaxf(c, 0.f), 15.f));
}

// One thread per (sequence, head): its token at position len - 1.
__global__ __launch_bounds__(64) void k_append(AttendArgs a) {
  const CacheView& c = a.c;
  const long long i = blockIdx.x * 64ll + threadIdx.x;
  if (i >= static_cast<long long>(a.n_seqs) * c.kv_heads) return;
  const int s = static_cast<int>(i / c.kv_heads), h = static_cast<int>(i - static_cast<long long>(s) * c.kv_heads);
  const int n = keys_of(a.lens, s, a.max_len, a.table_ld, c.ps);
  if (n == 0) return;
  const int t = (n - 1) % c.ps, id = page_at(a.table, a.table_ld, s, (n - 1) / c.ps, c.pages);
  if (id < 0) return;
  const size_t hb = head_block(c, a.layer, id, h);
  for (int is_v = 0; is_v < 2; ++is_v) {
    const void* x = is_v ? a.new_v : a.new_k;
    const size_t x0 = static_cast<size_t>(s) * a.new_ld + static_cast<size_t>(h) * c.dh;
    char* base = is_v ? c.v : c.k;
    const int per = c.dh / c.groups;
    for (int g = 0; g < c.groups; ++g) {
      float step = 0.f, least = 0.f;
      if (c.type == CT_INT4) {
        float lo = INFINITY, hi = -INFINITY;
        bool fin = true;
        for (int d = g * per; d < (g + 1) * per; ++d) {
          const float v = load_any(x, a.new_bf16, x0 + d);
          lo = fminf(lo, v);
          hi = fmaxf(hi, v);
          fin = fin && isfinite(v);
        }
        group_params(lo, hi, fin, step, least);
        reinterpret_cast<uint32_t*>(is_v ? c.vs : c.ks)[(hb * c.ps + t) * c.groups + g] =
            (__float_as_uint(step) >> 16) | (__float_as_uint(least) & 0xffff0000u);
      }
      for (int d = g * per; d < (g + 1) * per; ++d) {
        const float v = load_any(x, a.new_bf16, x0 + d);
        const size_t o = hb * c.ps * c.dh + (is_v ? static_cast<size_t>(d) * c.ps + t : static_cast<size_t>(t) * c.dh + d);
        if (c.type == CT_F32) {
          reinterpret_cast<float*>(base)[o] = v;
        } else if (c.type == CT_BF16) {
          reinterpret_cast<bf16_t*>(base)[o] = f32_to_bf16(v);
        } else {
          uint32_t* w = reinterpret_cast<uint32_t*>(base) + (o >> 3);
          const int sh = nibble_shift(static_cast<int>(o & 7));
          *w = (*w & ~(15u << sh)) | (group_code(v, step, least) << sh);
        }
      }
    }
  }
}

constexpr int kAttnThreads = 64;

// One wave per (sequence, head); a lane keeps its own running maximum, sum and
// output over keys lane, lane + 64, ...
__global__ __launch_bounds__(kAttnThreads) void k_attend(AttendArgs a) {
  const CacheView& c = a.c;
  const int s = blockIdx.x / a.heads, h = blockIdx.x % a.heads, lane = threadIdx.x;
  const int kv = h / (a.heads / c.kv_heads);
  const int n = keys_of(a.lens, s, a.max_len, a.table_ld, c.ps);
  __shared__ float s_q[128];
  __shared__ float s_o[kAttnThreads][129];
  for (int d = lane; d < c.dh; d += kAttnThreads)
    s_q[d] = load_any(a.q, a.q_bf16, static_cast<size_t>(s) * a.q_ld + static_cast<size_t>(h) * c.dh + d);
  for (int d = 0; d < c.dh; ++d) s_o[lane][d] = 0.f;
  __syncthreads();
  float m = -INFINITY, l = 0.f;
  for (int j = lane; j < n; j += kAttnThreads) {
    const int id = page_at(a.table, a.table_ld, s, j / c.ps, c.pages);
    if (id < 0) continue;
    const size_t hb = head_block(c, a.layer, id, kv);
    float dot = 0.f;
    for (int d = 0; d < c.dh; ++d) dot = fmaf(s_q[d], cache_value(c, hb, j % c.ps, d, 0), dot);
    const float sc = dot * a.scale, mn = fmaxf(m, sc);
    const float f = m == -INFINITY ? 0.f : expf(m - mn), p = expf(sc - mn);
    for (int d = 0; d < c.dh; ++d) s_o[lane][d] = fmaf(p, cache_value(c, hb, j % c.ps, d, 1), s_o[lane][d] * f);
    l = l * f + p;
    m = mn;
  }
  const float mx = wave_max(m);
  const float f = m == -INFINITY ? 0.f : expf(m - mx);
  const float sum = wave_sum(l * f);
  for (int d = 0; d < c.dh; ++d) s_o[lane][d] *= f;
  __syncthreads();
  for (int d = lane; d < c.dh; d += kAttnThreads) {
    float o = 0.f;
    for (int i = 0; i < kAttnThreads; ++i) o += s_o[i][d];
    o = sum > 0.f || sum != sum ? o / sum : 0.f;
    const size_t at = static_cast<size_t>(s) * a.out_ld + static_cast<size_t>(h) * c.dh + d;
    if (a.out_bf16) Elt<bf16_t>::store(static_cast<bf16_t*>(a.out), at, o);
    else static_cast<float*>(a.out)[at] = o;
  }
}

__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  const CacheView& c = a.c;
  const size_t per = static_cast<size_t>(c.kv_heads) * c.dh;
  const size_t total = static_cast<size_t>(a.n_seqs) * a.count * per;
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < total; i += gridDim.x * 256ull) {
    const size_t tok = i / per;
    const int hd = static_cast<int>(i - tok * per), h = hd / c.dh, d = hd - h * c.dh;
    const int s = static_cast<int>(tok / a.count);
    const long long j = static_cast<long long>(a.first[s]) + static_cast<long long>(tok - static_cast<size_t>(s) * a.count);
    const int n = keys_of(a.lens, s, 0x7fffffff, a.table_ld, c.ps);
    float k = 0.f, v = 0.f;
    if (j >= 0 && j < n) {
      const int id = page_at(a.table, a.table_ld, s, static_cast<int>(j / c.ps), c.pages);
      if (id >= 0) {
        const size_t hb = head_block(c, a.layer, id, h);
        k = cache_value(c, hb, static_cast<int>(j % c.ps), d, 0);
        v = cache_value(c, hb, static_cast<int>(j % c.ps), d, 1);
      }
    }
    a.out_k[i] = k;
    a.out_v[i] = v;
  }
}

}  // namespace

size_t attend_workspace(const CacheView& c, int n_seqs, int heads, int group, int max_len) { return 0; }

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s) {
  if (a.new_k != nullptr) {
    const long long n = static_cast<long long>(a.n_seqs) * a.c.kv_heads;
    hipLaunchKernelGGL(k_append, dim3(static_cast<unsigned>((n + 63) / 64)), dim3(64), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_attend, dim3(a.n_seqs * a.heads), dim3(kAttnThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_read(const ReadArgs& a, hipStream_t s) {
  const size_t total = static_cast<size_t>(a.n_seqs) * a.count * a.c.kv_heads * a.c.dh;
  const size_t wgs = (total + 255) / 256;
  hipLaunchKernelGGL(k_read, dim3(static_cast<unsigned>(wgs < 8192 ? wgs : 8192)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace pdec
