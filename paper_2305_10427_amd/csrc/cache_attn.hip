// Attention of single tokens over a paged cache, the append of a token, and
// the reading back of a cache's values.
//
//   o[s,h] = sum_j p_j v_j,  p = softmax_j(scale q[s,h] . k_j),  j < len[s]
// with k_j, v_j the key and value of head h / (heads / kv_heads) in slot
// j mod page_size of page table[s][j / page_size].  Keys of pages that do not
// exist (an id outside the pool) are left out; a row without keys is zero.
#include <type_traits>
#include <utility>

#include "common.h"
#include "mma.h"
#include "operators.h"

namespace pdec {

namespace {

constexpr float kFloatMax = 3.4028234664e38f, kBf16Max = 3.3895313892e38f;

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
  // the product is exact, and within the sum it cannot overflow; the sixteenth
  // value of a group can lie above float's largest
  const float x = fmaf(code, __uint_as_float(par << 16), __uint_as_float(par & 0xffff0000u));
  return x > kFloatMax ? kFloatMax : x;               // NaN stays
}

// The largest bfloat16 up to x (x itself if it is not finite).
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t u = __float_as_uint(x), low = u & 0xffffu;
  return __uint_as_float(u - low + (low != 0 && x < 0.f ? 0x10000u : 0u));
}

// Step and least value of a group with the extremes lo, hi: the least value is
// rounded down (to bfloat16's lowest at most) and the step up to bfloat16, so that
// the fifteen steps reach hi; the test of the step is an exact product.  A range
// beyond float's, and its step, are taken by half.  A group with a value that is
// not finite becomes NaN as a whole.
__device__ __forceinline__ void group_params(float lo, float hi, bool finite, float& step, float& least) {
  least = fmaxf(bf16_down(lo), -kBf16Max);
  const bool wide = hi - least > kFloatMax;
  const float range = wide ? hi * 0.5f - least * 0.5f : hi - least;
  step = bf16_down(range * (1.f / 15.f));
  if (step * 15.f < range) step = __uint_as_float(__float_as_uint(step) + 0x10000u);
  if (wide) step *= 2.f;
  if (!finite) step = 0.f, least = NAN;
}
__device__ __forceinline__ uint32_t group_code(float x, float step, float least) {
  if (!(step > 0.f)) return 0u;
  const float d = x - least;
  const float c = rintf(d > kFloatMax ? (x * 0.5f - least * 0.5f) / (step * 0.5f) : d / step);
  return static_cast<uint32_t>(fminf(fmaxf(c, 0.f), 15.f));
}

// --- the tile ------------------------------------------------------------------
//
// A workgroup takes up to 16 query rows that read the same key/value head: the
// beams of a group (up to 16 / G) times the G query heads of the key head, and a
// part of the key blocks of 32 positions.  For each block it finds the distinct
// (pages, valid keys) among its beams: beams that share a prefix share one
// item, so a page is read once however many of them refer to it.  Waves take
// items in turn; an item's keys are scored against all 16 rows on the matrix
// cores (16x16 tiles: rows are keys, columns are queries) and only the rows
// that own the item take the result.
//
// Key kappa of a block sits in row 4 (kappa / 8) + kappa % 4 of score tile
// (kappa / 4) % 2, so that lane (n, g) = (lane % 16, lane / 16) ends up with the
// scores of keys 8 g .. 8 g + 7 for query n, in the order in which the product
// with V wants its weights: eight consecutive keys a lane, and V's pages hold
// the keys of a dimension next to each other.
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kBlock = 32;                    // keys of an item
constexpr int kUnit = 4;                      // blocks handed out together (128 keys: whole pages)
constexpr float kLog2e = 1.4426950408889634f;

struct Item {
  int id0, id1;                               // pages of the block's halves (-1: none)
  int block;
  uint32_t rows_nv;                           // beams that own it (bits 16 ..), valid keys (low bits)
};

__device__ __forceinline__ void unpack_pair(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ float xor16_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor32_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor16_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float xor32_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sum of the two doubles of which lo and hi hold the words.
template <typename P> __device__ __forceinline__ double pair_sum(const P& lo, const P& hi) {
  auto at = [&](int i) { return __longlong_as_double(static_cast<long long>(static_cast<uint64_t>(hi[i]) << 32 | lo[i])); };
  return at(0) + at(1);
}
__device__ __forceinline__ double xor16_sum_d(double v) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const auto lo = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(u), static_cast<uint32_t>(u), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(u >> 32), static_cast<uint32_t>(u >> 32), false, false);
  return pair_sum(lo, hi);
}
__device__ __forceinline__ double xor32_sum_d(double v) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const auto lo = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(u), static_cast<uint32_t>(u), false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(u >> 32), static_cast<uint32_t>(u >> 32), false, false);
  return pair_sum(lo, hi);
}

// A product of bfloat16 parts starts with the smallest: one rounding at the full
// magnitude instead of one a part.
__device__ __forceinline__ floatx4_t mma_bf16(uint4 a, uint4 b, floatx4_t c) { return Mma<bf16_t>::step(a, b, c); }
__device__ __forceinline__ floatx4_t mma_f32(float a, float b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Eight floats rounded to bfloat16, and what they leave of v.
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void take_off(float* v, uint4 p) {   // v -= p
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] -= __uint_as_float(w[j] << 16);
    v[2 * j + 1] -= __uint_as_float(w[j] & 0xffff0000u);
  }
}

// Eight floats in three bfloat16 parts of 8 bits each, exactly: the first two are
// the largest bfloat16 below the magnitude of what is left (its bits less one, cut),
// so every part has the value's sign and none is 0 unless the value is (which must
// not be -0).  A product with an infinite key or value, or one that overflows, is
// then the same infinity in every part; parts rounded to nearest differ in sign or
// are 0, and their sum would be NaN.
__device__ __forceinline__ uint4 pack8_below(const float* v) {
  uint32_t u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) u[j] = __builtin_elementwise_sub_sat(__float_as_uint(v[j]), 1u);
  auto two = [&](int j) { return __builtin_amdgcn_perm(u[j + 1], u[j], 0x07060302u); };
  return make_uint4(two(0), two(2), two(4), two(6));
}
__device__ __forceinline__ void split8(float* v, uint4& p0, uint4& p1, uint4& p2) {
  p0 = pack8_below(v);
  take_off(v, p0);
  p1 = pack8_below(v);
  take_off(v, p1);
  p2 = pack8(v);
}

// The eight codes of a word as bfloat16 16 + code: a code fills the top of the
// mantissa of 16 (exact), two of them in a shift and an AND-OR (whose masks are
// kept in vector registers: the instruction takes no two constants).  Scores
// take the offset off with the least values; the product with V takes off
// 16 + 7.5 inside the matrix product and adds the middle of a group's range
// apart, because its sum over many keys of differing sign would otherwise be a
// small difference of large numbers.
__device__ __forceinline__ uint4 codes_bf16(uint32_t w, uint32_t m, uint32_t e) {
  return make_uint4(((w << 3) & m) | e, ((w >> 1) & m) | e, ((w >> 5) & m) | e, ((w >> 9) & m) | e);
}
__device__ __forceinline__ uint32_t in_vgpr(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
constexpr uint32_t kCodeMask = 0x00780078u, kCodeExp = 0x41804180u;
constexpr float kCodeMid = 7.5f;
constexpr uint32_t kMinusMid2 = 0xc1bcc1bcu;   // two bfloat16 of -(16 + 7.5)

// The append of a token, eight dimensions of its key or value a lane: entry i
// of a tile is beam i / (2 DH / 8), the key or value, and the dimensions.
template <int DH> struct AppendRow {
  static constexpr int L8 = DH / 8;
  int r, is_v, d, pos;
  float x[8];
  __device__ __forceinline__ void load(const AttendArgs& a, int kv, int seq0, int beams, int i) {
    r = i / (2 * L8);
    is_v = i / L8 & 1;
    d = 8 * (i & (L8 - 1));
    const bool in = r < beams;
    r = in ? r : 0;
    const void* src = is_v ? a.new_v : a.new_k;
    const size_t x0 = static_cast<size_t>(seq0 + r) * a.new_ld + static_cast<size_t>(kv) * DH + d;
    if (a.new_bf16) Vec16<bf16_t>::load(static_cast<const bf16_t*>(src), x0, x);
    else load_n<float, 8>(static_cast<const float*>(src), x0, x);
    const int n = keys_of(a.lens, seq0 + r, a.max_len, a.table_ld, a.c.ps);
    pos = in && a.lens[seq0 + r] == n ? n - 1 : -1;      // a length that was cut has its last position elsewhere
  }
};

// Writes it to page id (-1: not at all).  In 4 bits a group's extremes come from
// the lanes that hold it.  The slots belong to one sequence each, so the words
// that hold several tokens are read, changed and written by one lane.  All
// lanes call this together.
template <int CT, int DH>
__device__ __forceinline__ void append_row(const AttendArgs& a, int kv, const AppendRow<DH>& row_, int id) {
  const CacheView& c = a.c;
  constexpr int G = DH >= 32 ? DH / 32 : 1;
  const float* x = row_.x;
  const int is_v = row_.is_v, d = row_.d, pos = row_.pos;
  float step = 0.f, least = 0.f;
  if constexpr (CT == CT_INT4) {
    float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
      bad = isfinite(x[e]) ? bad : 1.f;
    }
    lo = fminf(lo, dpp_f<kDppXor1>(lo)); hi = fmaxf(hi, dpp_f<kDppXor1>(hi)); bad = fmaxf(bad, dpp_f<kDppXor1>(bad));
    if constexpr (DH >= 32) {
      lo = fminf(lo, dpp_f<kDppXor2>(lo)); hi = fmaxf(hi, dpp_f<kDppXor2>(hi)); bad = fmaxf(bad, dpp_f<kDppXor2>(bad));
    }
    group_params(lo, hi, bad == 0.f, step, least);
  }
  if (id < 0) return;
  const size_t hb = head_block(c, a.layer, id, kv);
  const int t = pos & (c.ps - 1);
  char* base = is_v ? c.v : c.k;
  const size_t row = (hb * c.ps + t) * DH + d;            // K
  if constexpr (CT == CT_INT4) {
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = group_code(x[e], step, least);
    if (d % 32 == 0)
      reinterpret_cast<uint32_t*>(is_v ? c.vs : c.ks)[(hb * c.ps + t) * G + d / 32] =
          (__float_as_uint(step) >> 16) | (__float_as_uint(least) & 0xffff0000u);
    uint32_t* w = reinterpret_cast<uint32_t*>(base);
    if (!is_v) {
      uint32_t word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) word |= code[e] << nibble_shift(e);
      w[row >> 3] = word;
    } else {
      const int sh = nibble_shift(t & 7);
      uint32_t old[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) old[e] = w[((hb * DH + d + e) * c.ps + t) >> 3];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[((hb * DH + d + e) * c.ps + t) >> 3] = (old[e] & ~(15u << sh)) | (code[e] << sh);
    }
  } else {
    typedef typename std::conditional<CT == CT_F32, float, bf16_t>::type T;
    T* w = reinterpret_cast<T*>(base);
    if (!is_v) {
      store8<T>(w, row, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) Elt<T>::store(w, (hb * DH + d + e) * c.ps + t, x[e]);
    }
  }
}

// out = o / l for four dimensions of a row; a row without keys is zero.
__device__ __forceinline__ void store_out(const AttendArgs& a, int s, int h, int d, const floatx4_t& o, float l) {
  const float inv = l != 0.f ? 1.f / l : 0.f;      // NaN stays
  const size_t at = static_cast<size_t>(s) * a.out_ld + static_cast<size_t>(h) * a.c.dh + d;
  if (a.out_bf16) {
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + at) =
        make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
  } else {
    *reinterpret_cast<floatx4_t*>(static_cast<float*>(a.out) + at) = floatx4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  }
}

// Lane L of every 16 lanes, to all of them (an operand modifier of the instruction that uses it).
template <int L> __device__ __forceinline__ float row_lane(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x150 + L, 0xF, 0xF, true));
}

typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// Calls f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>).
template <typename F, int... I> __device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void each(F&& f) { each_of(std::make_integer_sequence<int, N>{}, f); }

// The data of an item on its way: pieces of 16 bytes (8 where a row or the half
// of one is no longer) in the order in which they lie in memory, neighbouring
// lanes on neighbouring pieces, then through LDS into the order of the matrix
// cores.  A lane that loads its operands itself takes 16 bytes (4 bits: 4) from
// a row of its own, which keeps the address unit busy for 64 rows an
// instruction: 64 x 4 rows of 4,000 keys of 64, bfloat16 3.2 TB/s and 4 bits
// 1.1 TB/s that way.
//
// LDS: K rows in the order of the score tiles (key 8 a + 4 t + b in row
// 16 t + 4 a + b), V rows by dimension, both padded so that the 16 rows of a read
// start in different banks.  In 4 bits the (step, least) words of a row of
// lanes' eight keys stay in registers, one a lane (word w = key * groups + group
// in register w / 16 of lane w % 16); the keys' ones also lie behind their rows.
template <int CT, int DH> struct Stage {
  static constexpr int NU = DH >= 32 ? DH / 32 : 1;
  static constexpr int NW = NU >= 2 ? NU / 2 : 1;
  static constexpr int kRow = CT == CT_F32 ? 4 * DH : CT == CT_BF16 ? 2 * DH : DH / 2;      // bytes of a key
  static constexpr int kSeg = CT == CT_F32 ? 128 : CT == CT_BF16 ? 64 : 16;                 // of 32 keys of a dimension
  static constexpr int kPiece = CT == CT_INT4 ? 8 : 16;
  static constexpr int kRowLds = kRow + 16;                                                 // 4 bits: a key's words behind it
  static constexpr int kSegLds = kSeg > 16 ? kSeg + 16 : kSeg;
  static constexpr int kOut = 16 * (DH + 4) * 4;                                            // of a wave's output
  static constexpr int kBytes = kBlock * kRowLds + DH * kSegLds > kOut ? kBlock * kRowLds + DH * kSegLds : kOut;
  static constexpr int NK = (kBlock * kRow / kPiece + kWave - 1) / kWave;                   // pieces a lane
  static constexpr int NV = (DH * kSeg / kPiece + kWave - 1) / kWave;
  static constexpr int PK = kRow / kPiece, PH = kSeg / 2 / kPiece;                          // pieces of a key, of half a segment
  static constexpr bool kFullK = kBlock * PK % kWave == 0, kFullV = DH * 2 * PH % kWave == 0;
  typedef typename std::conditional<kPiece == 16, u32x4_t, u32x2_t>::type Piece;
  Piece k[NK], v[NV];
  uint32_t kp[CT == CT_INT4 ? NW : 1], vp[CT == CT_INT4 ? NW : 1];
  // A page that is missing is never used: any block serves as its address.
  __device__ __forceinline__ void load(const CacheView& c, int layer, int kv, const Item& it, int lane) {
    const int ps = c.ps, j0 = it.block * kBlock;
    const size_t hb0 = head_block(c, layer, max(it.id0, 0), kv), hb1 = head_block(c, layer, max(it.id1, 0), kv);
    const int s0 = j0 & (ps - 1), s1 = (j0 + 16) & (ps - 1);      // slots of the halves
    const char* k0 = c.k + (hb0 * ps + s0) * kRow;
    const char* k1 = c.k + (hb1 * ps + s1) * kRow;
    const int dim_bytes = ps * kSeg / kBlock;                     // from a dimension to the next
    const char* v0 = c.v + hb0 * DH * dim_bytes + s0 * kSeg / kBlock;
    const char* v1 = c.v + hb1 * DH * dim_bytes + s1 * kSeg / kBlock;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      int x = i * kWave + lane;
      if (!kFullK) x = min(x, kBlock * PK - 1);
      const bool up = x >= 16 * PK;
      k[i] = *reinterpret_cast<const Piece*>((up ? k1 : k0) + (x - (up ? 16 * PK : 0)) * kPiece);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      int dim, half, q;
      v_place(i, lane, ps, dim, half, q);
      v[i] = *reinterpret_cast<const Piece*>((half ? v1 : v0) + dim * dim_bytes + q * kPiece);
    }
    if constexpr (CT == CT_INT4) {
      const int n = lane & 15, g = lane >> 4;
      const size_t at = ((g < 2 ? hb0 * ps + s0 : hb1 * ps + s1) + 8 * (g & 1)) * NU + (NU >= 2 ? n : n & 7);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        kp[w] = reinterpret_cast<const uint32_t*>(c.ks)[at + 16 * w];
        vp[w] = reinterpret_cast<const uint32_t*>(c.vs)[at + 16 * w];
      }
    }
  }
  // Piece i of a lane: pages of 16 keys are taken one after the other, longer
  // ones a dimension at a time.
  static __device__ __forceinline__ void v_place(int i, int lane, int ps, int& dim, int& half, int& q) {
    int x = i * kWave + lane;
    if (!kFullV) x = min(x, DH * 2 * PH - 1);
    q = x % PH;
    if (ps == 16) {
      half = x >= DH * PH ? 1 : 0;
      dim = x / PH - half * DH;
    } else {
      half = x / PH & 1;
      dim = x / (2 * PH);
    }
  }
  __device__ __forceinline__ void store(char* lds, int lane, int ps) const {
    if constexpr (CT == CT_INT4) {
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int at = 16 * w + (NU >= 2 ? lane & 15 : lane & 7), j = at / NU;
        const int row = (j & 4) * 4 + (lane >> 4) * 4 + (j & 3);                            // of key 8 (lane / 16) + j
        *reinterpret_cast<uint32_t*>(lds + row * kRowLds + kRow + 4 * (at % NU)) = kp[w];
      }
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      int x = i * kWave + lane;
      if (!kFullK) x = min(x, kBlock * PK - 1);
      const int key = x / PK, row = (key & 4) * 4 + (key >> 3) * 4 + (key & 3);
      *reinterpret_cast<Piece*>(lds + row * kRowLds + x % PK * kPiece) = k[i];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      int dim, half, q;
      v_place(i, lane, ps, dim, half, q);
      *reinterpret_cast<Piece*>(lds + kBlock * kRowLds + dim * kSegLds + half * (kSeg / 2) + q * kPiece) = v[i];
    }
  }
};

template <int CT> constexpr int kSegLane = CT == CT_F32 ? 32 : CT == CT_BF16 ? 16 : 4;   // bytes of eight keys of a dimension

// Split of the launch: beams per tile, tiles of a group, parts of the keys.
// Part z takes units z, z + splits, ...: behind the beams' common prefix a block
// has an item for each of them, and units in turn spread those over the parts.
// Evenly only where there are many more of them than parts: 2 x 4 rows of 20,011 ..
// 32,749 keys, nine tenths in common, have 16 to 26 such units for 64 parts, so a
// wave has 4.2 items on average and 7 at most.
struct Plan {
  int rows_per_tile, tiles, splits;
};

// Waves a SIMD is to hold (workgroups a CU): what the registers of an instance and
// its LDS allow without spilling.
constexpr int waves_per_simd(int ct, int dh) {
  if (ct == CT_F32) return dh >= 128 ? 1 : dh == 64 ? 2 : dh == 32 ? 3 : 4;
  if (ct == CT_BF16) return dh >= 128 ? 1 : dh == 64 ? 3 : 4;
  return dh >= 128 ? 2 : dh == 64 ? 3 : 4;
}

// Long caches are bound by memory in float32 and bfloat16 (16 rows of 8,191 ..
// 16,381 keys, 16 heads of 64, bfloat16, 805 MB: 151 us, 5.3 TB/s; 8 heads of 64 in
// float32: 154 us, 5.2; reading alone reaches 5.9).  In 4 bits (64 x 4 rows of 4,000
// keys of 64, 312 MB: 124 us, 2.5 TB/s; 2 x 4 rows of 20,011 .. 32,749 keys, 4 heads
// of 128 for 16, 44 MB: 30.6 us) a wave issues vector instructions, which unpack
// codes and split weights, 38% of its time and waits 35%, and waves have unequal
// work.  Short ones are a chain of latencies - lengths, table, keys, products, the
// waves' join - of 6 us for one sentence.  With 512 workgroups (64 x 5 rows of 15 ..
// 138 keys, 8 heads, bfloat16, 29 MB) they take 16.3 us: the longest sentence's
// busiest wave has 5 items, one requested ahead, and waits 54% of its time; 1.6 of it
// is the append, whose stores have to land before its keys are read.
//
// Weights enter the product with V in three bfloat16 parts, float's own 2^-24,
// whatever the output's type: with two (2^-17) 1.0e-3 to 1.7e-3 of the bfloat16
// outputs were not the rounded exact sums, two to three times as many as from plain
// float.  The third costs the cache in 4 bits up to a tenth (64 x 4 rows of 4,000 keys
// of 64: 112 and 124 us), the others at most 0.5 us a call.
template <int CT, int DH>
__global__ __launch_bounds__(kThreads, waves_per_simd(CT, DH)) void k_attend(AttendArgs a, Plan pl) {
  constexpr int NU = DH >= 32 ? DH / 32 : 1;          // steps of 32 dimensions (bf16 products), groups of a cache in 4 bits
  constexpr int NT = DH / 16;                         // tiles of 16 dimensions
  constexpr int NF = CT == CT_F32 ? DH / 16 : 1;      // float: steps of 16 dimensions
  const CacheView& c = a.c;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int n = lane & 15, g = lane >> 4;
  const int G = a.heads / c.kv_heads;
  int wg = blockIdx.x;
  const int split = wg % pl.splits; wg /= pl.splits;
  const int kv = wg % c.kv_heads; wg /= c.kv_heads;
  const int tile = wg % pl.tiles;
  const int grp = wg / pl.tiles;
  const int beam0 = tile * pl.rows_per_tile;
  const int beams = min(pl.rows_per_tile, a.group - beam0);
  const int seq0 = grp * a.group + beam0;
  const int ps = c.ps;

  // each wave's own: its list of items, the data of one, and at the end its output
  typedef Stage<CT, DH> SG;
  struct WaveLds {
    Item item[kWave];
    int4 tup[kWave];
    union {
      char stage[SG::kBytes];
      float out[16][DH + 4];
    };
  };
  __shared__ __align__(16) char s_mem[kWaves * sizeof(WaveLds)];
  WaveLds* s_wave = reinterpret_cast<WaveLds*>(s_mem);
  WaveLds& my = s_wave[wave];
  char* lds = my.stage;
  const char* k_lds = lds + n * SG::kRowLds + (CT == CT_INT4 ? (DH >= 32 ? 4 * g : 4 * (g & 1)) : CT == CT_BF16 && DH < 32 ? 16 * (g & 1) : 16 * g);
  const char* v_lds = lds + kBlock * SG::kRowLds + n * SG::kSegLds + kSegLane<CT> * g;
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];

  // --- what depends on nothing else is requested first ---
  AppendRow<DH> ap;
  if (a.new_k != nullptr) ap.load(a, kv, seq0, beams, threadIdx.x);
  // a list: the lane's (block, beam) of kWave / beams blocks, their pages
  const int list_blocks = kWave / beams;
  const int b_l = lane / beams, r_l = lane - b_l * beams;
  const bool pair = b_l < list_blocks;
  auto block_of = [&](int i) { return ((i / kUnit) * pl.splits + split) * kUnit + i % kUnit; };   // my i-th block
  int id0 = -1, id1 = -1;
  auto fetch = [&](int list) {
    const int j = block_of(list * list_blocks + b_l) * kBlock / ps;
    id0 = pair && j < a.table_ld ? page_at(a.table, a.table_ld, seq0 + r_l, j, c.pages) : -1;
    id1 = ps > 16 ? id0 : pair && j + 1 < a.table_ld ? page_at(a.table, a.table_ld, seq0 + r_l, j + 1, c.pages) : -1;
  };
  fetch(0);
  const int len = pair ? keys_of(a.lens, seq0 + r_l, a.max_len, a.table_ld, ps) : 0;
  // queries: lane (n, g) holds dimensions 32 u + 8 g .. + 7 (float: 16 u + 4 g .. + 3) of row n
  const int beam_n = n / G;
  const bool row_ok = beam_n < beams;
  const size_t q0 = static_cast<size_t>(seq0 + (row_ok ? beam_n : 0)) * a.q_ld +
                    (static_cast<size_t>(kv) * G + (row_ok ? n % G : 0)) * DH;
  constexpr int QE = CT == CT_F32 ? 4 : 8, QU = CT == CT_F32 ? DH / 16 : NU;
  const int q_at = CT == CT_F32 ? 4 * g : DH >= 32 ? 8 * g : 8 * (g & 1);
  float qv[QU][QE];
  if (a.q_bf16) {
#pragma unroll
    for (int u = 0; u < QU; ++u) {
      const bf16_t* p = static_cast<const bf16_t*>(a.q) + q0 + 4 * QE * u + q_at;
      if constexpr (QE == 8) {
        Vec16<bf16_t>::load(p, 0, qv[u]);
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        unpack_pair(w.x, qv[u][0], qv[u][1]);
        unpack_pair(w.y, qv[u][2], qv[u][3]);
      }
    }
  } else {
#pragma unroll
    for (int u = 0; u < QU; ++u) load_n<float, QE>(static_cast<const float*>(a.q), q0 + 4 * QE * u + q_at, qv[u]);
  }
  int ap_id = -1;
  auto my_slot = [&](int pos) { return pos >= 0 && pos / (kUnit * kBlock) % pl.splits == split; };
  if (a.new_k != nullptr && my_slot(ap.pos)) ap_id = page_at(a.table, a.table_ld, seq0 + ap.r, ap.pos / ps, c.pages);

  const float s2 = a.scale * kLog2e;                  // scores come out in units of log 2
  const float sq = DH >= 32 ? s2 : 0.5f * s2;         // 16 dimensions fill a step of 32 twice, each time by half
  uint4 qf[CT == CT_F32 ? 1 : NU][3];
  floatx4_t q32[NF];
  uint4 qpar = make_uint4(0u, 0u, 0u, 0u);            // 4 bits: what multiplies a key's (step, least) words
  if constexpr (CT == CT_F32) {
#pragma unroll
    for (int u = 0; u < NF; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) q32[u][e] = row_ok ? s2 * qv[u][e] : 0.f;
  } else {
    // A score is sum_u step (sum_d (16 + code) q - 16 qs) + least qs with qs the
    // sum of q over group u: the last two terms are a product of the key's words
    // with (-16 qs, qs), a row of lanes for each of four bfloat16 parts of those.
    // The terms are several times the score, so qs is summed in double.
    double par[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) par[e] = 0.0;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      float* v = qv[u];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = row_ok ? sq * v[e] + 0.f : 0.f;   // no -0
      if constexpr (CT == CT_INT4) {
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += static_cast<double>(v[e]);
        par[2 * u + 1] = xor32_sum_d(xor16_sum_d(sum));
        par[2 * u] = -16.0 * par[2 * u + 1];
      }
      split8(v, qf[u][0], qf[u][1], qf[u][2]);
    }
    if constexpr (CT == CT_INT4) {
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = static_cast<float>(par[e]);
        const uint4 x = pack8(f);
        if (g == part) qpar = x;
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float lo, hi;
          unpack_pair(w[e / 2], lo, hi);
          par[e] -= static_cast<double>(e % 2 ? hi : lo);
        }
      }
    }
  }
  const int longest = static_cast<int>(wave_max_u32(static_cast<uint32_t>(len)));
  const int units = (longest + kUnit * kBlock - 1) / (kUnit * kBlock);
  const int my_blocks = split < units ? (units - split + pl.splits - 1) / pl.splits * kUnit : 0;
  const int lists = (my_blocks + list_blocks - 1) / list_blocks;

  // The items of list `list` (every wave makes the same one, without a word to
  // the others) from the pages that have been fetched; then the next ones are.
  auto make_list = [&](int list) -> int {
    const int block = block_of(list * list_blocks + b_l);
    const int nv = max(0, min(kBlock, len - block * kBlock));
    const int4 t = make_int4(nv > 0 ? id0 : -1, nv > 16 ? id1 : -1, nv, 0);
    wave_lds_sync();
    my.tup[lane] = t;
    wave_lds_sync();
    bool lead = t.x >= 0 || t.y >= 0;
    uint32_t rows = 0;
    for (int o = 0; o < beams; ++o) {
      const int4 x = my.tup[min(b_l * beams + o, kWave - 1)];
      const bool same = x.x == t.x && x.y == t.y && x.z == t.z;
      rows |= same ? 1u << o : 0u;
      if (same && o < r_l) lead = false;
    }
    const uint64_t vote = __ballot(lead);
    if (lead) my.item[__popcll(vote & ((1ull << lane) - 1))] = Item{t.x, t.y, block, rows << 16 | static_cast<uint32_t>(nv)};
    wave_lds_sync();
    if (list + 1 < lists) fetch(list + 1);
    return __popcll(vote);
  };
  int list = 0, n_items = lists > 0 ? make_list(0) : 0, at_item = wave;
  // The wave's next item: every kWaves-th of all lists'.
  auto seek = [&](Item& it) -> bool {
    while (at_item >= n_items) {
      at_item -= n_items;
      if (++list >= lists) return false;
      n_items = make_list(list);
    }
    const Item x = my.item[at_item];
    at_item += kWaves;
    it.id0 = __builtin_amdgcn_readfirstlane(x.id0);
    it.id1 = __builtin_amdgcn_readfirstlane(x.id1);
    it.block = __builtin_amdgcn_readfirstlane(x.block);
    it.rows_nv = __builtin_amdgcn_readfirstlane(x.rows_nv);
    return true;
  };

  // the step's own token, by the workgroup whose part holds its position
  if (a.new_k != nullptr) {
    append_row<CT, DH>(a, kv, ap, ap_id);
    for (int i = kThreads; i < beams * 2 * AppendRow<DH>::L8; i += kThreads) {
      ap.load(a, kv, seq0, beams, i + threadIdx.x);
      append_row<CT, DH>(a, kv, ap, my_slot(ap.pos) ? page_at(a.table, a.table_ld, seq0 + ap.r, ap.pos / ps, c.pages) : -1);
    }
    __threadfence_block();
    __syncthreads();
  }

  const uint32_t cm = CT == CT_INT4 ? in_vgpr(kCodeMask) : 0u, ce = CT == CT_INT4 ? in_vgpr(kCodeExp) : 0u;
  float m = -INFINITY, l = 0.f;
  floatx4_t acc[NT];
  float mid[NU];                                      // 4 bits: sum of p times the middle of a key's group, own keys
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < NU; ++u) mid[u] = 0.f;

  // a wave's items: one in LDS, the next one on its way in registers
  {
    Stage<CT, DH> st;
    uint32_t kp[SG::NW], vp[SG::NW];
    Item next;
    bool more = seek(next);
    if (more) st.load(c, a.layer, kv, next, lane);
    while (more) {
      const Item it = next;
      wave_lds_sync();                                   // the wave is done with the item before
      st.store(lds, lane, ps);
#pragma unroll
      for (int w = 0; w < SG::NW; ++w) {
        if constexpr (CT == CT_INT4) kp[w] = st.kp[w], vp[w] = st.vp[w];
      }
      wave_lds_sync();
      more = seek(next);
      if (more) st.load(c, a.layer, kv, next, lane);
      const int nv = it.rows_nv & 0xffff;
      const bool own = row_ok && ((it.rows_nv >> 16) >> beam_n & 1u);
      const bool whole = nv == kBlock && it.id0 >= 0 && it.id1 >= 0;
      // --- scores of keys 8 g + j, in units of log 2 ---
      constexpr int NW = SG::NW;
      float sc[8], kstep[NW];
      if constexpr (CT == CT_INT4) {
#pragma unroll
        for (int w = 0; w < NW; ++w) kstep[w] = __uint_as_float(kp[w] << 16);
      }
      each<2>([&](auto t_) {
        constexpr int t = decltype(t_)::value;
        floatx4_t d = {0.f, 0.f, 0.f, 0.f};
        if constexpr (CT == CT_F32) {
#pragma unroll
          for (int u = 0; u < NF; ++u) {
            const floatx4_t x = *reinterpret_cast<const floatx4_t*>(k_lds + t * 16 * SG::kRowLds + 64 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) d = mma_f32(x[e], q32[u][e], d);
          }
        } else if constexpr (CT == CT_BF16) {
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            const uint4 x = *reinterpret_cast<const uint4*>(k_lds + t * 16 * SG::kRowLds + 64 * u);
#pragma unroll
            for (int part = 2; part >= 0; --part) d = mma_bf16(x, qf[u][part], d);
          }
        } else {
          const uint32_t* w4 = reinterpret_cast<const uint32_t*>(lds + (16 * t + n) * SG::kRowLds + SG::kRow);
          d = mma_bf16(make_uint4(w4[0], NU > 1 ? w4[NU > 1 ? 1 : 0] : 0u, NU > 2 ? w4[NU > 2 ? 2 : 0] : 0u, NU > 2 ? w4[NU > 2 ? 3 : 0] : 0u),
                       qpar, d);
          each<NU>([&](auto u_) {
            constexpr int u = decltype(u_)::value;
            floatx4_t x = {0.f, 0.f, 0.f, 0.f};
            const uint4 w = codes_bf16(*reinterpret_cast<const uint32_t*>(k_lds + t * 16 * SG::kRowLds + 16 * u), cm, ce);
#pragma unroll
            for (int part = 2; part >= 0; --part) x = mma_bf16(w, qf[u][part], x);
            each<4>([&](auto i_) {
              constexpr int i2 = decltype(i_)::value, at = (4 * t + i2) * NU + u;
              d[i2] = fmaf(row_lane<at % 16>(kstep[at / 16]), x[i2], d[i2]);
            });
          });
        }
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) sc[4 * t + i2] = d[i2];
      });
      uint32_t live = 0xff;                             // keys of this lane that exist
      if (!whole) {
        asm volatile("");                               // a branch: most items skip this
        const int here = (g < 2 ? it.id0 : it.id1) >= 0 ? max(0, min(8, nv - 8 * g)) : 0;
        live = (1u << here) - 1u;
#pragma unroll
        for (int j = 0; j < 8; ++j) sc[j] = (live >> j & 1u) ? sc[j] : -INFINITY;
      }
      // --- running softmax ---
      float mx = fmaxf(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])), fmaxf(fmaxf(sc[4], sc[5]), fmaxf(sc[6], sc[7])));
      mx = xor32_max(xor16_max(mx));
      const float mn = fmaxf(m, mx);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      const float top = mn == -INFINITY ? 0.f : mn;       // scores that overflowed have no weight
      float p[8], sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = __builtin_amdgcn_exp2f(sc[j] - top);        // 0 for a key that does not exist
        sum += p[j];
      }
      // --- weights times V ---
      // 128 dimensions in 4 bits: a group's sums are taken over before the next
      // group's are made (the registers of all of them do not fit two waves)
      constexpr bool kByGroup = CT == CT_INT4 && DH >= 128;
      constexpr int NG = NT / NU;
      floatx4_t o[kByGroup ? NG : NT];
      float om[NU];
      if constexpr (CT == CT_F32) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          floatx4_t x[2];
          x[0] = *reinterpret_cast<const floatx4_t*>(v_lds + t * 16 * SG::kSegLds);
          x[1] = *reinterpret_cast<const floatx4_t*>(v_lds + t * 16 * SG::kSegLds + 16);
          if (!whole) {                                   // what lies behind the sequence's end may be anything
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j >> 2][j & 3] = (live >> j & 1u) ? x[j >> 2][j & 3] : 0.f;
          }
          o[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 8; ++j) o[t] = mma_f32(x[j >> 2][j & 3], p[j], o[t]);
        }
      } else if constexpr (CT == CT_BF16) {
        uint4 mk = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (!whole) {
          auto two = [&](int j) { return ((live >> j & 1u) ? 0xffffu : 0u) | ((live >> (j + 1) & 1u) ? 0xffff0000u : 0u); };
          mk = make_uint4(two(0), two(2), two(4), two(6));
        }
        uint4 hi, lo, lo2;
        split8(p, hi, lo, lo2);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          uint4 x = *reinterpret_cast<const uint4*>(v_lds + t * 16 * SG::kSegLds);
          if (!whole) x = make_uint4(x.x & mk.x, x.y & mk.y, x.z & mk.z, x.w & mk.w);
          o[t] = mma_bf16(x, lo2, floatx4_t{0.f, 0.f, 0.f, 0.f});
          o[t] = mma_bf16(x, lo, o[t]);
          o[t] = mma_bf16(x, hi, o[t]);
        }
      } else {
        const uint4 off = make_uint4(kMinusMid2, kMinusMid2, kMinusMid2, kMinusMid2);
        float vstep[NW], vmid[NW];                        // a group's step and the middle of its range
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          if (!whole) {                                   // what lies behind the sequence's end may be anything
            const int key = (16 * w + (NU >= 2 ? n : n & 7)) / NU;
            vp[w] = (live >> key & 1u) ? vp[w] : 0u;
          }
          vstep[w] = __uint_as_float(vp[w] << 16);
          vmid[w] = fmaf(kCodeMid, vstep[w], __uint_as_float(vp[w] & 0xffff0000u));
        }
        each<NU>([&](auto u_) {
          constexpr int u = decltype(u_)::value;
          float r[8];
          om[u] = 0.f;
          each<8>([&](auto j_) {
            constexpr int j = decltype(j_)::value, at = j * NU + u;
            r[j] = row_lane<at % 16>(vstep[at / 16]) * p[j];
            om[u] = fmaf(row_lane<at % 16>(vmid[at / 16]), p[j], om[u]);
          });
          const uint4 hi = pack8(r);
          take_off(r, hi);
          const uint4 lo = pack8(r);
          take_off(r, lo);
          const uint4 lo2 = pack8(r);
          floatx4_t base = mma_bf16(off, lo2, floatx4_t{0.f, 0.f, 0.f, 0.f});
          base = mma_bf16(off, lo, base);
          base = mma_bf16(off, hi, base);
          constexpr int o0 = kByGroup ? 0 : u * NG;
#pragma unroll
          for (int t = 0; t < NG; ++t) {
            const uint4 w = codes_bf16(*reinterpret_cast<const uint32_t*>(v_lds + (u * NG + t) * 16 * SG::kSegLds), cm, ce);
            o[o0 + t] = mma_bf16(w, hi, base);
            o[o0 + t] = mma_bf16(w, lo, o[o0 + t]);
            o[o0 + t] = mma_bf16(w, lo2, o[o0 + t]);
          }
          if constexpr (kByGroup) {
            if (own) {
#pragma unroll
              for (int t = 0; t < NG; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[u * NG + t][e] = fmaf(acc[u * NG + t][e], f, o[t][e]);
            }
          }
        });
      }
      if (own) {
        l = fmaf(l, f, sum);
        m = mn;
        if constexpr (CT == CT_INT4) {
#pragma unroll
          for (int u = 0; u < NU; ++u) mid[u] = fmaf(mid[u], f, om[u]);
        }
        if constexpr (!kByGroup) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(acc[t][e], f, o[t][e]);
        }
      }
    }
  }

  // --- the waves' parts ---
  l = xor32_sum(xor16_sum(l));
  if constexpr (CT == CT_INT4) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const float x = xor32_sum(xor16_sum(mid[u]));
#pragma unroll
      for (int t = u * (NT / NU); t < (u + 1) * (NT / NU); ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] += x;
    }
  }
  wave_lds_sync();                                    // the wave is done with its last item
  if (g == 0) {
    s_m[wave][n] = m;
    s_l[wave][n] = l;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) *reinterpret_cast<floatx4_t*>(&my.out[n][16 * t + 4 * g]) = acc[t];
  __syncthreads();
  const int rows = beams * G;
  const int parts = a.n_seqs * a.heads;
  for (int i = threadIdx.x; i < rows * (DH / 4); i += kThreads) {
    const int r = i / (DH / 4), d = 4 * (i - r * (DH / 4));
    float mt = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mt = fmaxf(mt, s_m[w][r]);
    float lt = 0.f;
    floatx4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = s_m[w][r] == -INFINITY && !(s_l[w][r] != 0.f) ? 0.f : __builtin_amdgcn_exp2f(s_m[w][r] - mt);
      lt = fmaf(s_l[w][r], f, lt);
      const floatx4_t x = *reinterpret_cast<const floatx4_t*>(&s_wave[w].out[r][d]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], f, o[e]);
    }
    const int s = seq0 + r / G, h = kv * G + r % G;
    if (pl.splits == 1) {
      store_out(a, s, h, d, o, lt);
    } else {
      const size_t part = static_cast<size_t>(split) * parts + static_cast<size_t>(s) * a.heads + h;
      float* base = reinterpret_cast<float*>(a.ws);
      *reinterpret_cast<floatx4_t*>(base + part * DH + d) = o;
      if (d == 0) reinterpret_cast<float2*>(base + static_cast<size_t>(pl.splits) * parts * DH)[part] = make_float2(mt, lt);
    }
  }
}

// The parts of a row's keys: a workgroup per row, DH / 4 lanes for each
// kJoinThreads / (DH / 4)-th of the parts, then those sums in order.  4 .. 5 us: a
// launch and two rounds of loads.
constexpr int kJoinThreads = 256;

template <int DH>
__global__ __launch_bounds__(kJoinThreads) void k_join(AttendArgs a, int splits) {
  constexpr int L = DH / 4, Z = kJoinThreads / L;
  const size_t row = blockIdx.x, parts = static_cast<size_t>(a.n_seqs) * a.heads;
  const int dl = threadIdx.x % L, zl = threadIdx.x / L;
  const float* base = reinterpret_cast<const float*>(a.ws);
  const float2* ml = reinterpret_cast<const float2*>(base + splits * parts * DH);
  __shared__ float s_m[kJoinThreads], s_l[Z];
  __shared__ floatx4_t s_o[Z][L];
  float mt = -INFINITY;
  for (int z = threadIdx.x; z < splits; z += kJoinThreads) mt = fmaxf(mt, ml[z * parts + row].x);
  mt = wave_max(mt);
  if ((threadIdx.x & (kWave - 1)) == 0) s_m[threadIdx.x / kWave] = mt;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / kWave; ++w) mt = fmaxf(mt, s_m[w]);
  float lt = 0.f;
  floatx4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int z = zl; z < splits; z += Z) {
    const float2 x = ml[z * parts + row];
    const floatx4_t v = *reinterpret_cast<const floatx4_t*>(base + (z * parts + row) * DH + 4 * dl);
    const float f = x.x == -INFINITY && !(x.y != 0.f) ? 0.f : __builtin_amdgcn_exp2f(x.x - mt);
    lt = fmaf(x.y, f, lt);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], f, o[e]);
  }
  s_o[zl][dl] = o;
  if (dl == 0) s_l[zl] = lt;
  __syncthreads();
  if (zl == 0) {
#pragma unroll 4
    for (int i = 1; i < Z; ++i) {
      lt += s_l[i];
      const floatx4_t v = s_o[i][dl];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += v[e];
    }
    store_out(a, static_cast<int>(row / a.heads), static_cast<int>(row % a.heads), 4 * dl, o, lt);
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

namespace {

// Beams per tile: whole beams within 16 query rows.  Parts of the keys: as many
// whole ones as the chip holds workgroups at once, a second round of workgroups
// costing more than it evens out (64 x 4 rows of 4,000 keys, 4 heads of 64: bfloat16
// 94 us with 768 workgroups, 105 with 1,024; 4 bits 64 and 69); but one below
// kSplitUnits units, where joining the parts costs about what the workgroup's longer
// way does (5 rows of 8 heads, bfloat16, one part / parts of a unit and their join:
// 138 keys 9.2 / 9.9 us, 300 12.3 / 11.2, 600 17.9 / 12.4, 1,024 26.3 / 13.1; with the
// host's part of two launches 300 keys 12.2 / 12.7).
constexpr int kCus = 256;
constexpr int kSplitUnits = 4;
Plan plan_attend(const CacheView& c, int n_seqs, int heads, int group, int max_len) {
  Plan p;
  const int G = heads / c.kv_heads;
  p.rows_per_tile = 16 / G < group ? 16 / G : group;
  p.tiles = (group + p.rows_per_tile - 1) / p.rows_per_tile;
  const int units = (max_len + kUnit * kBlock - 1) / (kUnit * kBlock);
  const long long wgs = static_cast<long long>(n_seqs / group) * p.tiles * c.kv_heads;
  const long long want = kCus * waves_per_simd(c.type, c.dh) / wgs;
  p.splits = static_cast<int>(want < units ? want : units);
  if (units < kSplitUnits || p.splits < 1) p.splits = 1;
  return p;
}

template <int CT, int DH>
hipError_t launch_attend_t(const AttendArgs& a, const Plan& p, hipStream_t s) {
  const long long wgs = static_cast<long long>(a.n_seqs / a.group) * p.tiles * a.c.kv_heads * p.splits;
  const dim3 grid(static_cast<unsigned>(wgs)), block(kThreads);
  hipLaunchKernelGGL((k_attend<CT, DH>), grid, block, 0, s, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(k_join<DH>, dim3(a.n_seqs * a.heads), dim3(kJoinThreads), 0, s, a, p.splits);
  return hipGetLastError();
}

template <int CT>
hipError_t launch_attend_ct(const AttendArgs& a, const Plan& p, hipStream_t s) {
  switch (a.c.dh) {
    case 16: return launch_attend_t<CT, 16>(a, p, s);
    case 32: return launch_attend_t<CT, 32>(a, p, s);
    case 64: return launch_attend_t<CT, 64>(a, p, s);
    default: return launch_attend_t<CT, 128>(a, p, s);
  }
}

}  // namespace

size_t attend_workspace(const CacheView& c, int n_seqs, int heads, int group, int max_len) {
  const Plan p = plan_attend(c, n_seqs, heads, group, max_len);
  return p.splits == 1 ? 0 : static_cast<size_t>(p.splits) * n_seqs * heads * (c.dh * 4 + 8);
}

// Parts are made up to kCus * waves_per_simd (at most 4 kCus) workgroups of at
// most 16 rows.
size_t attend_workspace_most(const CacheView& c) { return static_cast<size_t>(4 * kCus) * 16 * (c.dh * 4 + 8); }

hipError_t launch_cache_attend(const AttendArgs& a, hipStream_t s) {
  const Plan p = plan_attend(a.c, a.n_seqs, a.heads, a.group, a.max_len);
  if (a.c.type == CT_F32) return launch_attend_ct<CT_F32>(a, p, s);
  if (a.c.type == CT_BF16) return launch_attend_ct<CT_BF16>(a, p, s);
  return launch_attend_ct<CT_INT4>(a, p, s);
}

hipError_t launch_cache_read(const ReadArgs& a, hipStream_t s) {
  const size_t total = static_cast<size_t>(a.n_seqs) * a.count * a.c.kv_heads * a.c.dh;
  const size_t wgs = (total + 255) / 256;
  hipLaunchKernelGGL(k_read, dim3(static_cast<unsigned>(wgs < 8192 ? wgs : 8192)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace pdec
