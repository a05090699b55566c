// Rows of the 4-bit cache written and read: kept rows of a bf16 cache (the
// compaction of Section 6, with four bits an element) and new tokens' rows are
// quantised into pages, and rows are read back as bf16.  Memory-bound: a row's
// 4 d bytes of K and V and its 9 d / 8 bytes in the cache move once.  839 thousand
// kept rows of 128 elements, 550 MB: compaction 95 us (5.8 TB/s), reading back 83
// (6.6 TB/s, near the copy rate).  An uneven packed batch of 1.45 million, 953 MB:
// compaction 173 us (5.5 TB/s), reading back 143 (6.7).  What bounds compaction is
// instructions: 0.66 issued a cycle and scheduler, the ALU pipe at 54%, DRAM at 67%.
// Single new rows cost more than their bytes: a row's V codes are 16-bit halves of
// words that two rows share, 64 bytes of them in eight sectors, which is the price
// of an order that attention reads without exchanging anything.  65536 rows, 43 MB:
// 17.9 us, where the copy rate would take 6.3.
// Both, of the first, step by step: a warp a row, with two-byte stores, 718 us; a
// warp a whole record of 128 elements 199; half a record (64 registers, 32 warps an
// SM) 191; indexes divided by products 181.
#include <cuda_runtime.h>

#include <cstdint>

#include "q4_common.cuh"

namespace rolekv {
namespace {

constexpr int kThreads = 256;
// Calls of so many rows a sequence go by whole (or half) records; with fewer,
// most lanes of a record's warp would have none.  By rows against by records, us,
// by rows a sequence, 8 heads (records: rows at the start of one, and 5 rows on):
//   d 128, 32 layers of 16 sequences:  1: 3.3, 6.4   4: 6.4, 10 to 12   6: 8.7, 10 to 12   8: 9.9, 10 to 12
//          32 layers of 256:           1: 18, 53     4: 64, 55 to 97    6: 95, 57 to 99    8: 125, 59 to 101
//   d 64,  32 layers of 256:           1: 18, 56     4: 33, 56 to 59    6: 49, 57 to 60    8: 64, 58 to 61
// (one layer of 4 sequences: 2.3 and 3.1 at any of these)
constexpr int kRecordRows = 7;
// In large calls a warp takes kRun items one after another, so that what a unit
// looks up (slots, lengths, the packed rows before it) is looked up once.  One item
// against four, us, by waves of the SMs' 32 warps, 8 heads of 1024 rows: 2.1: 11.0,
// 13.1   4.3: 19.3, 20.5   8.6: 36.5, 34.2   34: 140, 123.  The uneven packed batch
// above, with its reading back: 366, 319 (two: 333, eight: 322).  Reading back has
// less to look up and gains nothing (8.6 waves: 64, 70).
constexpr int kRun = 4;
constexpr int kRunWaves = 6;
// A warp that stores single rows takes so many heads in calls of so many waves.  One
// head against four, us, a row of 8 heads of 128 elements:  0.8 waves: 3.3, 4.1
// 1.7: 4.9, 4.5   3.4: 8.2, 6.6   6.7: 14.7, 10.0 (eight heads: 10.5)   13: 27.7,
// 17.9 (eight: 16.9).
constexpr int kRunHeads = 4;
constexpr int kRunHeadsWaves = 2;

// Loads that skip L1.
__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_stream(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

template <int N>
__device__ __forceinline__ void store_words(uint8_t* p, const uint32_t* w) {
  if constexpr (N == 4)
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if constexpr (N == 4) {
    const uint4 x = load_stream(reinterpret_cast<const uint4*>(p));
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = load_stream(reinterpret_cast<const uint2*>(p));
    w[0] = x.x, w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// The rows that one (layer, sequence, head) writes.
struct StoreUnit {
  int slot, pos, rows, n;       // rows: to write; n: tokens the indexes may name
  int64_t kb, vb, i0;           // element offsets of K and V, and of the indexes
};

// By whole warps; no rows where nothing is written.
__device__ __forceinline__ StoreUnit store_unit(const Q4StoreArgs& a, int l, int s, int h) {
  StoreUnit u{};
  u.slot = q4_slot(a.p, s, a.p.status);
  u.pos = u.slot < 0 ? -1 : a.pos[u.slot];
  if (u.pos < 0) return u;
  if (q4_repeated(a.p, s, u.slot)) {
    if (a.p.status != nullptr) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
    return u;
  }
  int64_t tok0 = 0;
  if (a.keep_idx == nullptr) {
    u.n = a.rows_max;
    u.rows = a.count == nullptr ? a.rows_max : a.count[u.slot];
    u.rows = u.rows < 0 ? 0 : (u.rows < a.rows_max ? u.rows : a.rows_max);
  } else if (a.varlen) {
    tok0 = a.cu_seqlens[s];
    u.n = a.cu_seqlens[s + 1] - a.cu_seqlens[s];
    int part = 0;                                   // (all rows of a head are fewer than 2^31)
    for (int x = threadIdx.x & 31; x < s; x += 32)
      part += static_cast<int>(kept_rows(a.cu_seqlens[x + 1] - a.cu_seqlens[x], a.budget_fx, a.kept_extra));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    u.i0 = (static_cast<int64_t>(l) * a.p.Hkv + h) * a.Ktot + part;
    u.rows = static_cast<int>(kept_rows(u.n, a.budget_fx, a.kept_extra));
  } else {
    u.n = a.n_max;
    u.i0 = ((static_cast<int64_t>(l) * a.p.b + s) * a.p.Hkv + h) * a.K_dense;
    u.rows = a.K_dense;
  }
  u.kb = l * a.k_layer + (a.varlen ? tok0 * a.k_tok : s * a.k_seq) + h * a.k_head;
  u.vb = l * a.v_layer + (a.varlen ? tok0 * a.v_tok : s * a.v_seq) + h * a.v_head;
  return u;
}

// What a warp of a grid works on: item `item` of per_unit of unit (l, s, h), the
// warps of all units one after another (past the last one: l = L).  by_heads: h
// counts heads, or groups of them.
struct WarpItem {
  int l, s, h, item;
};
__device__ __forceinline__ WarpItem warp_item(const PagedArgs& p, const Div32& per_unit, const Div32& by_heads) {
  const int64_t w = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const uint32_t u = w >> 31 == 0 ? static_cast<uint32_t>(w) / per_unit : static_cast<uint32_t>(w / per_unit.d);
  const uint32_t seq = u / by_heads, l = seq / p.by_seqs;
  return {static_cast<int>(l), static_cast<int>(seq - l * p.by_seqs.d), static_cast<int>(u - seq * by_heads.d),
          static_cast<int>(w - static_cast<int64_t>(u) * per_unit.d)};
}

// Four elements of one lane, eight lanes a group: their codes in 16 bits, and
// the group's scale.
__device__ __forceinline__ uint32_t quantise4(uint2 x, uint32_t* scale_bits) {
  uint32_t m = __vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu);
  m = max(m & 0xFFFFu, m >> 16);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const Q4Scale s = q4_scale_of(m);
  *scale_bits = s.bits;
  if (s.inv == 0.f) return 0x8888u;
  const uint32_t c0 = q4_code(__uint_as_float(x.x << 16), s.inv) & 15u;
  const uint32_t c1 = q4_code(__uint_as_float(x.x & 0xFFFF0000u), s.inv) & 15u;
  const uint32_t c2 = q4_code(__uint_as_float(x.y << 16), s.inv) & 15u;
  const uint32_t c3 = q4_code(__uint_as_float(x.y & 0xFFFF0000u), s.inv) & 15u;
  return c0 | (c1 << 4) | (c2 << 8) | (c3 << 12);
}

// A row to d / 4 lanes, four elements each, of N heads.
template <int D, int N>
__global__ void __launch_bounds__(kThreads) q4_store_kernel(const Q4StoreArgs a, const Div32 per_unit,
                                                            const Div32 by_groups) {
  constexpr int kLanes = D / 4;                     // lanes of a row
  const WarpItem it = warp_item(a.p, per_unit, by_groups);
  const int l = it.l, s = it.s, h0 = it.h * N, heads = a.p.Hkv - h0;
  wait_for_previous_kernels();
  if (l >= a.p.L) return;
  const StoreUnit x = store_unit(a, l, s, h0);
  const int lane = threadIdx.x & 31, i = lane % kLanes;
  const int j = it.item * (32 / kLanes) + lane / kLanes;
  const bool there = j < x.rows;
  const int64_t i_head = a.varlen ? a.Ktot : a.K_dense;
  uint2 kv[N], vv[N];
  int32_t idx[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    kv[n] = vv[n] = make_uint2(0, 0);
    idx[n] = -1;
    if (!there || n >= heads) continue;
    if (a.keep_idx == nullptr)
      idx[n] = j;
    else if (in_bounds(x.i0 + n * i_head + j, 1, a.ext_keep, a.p.status))
      idx[n] = a.keep_idx[x.i0 + n * i_head + j];
    if (idx[n] >= x.n) {
      if (a.p.status != nullptr && i == 0) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
      idx[n] = -1;
    }
    const int64_t ko = x.kb + n * a.k_head + idx[n] * a.k_tok + 4 * i;
    const int64_t vo = x.vb + n * a.v_head + idx[n] * a.v_tok + 4 * i;
    if (idx[n] >= 0 && in_bounds(ko, 4, a.ext_k, a.p.status)) kv[n] = *reinterpret_cast<const uint2*>(a.k + ko);
    if (idx[n] >= 0 && in_bounds(vo, 4, a.ext_v, a.p.status)) vv[n] = *reinterpret_cast<const uint2*>(a.v + vo);
  }
  const int64_t row = static_cast<int64_t>(x.pos) + j;
  int64_t rec = there ? q4_record(a.p, x.slot, l, h0, static_cast<int>(row / kQ4Rows)) : -1;
  if (there && rec < 0 && a.p.status != nullptr && i == 0) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
  const int r = static_cast<int>(row % kQ4Rows);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n >= heads) break;
    uint32_t ks, vs;
    const uint32_t kc = quantise4(kv[n], &ks), vc = quantise4(vv[n], &vs);
    if (rec >= 0 && in_bounds(rec, q4_record_bytes(D), a.p.ext_pool, a.p.status)) {
      uint8_t* p = a.p.pool + rec;
      *reinterpret_cast<uint16_t*>(p + q4_k_piece(D, r, 4 * i)) = static_cast<uint16_t>(kc);
      *reinterpret_cast<uint16_t*>(p + q4_v_piece(D, r, 4 * i)) = static_cast<uint16_t>(vc);
      if ((i & 7) == 0) {
        if ((ks == 0x7FC0u || vs == 0x7FC0u) && a.p.status != nullptr) atomicOr(a.p.status, ROLEKV_STATUS_NONFINITE);
        // (an empty slot: K scales of -0)
        *reinterpret_cast<uint16_t*>(p + q4_k_scales(D) + q4_scale(D, r, i >> 3)) =
            static_cast<uint16_t>(idx[n] >= 0 ? ks : 0x8000u);
        *reinterpret_cast<uint16_t*>(p + q4_v_scales(D) + q4_scale(D, r, i >> 3)) = static_cast<uint16_t>(vs);
      }
      rec += static_cast<int64_t>(a.p.recs_per_page.d) * q4_record_bytes(D);   // the next head's
    }
  }
}

// ------------------------------------------------------------ whole records --
//
// A warp to a record.  Lane 4 g + t holds the elements of its own words (see
// q4_format.h): of K, 8 elements of each group of rows g and g + 8; of V, 4 of
// each group of rows 2t, 2t + 1 and 8 + 2t, 9 + 2t.  So the codes are packed
// where they are loaded, the largest of a group is a few shuffles away, and
// every store of codes is 32 consecutive pieces.

// Of N packed maxima (two groups each) of every lane, the largest
// over the N lanes STEP apart: lane i of them gets maxima i.
template <int N, int STEP>
__device__ __forceinline__ uint32_t max_scatter(uint32_t* m, int i) {
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1) {
    const bool upper = (i & n) != 0;
#pragma unroll
    for (int x = 0; x < n; ++x) {
      const uint32_t keep = upper ? m[x + n] : m[x], give = upper ? m[x] : m[x + n];
      m[x] = __vmaxu2(keep, __shfl_xor_sync(0xffffffffu, give, n * STEP));
    }
  }
  return m[0];
}

// The larger halves of two words, side by side.
__device__ __forceinline__ uint32_t halves_max(uint32_t x, uint32_t y) {
  return __vmaxu2(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
}

// Codes of eight elements (pairs of bf16), the first in the low nibble, the
// first four by one scale and the others by another.  The sum with 128 leaves
// floor(x / scale + 1/2) + 8 in its byte 2, alone (its smallest step, 2^-16, and
// the product's rounding are well below the 2^-14 of q4_code).
__device__ __forceinline__ uint32_t pack_codes(const uint32_t* x, const uint32_t* y, float inv_x, float inv_y) {
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t w = e < 4 ? x[e / 2] : y[e / 2 - 2];
    const float v = __uint_as_float((e & 1) ? w & 0xFFFF0000u : w << 16);
    b[e] = __float_as_uint(__fmaf_rn(v, e < 4 ? inv_x : inv_y, 136.5f + 0x1p-14f));
  }
  const uint32_t even = __byte_perm(__byte_perm(b[0], b[2], 0x0062), __byte_perm(b[4], b[6], 0x0062), 0x5410);
  const uint32_t odd = __byte_perm(__byte_perm(b[1], b[3], 0x0062), __byte_perm(b[5], b[7], 0x0062), 0x5410);
  return even + odd * 16u;
}

// The larger |x| of pairs of bf16 (a NaN if either is one).
__device__ __forceinline__ uint32_t abs_max(uint32_t x, uint32_t y) {
  const __nv_bfloat162 m = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&x)),
                                       __habs2(*reinterpret_cast<const __nv_bfloat162*>(&y)));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// Is either half of a packed maximum an infinity or a NaN?
__device__ __forceinline__ bool not_finite(uint32_t m) {
  return (m & 0xFFFFu) >= 0x7F80u || (m >> 16) >= 0x7F80u;
}

// A warp to `run` items of 8 rows of 128 elements or 16 of 64: a half of a record,
// or both.
template <int D>
__global__ void __launch_bounds__(kThreads, 4) q4_store_records_kernel(const Q4StoreArgs a, const Div32 per_unit,
                                                                       const int run) {
  constexpr int J = D / kQ4Group;
  constexpr int H = D == 128 ? 1 : 2;               // halves of a record
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const WarpItem it = warp_item(a.p, per_unit, a.p.by_heads);
  const int l = it.l, s = it.s, h = it.h;
  wait_for_previous_kernels();
  if (l >= a.p.L) return;
  // (a packed batch's short sequences leave most of the longest one's items
  // without rows: these go by the length alone)
  if (a.varlen &&
      (it.item * run - 2) * 8 * H >= kept_rows(a.cu_seqlens[s + 1] - a.cu_seqlens[s], a.budget_fx, a.kept_extra))
    return;
  const StoreUnit x = store_unit(a, l, s, h);
  if (x.rows == 0) return;
  for (int item = it.item * run; item < (it.item + 1) * run; ++item) {
    const int half0 = H == 1 ? item & 1 : 0;        // the first half
    const int64_t rec = x.pos / kQ4Rows + static_cast<int64_t>(H == 1 ? item >> 1 : item);
    const int64_t first = rec * kQ4Rows + half0 * 8 - x.pos;   // row of the unit that is the item's row 0
    if (first >= x.rows) return;
    if (first + 8 * H <= 0) continue;
    const int64_t at = q4_record(a.p, x.slot, l, h, static_cast<int>(rec));
    if (at < 0 || !in_bounds(at, q4_record_bytes(D), a.p.ext_pool, a.p.status)) {
      if (at < 0 && a.p.status != nullptr && lane == 0) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
      continue;
    }
    // lanes 0 .. 8 H - 1: the token of each row; -1 an empty slot, -2 not a row of
    // this call
    int token = -2;
    if (lane < 8 * H && first + lane >= 0 && first + lane < x.rows) {
      const int64_t j = first + lane;
      token = -1;
      if (a.keep_idx == nullptr)
        token = static_cast<int>(j);
      else if (in_bounds(x.i0 + j, 1, a.ext_keep, a.p.status))
        token = max(a.keep_idx[x.i0 + j], -1);
      if (token >= x.n) {
        if (a.p.status != nullptr) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
        token = -1;
      }
    }
    // All loads at once.  Rows without a token read token 0 and count as zeros:
    // their maxima are masked, and a scale of 0 gives every finite element the
    // code 0.
    uint32_t k[H][J][4], v[H][2][J][2];
    int kt[H], vt[H][2];
#pragma unroll
    for (int hf = 0; hf < H; ++hf) {
      kt[hf] = __shfl_sync(0xffffffffu, token, hf * 8 + g);
      const int64_t ko = x.kb + max(kt[hf], 0) * a.k_tok + 8 * t;
      const bool kin = in_bounds(ko, D - 24, a.ext_k, a.p.status);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        uint4 y = make_uint4(0, 0, 0, 0);
        if (kin) y = load_stream(reinterpret_cast<const uint4*>(a.k + ko + 32 * j));
        k[hf][j][0] = y.x, k[hf][j][1] = y.y, k[hf][j][2] = y.z, k[hf][j][3] = y.w;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        vt[hf][i] = __shfl_sync(0xffffffffu, token, hf * 8 + 2 * t + i);
        const int64_t vo = x.vb + max(vt[hf][i], 0) * a.v_tok + 4 * g;
        const bool vin = in_bounds(vo, D - 28, a.ext_v, a.p.status);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          uint2 y = make_uint2(0, 0);
          if (vin) y = load_stream(reinterpret_cast<const uint2*>(a.v + vo + 32 * j));
          v[hf][i][j][0] = y.x, v[hf][i][j][1] = y.y;
        }
      }
    }
    uint8_t* const p = a.p.pool + at;
    bool nonfinite = false;
    {
      // K: maxima of a pair of groups of a row (two pairs, of one row or of two),
      // over the row's four lanes; lanes t and t + 2 work out the scales of pair
      // t mod 2 and hand them round
      uint32_t m[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t* c = H == 1 ? k[0][2 * y + i] : k[H - 1 < y ? H - 1 : y][i];
          w[i] = abs_max(abs_max(c[0], c[1]), abs_max(c[2], c[3]));
        }
        m[y] = halves_max(w[0], w[1]);
        m[y] = __vmaxu2(m[y], __shfl_xor_sync(0xffffffffu, m[y], 2));
      }
      uint32_t mine = max_scatter<2, 1>(m, t & 1);
      const bool odd = __any_sync(0xffffffffu, not_finite(mine));
      const int hm = H == 1 ? 0 : t & 1, jm = H == 1 ? 2 * (t & 1) : 0;
      const int km = H == 1 || hm == 0 ? kt[0] : kt[H - 1];
      mine = km < 0 ? 0u : mine;
      const Q4Scale q0 = q4_scale_of(mine & 0xFFFFu), q1 = q4_scale_of(mine >> 16);
      nonfinite |= not_finite(mine);
      if (km >= -1 && t < 2)                          // (an empty slot: -0)
        *reinterpret_cast<uint32_t*>(p + q4_k_scales(D) + q4_scale(D, (half0 + hm) * 8 + g, jm)) =
            km < 0 ? 0x80008000u : q0.bits | (q1.bits << 16);
#pragma unroll
      for (int hf = 0; hf < H; ++hf) {
        uint32_t w[J];
        float inv[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int owner = H == 1 ? j / 2 : hf;
          inv[j] = __shfl_sync(0xffffffffu, (j & 1) ? q1.inv : q0.inv, (lane & 28) | owner);
          w[j] = pack_codes(k[hf][j], k[hf][j] + 2, inv[j], inv[j]);
        }
        if (odd) {                                    // (0 times an infinity is not 0)
#pragma unroll
          for (int j = 0; j < J; ++j) w[j] = inv[j] == 0.f ? 0x88888888u : w[j];
        }
        if (kt[hf] >= -1) store_words<J>(p + (half0 + hf) * 4 * D + lane * 4 * J, w);
      }
    }
    {
      // V: maxima of group j of rows 2t and 2t + 1 (four, over halves and groups),
      // over the eight lanes g; lanes g and g + 4 work out the scales of number
      // g mod 4
      uint32_t m[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t* c = v[y / J][i][y % J];
          w[i] = abs_max(c[0], c[1]);
        }
        m[y] = halves_max(w[0], w[1]);
        m[y] = __vmaxu2(m[y], __shfl_xor_sync(0xffffffffu, m[y], 16));
      }
      uint32_t mine = max_scatter<4, 4>(m, g & 3);
      const bool odd = __any_sync(0xffffffffu, not_finite(mine));
      const int hm = (g & 3) / J, jm = (g & 3) % J;
      const int t0 = H == 1 || hm == 0 ? vt[0][0] : vt[H - 1][0], t1 = H == 1 || hm == 0 ? vt[0][1] : vt[H - 1][1];
      mine &= (t0 < 0 ? 0u : 0xFFFFu) | (t1 < 0 ? 0u : 0xFFFF0000u);
      const Q4Scale q0 = q4_scale_of(mine & 0xFFFFu), q1 = q4_scale_of(mine >> 16);
      nonfinite |= not_finite(mine);
      uint8_t* const sc = p + q4_v_scales(D) + q4_scale(D, (half0 + hm) * 8 + 2 * t, jm);
      if (g < 4 && t0 >= -1) *reinterpret_cast<uint16_t*>(sc) = static_cast<uint16_t>(q0.bits);
      if (g < 4 && t1 >= -1) *reinterpret_cast<uint16_t*>(sc + 2 * J) = static_cast<uint16_t>(q1.bits);
#pragma unroll
      for (int hf = 0; hf < H; ++hf) {
        uint32_t w[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int from = 4 * (hf * J + j) | t;
          const float inv0 = __shfl_sync(0xffffffffu, q0.inv, from), inv1 = __shfl_sync(0xffffffffu, q1.inv, from);
          w[j] = pack_codes(v[hf][0][j], v[hf][1][j], inv0, inv1);
          if (odd) {
            if (inv0 == 0.f) w[j] = (w[j] & 0xFFFF0000u) | 0x8888u;
            if (inv1 == 0.f) w[j] = (w[j] & 0xFFFFu) | 0x88880000u;
          }
        }
        uint8_t* const y = p + q4_v_codes(D) + (half0 + hf) * 4 * D + lane * 4 * J;
        const bool h0 = vt[hf][0] >= -1, h1 = vt[hf][1] >= -1;
        if (h0 && h1) {
          store_words<J>(y, w);
        } else if (h0 || h1) {                        // the other row of the words is not this call's
#pragma unroll
          for (int j = 0; j < J; ++j)
            *reinterpret_cast<uint16_t*>(y + 4 * j + (h0 ? 0 : 2)) = static_cast<uint16_t>(h0 ? w[j] : w[j] >> 16);
        }
      }
    }
    if (nonfinite && a.p.status != nullptr) atomicOr(a.p.status, ROLEKV_STATUS_NONFINITE);
  }
}

// Codes of two nibbles of a word (bits 0..3 and 16..19) less 8 as bf16 numbers,
// times their scales, each product rounded once to bf16.
__device__ __forceinline__ uint32_t two_values(uint32_t w, uint32_t scales) {
  const uint32_t c = (w & 0x000F000Fu) | 0x43004300u;          // 128 + code
  const uint32_t off = 0xC308C308u;                            // -136
  const __nv_bfloat162 x = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&c),
                                   *reinterpret_cast<const __nv_bfloat162*>(&off));
  const __nv_bfloat162 y = __hmul2(x, *reinterpret_cast<const __nv_bfloat162*>(&scales));
  return *reinterpret_cast<const uint32_t*>(&y);
}

template <int D>
__global__ void __launch_bounds__(kThreads) q4_expand_kernel(const Q4ExpandArgs a, const Div32 per_unit) {
  constexpr int J = D / kQ4Group;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const WarpItem it = warp_item(a.p, per_unit, a.p.by_heads);
  const int l = it.l, s = it.s, h = it.h;
  wait_for_previous_kernels();
  if (l >= a.p.L) return;
  const int slot = q4_slot(a.p, s, a.p.status);
  const int len = q4_len(a.p, slot, a.p.status);
  if (len == 0) return;
  const int start = a.start == nullptr ? 0 : a.start[slot];
  if (start < 0 || start >= len) return;
  const int rows = min(a.rows, len - start);        // to read
  const int rec = start / kQ4Rows + it.item;
  const int first = rec * kQ4Rows - start;          // output row of the record's row 0
  if (first >= rows) return;
  const int64_t at = q4_record(a.p, slot, l, h, rec);
  if (at < 0) {                                     // rows that are absent: nothing to give back
    if (a.p.status != nullptr && lane == 0) atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
    return;
  }
  if (!in_bounds(at, q4_record_bytes(D), a.p.ext_pool, a.p.status)) return;
  const uint8_t* const p = a.p.pool + at;
  uint32_t kw[2][J], vw[2][J], ksc[2][J / 2], vsc[2][J];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    load_words<J>(kw[hf], p + hf * 4 * D + lane * 4 * J);
    load_words<J>(vw[hf], p + q4_v_codes(D) + hf * 4 * D + lane * 4 * J);
    load_words<J / 2>(ksc[hf], p + q4_k_scales(D) + q4_scale(D, hf * 8 + g, 0));
    load_words<J>(vsc[hf], p + q4_v_scales(D) + q4_scale(D, hf * 8 + 2 * t, 0));
  }
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int row = first + hf * 8 + g;
    const int64_t ko = l * a.k_layer + s * a.k_seq + h * a.k_head + static_cast<int64_t>(row) * a.k_tok + 8 * t;
    if (row >= 0 && row < rows && in_bounds(ko, D - 24, a.ext_k, a.p.status)) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t sc = __byte_perm(ksc[hf][j / 2] & 0x7FFF7FFFu, 0, (j & 1) ? 0x3232 : 0x1010);
        uint32_t r[4];                              // elements i and i + 4
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = two_values(kw[hf][j] >> (4 * i), sc);
        *reinterpret_cast<uint4*>(a.k + ko + 32 * j) =
            make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410),
                       __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
      }
    }
    uint2 out[2][J];                                // of rows 2t and 2t + 1
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t sc = __byte_perm(vsc[hf][j / 2], vsc[hf][J / 2 + j / 2], (j & 1) ? 0x7632 : 0x5410);
      uint32_t r[4];                                // element i of both rows
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = two_values(vw[hf][j] >> (4 * i), sc);
      out[0][j] = make_uint2(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410));
      out[1][j] = make_uint2(__byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = first + hf * 8 + 2 * t + i;
      const int64_t vo = l * a.v_layer + s * a.v_seq + h * a.v_head + static_cast<int64_t>(r) * a.v_tok + 4 * g;
      if (r >= 0 && r < rows && in_bounds(vo, D - 28, a.ext_v, a.p.status)) {
#pragma unroll
        for (int j = 0; j < J; ++j) *reinterpret_cast<uint2*>(a.v + vo + 32 * j) = out[i][j];
      }
    }
  }
}

}  // namespace

// Records that rows consecutive rows of a sequence lie in, wherever they begin.
static int records_of(int64_t rows) { return static_cast<int>((rows + kQ4Rows - 2) / kQ4Rows + 1); }

template <class Args, class... More>
static cudaError_t launch_warps(void (*kernel)(Args, Div32, More...), const Args& a, int64_t units, int per_unit,
                                cudaStream_t stream, More... more) {
  const int64_t warps = units * per_unit;
  const unsigned grid = static_cast<unsigned>((warps + kThreads / 32 - 1) / (kThreads / 32));
  return launch_early(kernel, grid, kThreads, 0, stream, 1, a, make_div(static_cast<uint32_t>(per_unit)), more...);
}

// A call of so many waves of warps?
static bool fills(int64_t warps, int waves) { return warps >= int64_t{waves} * 32 * device_sms(); }

cudaError_t launch_q4_store(const Q4StoreArgs& a, cudaStream_t stream) {
  if (a.rows_max == 0) return cudaSuccess;
  const int64_t seqs = static_cast<int64_t>(a.p.L) * a.p.b, units = seqs * a.p.Hkv;
  if (a.rows_max >= kRecordRows) {
    auto* kernel = a.p.d == 128 ? q4_store_records_kernel<128> : q4_store_records_kernel<64>;
    const int items = records_of(a.rows_max) * (a.p.d == 128 ? 2 : 1);
    const int run = fills(units * items, kRunWaves) ? kRun : 1;
    return launch_warps(kernel, a, units, (items + run - 1) / run, stream, run);
  }
  const int items = a.p.d == 128 ? a.rows_max : (a.rows_max + 1) / 2;
  if (fills(units * items, kRunHeadsWaves)) {
    auto* kernel = a.p.d == 128 ? q4_store_kernel<128, kRunHeads> : q4_store_kernel<64, kRunHeads>;
    const int groups = (a.p.Hkv + kRunHeads - 1) / kRunHeads;
    return launch_warps(kernel, a, seqs * groups, items, stream, make_div(static_cast<uint32_t>(groups)));
  }
  auto* kernel = a.p.d == 128 ? q4_store_kernel<128, 1> : q4_store_kernel<64, 1>;
  return launch_warps(kernel, a, units, items, stream, a.p.by_heads);
}

cudaError_t launch_q4_expand(const Q4ExpandArgs& a, cudaStream_t stream) {
  if (a.rows == 0) return cudaSuccess;
  auto* kernel = a.p.d == 128 ? q4_expand_kernel<128> : q4_expand_kernel<64>;
  return launch_warps(kernel, a, static_cast<int64_t>(a.p.L) * a.p.b * a.p.Hkv, records_of(a.rows), stream);
}

}  // namespace rolekv
