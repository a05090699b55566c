// One decode step of attention through a cache of 4-bit rows in pages:
//   out_g = sum_j softmax_j(scale q_g . k_j) v_j
// over the lens[slot] rows of every sequence, for each (layer, sequence, KV
// head) and its G query heads.  Memory-bound: 9 d / 8 bytes a row, read once.
//
// The lengths are on the device alone, so the rows are shared out there: all
// units' pieces (two records, 32 rows) in a row, an equal run of them to each
// CTA.  A run covers whole units, whose outputs the CTA writes, and at its ends
// parts of units, whose sums go to the workspace (two at most a CTA) for a
// second launch to join.  In a CTA each of four warps takes every fourth piece,
// from a ring of its own, and no warp waits for another until a unit ends.  A
// fifth warp looks the pieces up, 32 at a time, and keeps the rings full: a bulk
// copy a piece (two where its records lie in different pages).
//
// Products (m16n8k16, fp16 operands, fp32 sums; the codes' order in a record
// is the operands' order in registers, see q4_format.h).  A code becomes an
// operand in two steps: a mask that also sets the exponent gives 1024 + code
// (nibbles 0, 4 of a word) or 1024 + 16 code (nibbles 1, 5), and an fp16 addition
// takes the 1024 and the offset of 8 off, exactly (a published way to turn whole
// numbers into floating point; the factor of 16 goes into q and the outputs).  (Left as subnormal numbers,
// code * 2^-24, they would cost the mask alone, but the tensor cores align a
// product's bits by its operands' exponents, and sums came out with 17 bits.)
//   S = K Q^T   16 rows x heads.  q is scaled by a power of two to below 2^15,
//     and then is exact in fp16 (elements below 2^-25 of a head's largest lose
//     bits, 2^-39 of it at most), and by 2^-4 where codes come times 16.  Each
//     group's sum is scaled in fp32, q's power of two still on: a row's sum stays
//     below 7 * 128 * 2^15 scales, within fp32 for scales below 2^103, keys below
//     2^105.  (As Q K^T the logits would come out in the layout that the next
//     product wants, but half of its rows, and of the registers that hold q,
//     would be zeros.)
//   O = V^T P   16 elements x heads over 16 rows.  The probabilities change
//     places through shared memory; a row's times its V scale is a lane's own
//     value.  It goes in as two fp16 numbers, the upper bits and the rest, so
//     that 22 bits count.  The probabilities are taken times a power of two, by
//     the largest V scale so far, which keeps the numbers below 2^15 and the
//     largest above 2^10, so that fp16's smallest step is 2^-34 of the largest at
//     most.  The power is no part of the softmax's reference (which would save
//     the product, 1% of the time): beside large logits fp32 has no room for it,
//     and the probabilities' sums would span more powers of two than fp32 has.
//     A warp's sums leave it as means, the power taken off.
// What bounds it is issue that stalls: some 390 instructions a record and warp, of
// which about 145 make operands of codes, at 0.61 a cycle and scheduler, with no
// pipe above half (ALU 46%, FMA 40%, tensor 30%, DRAM 49%).  Without a gap they
// would take 81 us of an uneven batch's 158 (600 MB, 3.8 TB/s; its bytes alone 88).
// A scheduler's three warps wait for results of fixed latency (1.4 cycles an
// instruction), for one another (0.85) and for bursts on the math pipes (0.7), and
// hardly for copies (0.5).  131072 rows of 8 heads, 151 MB: 45 us, 3.4 TB/s.  (All
// of a piece's work but one read left out, the batch took 106 us of the 152 before
// records were summed apart; the copies left out instead, 147 of 160 before there
// was a fifth warp.)  Three CTAs an SM at 128 registers a thread; two take 224 us.
// Records one by one, which fit four, took 162 where two by two took 157.
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "q4_common.cuh"

namespace rolekv {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kBlock = kThreads + 32;   // and the warp that feeds them
constexpr int kJoinWarps = 16;      // of a CTA that joins the parts of a unit
constexpr int kHeads = 8;           // columns of the products: query heads of a KV head
constexpr int kRecs = 2;            // records of a piece
constexpr int kPieceRows = kRecs * kQ4Rows;
constexpr int kSlack = 4;           // powers of two a logit may pass the largest so far by before the sums are rescaled
constexpr int kMaxRoom = 96;        // of the power of two that probabilities are taken times
constexpr int kTurn = 12;           // floats of a row of probabilities (eight, and room against bank conflicts)

// How the rows are shared: an even run of pieces to each CTA, with what is to
// join listed by CTA or, for few units of many parts, by unit; or a unit to each.
enum { kShared = 0, kFewUnits = 1, kOneUnit = 2 };
// Units of so many pieces at most go to a CTA each: no parts, no second launch.
// Shared against whole, us, by rows of a unit of 8 heads:  128: 7.1, 5.6   256:
// 8.4, 6.6   384: 8.6, 7.4   512: 8.6, 8.4 (2 units);  128: 9.1, 6.4   256: 11.0,
// 7.8   384: 15.3, 9.2   512: 17.7, 10.5 (256);  128: 51, 60   256: 73, 78   384:
// 89, 94 (512 sequences);  128: 294, 245   256: 388, 304   384: 479, 363 (2048
// sequences);  128: 183, 240   256: 247, 301   384: 312, 360 (64 sequences of 32
// layers, where whole units cost a quarter).
constexpr int kWholePieces = 12;

template <int D>
struct Shape {
  static constexpr int kGroups = D / kQ4Group;
  static constexpr int kRecord = 18 * D;
  static constexpr int kPiece = kRecs * kRecord;
  static constexpr int kStages = D == 128 ? 3 : 6;        // pieces a warp has in flight
  // dynamic shared memory: a part for each warp, the warps' sums of four heads
  // at a time, the batch's lengths
  static constexpr int kRing = 0;
  static constexpr int kTurnAt = kRing + kStages * kPiece;    // probabilities, row by row
  static constexpr int kFull = kTurnAt + kPieceRows * kTurn * 4;  // a stage has landed
  static constexpr int kEmpty = kFull + 64;               // has been read
  static constexpr int kRows = kEmpty + 64;               // rows in use of its records (eight bits each)
  static constexpr int kWarp = kRows + 64;
  static constexpr int kHead = D + 4;                     // floats of a head's sums
  static constexpr int kSums = kWarps * kWarp;
  static constexpr int kLens = kSums + kWarps * 4 * kHead * 4;
};

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, const float* c) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
      "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Two numbers below 65504 as fp16, cut to its eleven bits, and what that leaves
// of them.
__device__ __forceinline__ void split_half2(float x, float y, uint32_t* upper, uint32_t* rest) {
  uint32_t h;
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(y), "f"(x));
  float dx, dy;                                     // x - h and y - h, exactly
  asm("{\n\t.reg .b16 lo, hi, minus;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "mov.b16 minus, 0xBC00;\n\t"                 // -1
      "fma.rn.f32.f16 %0, lo, minus, %3;\n\t"
      "fma.rn.f32.f16 %1, hi, minus, %4;\n\t}"
      : "=f"(dx), "=f"(dy)
      : "r"(h), "f"(x), "f"(y));
  *upper = h;
  *rest = pack_half2(dx, dy);
}

// Two fp16 sums.
__device__ __forceinline__ uint32_t add_half2(uint32_t x, uint32_t y) {
  const __half2 h = __hadd2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&y));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// x & y | z.  (Written out with two constants, it takes two instructions.)
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t y, uint32_t z) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(y), "r"(z));
  return r;
}

// Codes without their offset of 8 as fp16 numbers: nibbles 0 and 4 of a word,
// and nibbles 1 and 5 times 16.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) {
  return add_half2(and_or(w, 0x000F000Fu, 0x64006400u), 0xE408E408u);   // -1032
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w) {
  return add_half2(and_or(w, 0x00F000F0u, 0x64006400u), 0xE480E480u);   // -1152
}

// 1 / x, off by 2^-23 of it.
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// N 32-bit words of shared memory.
template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if constexpr (N == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x, w[1] = x.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Where the pieces of a call lie: all (layer, sequence, head) units one after
// another, a unit's pieces in order.
struct Span {
  const int32_t* cum;             // [b + 1] pieces of a head of the sequences before
  int64_t per_layer;              // pieces of a layer
  int32_t b, Hkv;
};

struct Place {
  int l, s, h, piece;             // piece: of the unit
  int64_t start, end;             // the unit's pieces
};

// x / y and the remainder, in 32 bits where they hold x (a 64-bit division
// takes some 80 instructions).
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y, int64_t* rest) {
  if (((x | y) >> 32) == 0) {
    const uint32_t q = static_cast<uint32_t>(x) / static_cast<uint32_t>(y);
    *rest = static_cast<uint32_t>(x) - q * static_cast<uint32_t>(y);
    return q;
  }
  const int64_t q = x / y;
  *rest = x - q * y;
  return q;
}

__device__ __forceinline__ Place place_of(const Span& sp, int64_t x) {
  Place p;
  int64_t r, rest;
  p.l = static_cast<int>(divide(x, sp.per_layer, &r));
  const int key = static_cast<int>(divide(r, sp.Hkv, &rest));
  int lo = 0, hi = sp.b - 1;                        // the last sequence that begins at or before key
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sp.cum[mid] <= key)
      lo = mid;
    else
      hi = mid - 1;
  }
  p.s = lo;
  const int n = sp.cum[lo + 1] - sp.cum[lo];
  p.h = static_cast<int>(divide(r - static_cast<int64_t>(sp.Hkv) * sp.cum[lo], n, &rest));
  p.piece = static_cast<int>(rest);
  p.start = x - p.piece;
  p.end = p.start + n;
  return p;
}

// The unit behind p (there is one).
__device__ __forceinline__ void next_unit(const Span& sp, Place* p) {
  if (++p->h == sp.Hkv) {
    p->h = 0;
    do {
      if (++p->s == sp.b) {
        p->s = 0;
        ++p->l;
      }
    } while (sp.cum[p->s] == sp.cum[p->s + 1]);
  }
  p->start = p->end;
  p->end += sp.cum[p->s + 1] - sp.cum[p->s];
}

// The four warps of a CTA that work on the rows meet.
__device__ __forceinline__ void sync_consumers() {
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
}
// After a wait has run out, how long copies in flight are given to land.
constexpr uint64_t kDrainNs = 50000000ull;

// What they work on: kept in shared memory, out of the way of the loop over the
// rows.
struct Work {
  Place unit;
  int64_t x, end;                 // its pieces in this CTA's run
};

__device__ __forceinline__ int4* join_of(const Q4DecodeArgs& a) {
  return reinterpret_cast<int4*>(a.part + static_cast<int64_t>(2) * a.ctas * a.G * (a.p.d + 2));
}

template <int D>
__global__ void __launch_bounds__(kBlock, kQ4DecodeCtasPerSm) q4_decode_kernel(const Q4DecodeArgs a, int share) {
  using Sh = Shape<D>;
  constexpr int J = Sh::kGroups, REC = Sh::kRecord, PIECE = Sh::kPiece, S = Sh::kStages, HEAD = Sh::kHead;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_flag;
  __shared__ float2 stat[kWarps][kHeads];               // a warp's reference and sum per head
  __shared__ int scan[kWarps];
  __shared__ Work work;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  uint8_t* const mine = smem + (warp < kWarps ? warp : 0) * Sh::kWarp;
  uint64_t* const full = reinterpret_cast<uint64_t*>(mine + Sh::kFull);
  float* sums = reinterpret_cast<float*>(smem + Sh::kSums);
  int32_t* cum = reinterpret_cast<int32_t*>(smem + Sh::kLens);
  if (lane == 0 && warp < kWarps) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&full[i] + (Sh::kEmpty - Sh::kFull) / 8, 1);
    }
    fence_mbar_init();
  }
  if (threadIdx.x == 0) abort_flag = 0;
  wait_for_previous_kernels();

  const bool one = share == kOneUnit;               // unit blockIdx.x, whole
  const uint32_t seq = blockIdx.x / a.p.by_heads, layer = seq / a.p.by_seqs;
  const int h1 = static_cast<int>(blockIdx.x - seq * a.p.by_heads.d), s1 = static_cast<int>(seq - layer * a.p.by_seqs.d),
            l1 = static_cast<int>(layer);
  const auto pieces_of = [&](int s, int32_t* report) {
    return (q4_len(a.p, q4_slot(a.p, s, report), report) + kPieceRows - 1) / kPieceRows;
  };
  // The pieces before each sequence: a warp sums a quarter of the sequences, and
  // adds what the warps before it found.
  if (threadIdx.x == 0) cum[0] = 0;
  if (one) {
    if (threadIdx.x == 0) cum[1] = pieces_of(s1, a.p.status);
    __syncthreads();
  } else {
    int32_t* const report = blockIdx.x == 0 ? a.p.status : nullptr;
    const int quarter = ((a.p.b + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int from = warp * quarter, to = warp < kWarps ? (from + quarter < a.p.b ? from + quarter : a.p.b) : 0;
    int sum = 0;
#pragma unroll 4
    for (int s0 = from; s0 < to; s0 += 32) {
      int n = s0 + lane < to ? pieces_of(s0 + lane, report) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, n, o);
        if (lane >= o) n += y;
      }
      if (s0 + lane < to) cum[s0 + lane + 1] = sum + n;
      sum += __shfl_sync(0xffffffffu, n, 31);
    }
    if (lane == 0 && warp < kWarps) scan[warp] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp && w < kWarps; ++w) before += scan[w];
    for (int s = from + lane; s < to; s += 32) cum[s + 1] += before;
    __syncthreads();
  }
  const auto span = [&] {
    return one ? Span{cum, cum[1], 1, 1} : Span{cum, static_cast<int64_t>(a.p.Hkv) * cum[a.p.b], a.p.b, a.p.Hkv};
  };
  const auto place = [&](int64_t x) {
    Place p = place_of(span(), x);
    if (one) p.l = l1, p.s = s1, p.h = h1;
    return p;
  };
  const int64_t all = span().per_layer * (one ? 1 : a.p.L);
  int64_t rest_;
  const int64_t run = one ? all : (divide(all + gridDim.x - 1, gridDim.x, &rest_) + kWarps - 1) / kWarps * kWarps;
  const int64_t x0 = one ? 0 : blockIdx.x * run, x1 = x0 + run < all ? x0 + run : all;
  const int G = a.G;
  const bool few = share == kFewUnits;

  // sequences without a row: zeros
  if (one) {
    if (x1 == 0) {
      for (int i = threadIdx.x; i < G * D; i += kBlock) a.out[static_cast<int64_t>(blockIdx.x) * G * D + i] = 0.f;
      return;
    }
  } else {
    for (int s = blockIdx.x; s < a.p.b; s += gridDim.x)
      if (cum[s] == cum[s + 1])
        for (int l = 0; l < a.p.L; ++l) {
          const int64_t unit = (static_cast<int64_t>(l) * a.p.b + s) * a.p.Hkv;
          for (int i = threadIdx.x; i < a.p.Hkv * G * D; i += kBlock) a.out[unit * G * D + i] = 0.f;
          for (int h = threadIdx.x; few && h < a.p.Hkv; h += kBlock) join_of(a)[unit + h] = make_int4(-1, 0, 0, 0);
        }
  }
  // What to join: by the CTA that begins a cut unit, or, with few units, by unit.
  int4* join = join_of(a);
  if (x0 >= x1) {
    if (threadIdx.x == 0 && share == kShared) join[blockIdx.x] = make_int4(-1, 0, 0, 0);
    return;
  }

  if (warp == kWarps) {
    // ------------------------------------------------------------- feeding --
    // Piece k of the run goes to warp k mod 4.  A lane looks up one of 32: where
    // its records would lie in page 0, and their pages, whose loads are not
    // waited for until the 32 before them are on their way.
    struct Look {
      int64_t base[kRecs];
      int32_t page[kRecs];
      int rows;
    };
    const int total = static_cast<int>(x1 - x0), recs_per_page = a.p.page_rows / kQ4Rows;
    const auto look_up = [&](int k) {
      Look y;
      y.rows = 0;
      if (k >= total) return y;
      const Place p = place(x0 + k);
      const int slot = q4_slot(a.p, p.s, nullptr), len = q4_len(a.p, slot, nullptr);
      const int32_t* row = a.p.table + static_cast<int64_t>(slot) * a.p.max_pages;
#pragma unroll
      for (int r = 0; r < kRecs; ++r) {
        const int left = len - p.piece * kPieceRows - r * kQ4Rows;
        const int rec = p.piece * kRecs + r, col = static_cast<int>(static_cast<uint32_t>(rec) / a.p.recs_per_page);
        y.base[r] = p.l * a.p.s_layer +
                    (static_cast<int64_t>(p.h) * recs_per_page + (rec - col * recs_per_page)) * static_cast<int64_t>(REC);
        y.page[r] = left > 0 ? row[col] : -2;       // (rows in use lie within the table)
        y.rows |= (left < 0 ? 0 : (left < kQ4Rows ? left : kQ4Rows)) << (8 * r);
      }
      return y;
    };
    bool dead = false;
    Look next = look_up(lane);
    for (int k0 = 0; k0 < total && !dead; k0 += 32) {
      const Look y = next;
      next = look_up(k0 + 32 + lane);
      int64_t at[kRecs];
      int rows = 0;
#pragma unroll
      for (int r = 0; r < kRecs; ++r) {
        at[r] = -1;
        if (k0 + lane >= total || y.page[r] == -2) continue;
        if (y.page[r] >= 0 && y.page[r] < a.p.n_pages) {
          at[r] = y.base[r] + y.page[r] * a.p.s_page;
          if (!in_bounds(at[r], REC, a.p.ext_pool, a.p.status)) at[r] = -1;
        } else if (a.p.status != nullptr) {
          atomicOr(a.p.status, ROLEKV_STATUS_BAD_INDEX);
        }
        if (at[r] >= 0) rows |= y.rows & (255 << (8 * r));
      }
      for (int i = 0; i < 32 && k0 + i < total && !dead; ++i) {
        if (lane == i) {
          const int k = k0 + i, n = k / kWarps, stage = n % S;
          uint8_t* const to = smem + (k % kWarps) * Sh::kWarp;
          uint64_t* const bar = reinterpret_cast<uint64_t*>(to + Sh::kFull) + stage;
          dead = n >= S && !mbar_wait(bar + (Sh::kEmpty - Sh::kFull) / 8, (n / S - 1) & 1, &abort_flag, a.p.status);
          if (!dead) {
            reinterpret_cast<int*>(to + Sh::kRows)[stage] = rows;
            uint8_t* const ring = to + Sh::kRing + stage * PIECE;
            if (at[0] >= 0 && at[1] == at[0] + REC) {
              mbar_arrive_expect_tx(bar, PIECE);
              bulk_copy_g2s(ring, a.p.pool + at[0], PIECE, bar);
            } else {
              mbar_arrive_expect_tx(bar, (at[0] >= 0 ? REC : 0) + (at[1] >= 0 ? REC : 0));
              if (at[0] >= 0) bulk_copy_g2s(ring, a.p.pool + at[0], REC, bar);
              if (at[1] >= 0) bulk_copy_g2s(ring + REC, a.p.pool + at[1], REC, bar);
            }
          }
        }
        dead = __any_sync(0xffffffffu, dead);
      }
    }
    // (a wait that ran out: the copies still in flight land before the CTA leaves)
    if (dead && lane < kWarps * S) {
      uint64_t* const bar =
          reinterpret_cast<uint64_t*>(smem + (lane / S) * Sh::kWarp + Sh::kFull) + lane % S;
      mbar_wait_for(bar, 0, nullptr, nullptr, kDrainNs);
      mbar_wait_for(bar, 1, nullptr, nullptr, kDrainNs);
    }
    return;
  }

  bool alive = true;
  int n = 0;                                        // pieces this warp has done
  int stage = 0;                                    // n mod S
  uint32_t phase = 0;                               // n / S mod 2
  const int count = static_cast<int>((x1 - x0 - warp + kWarps - 1) / kWarps);
  if (threadIdx.x == 0) {
    work.unit = place(x0);
    work.x = x0;
    work.end = work.unit.end < x1 ? work.unit.end : x1;
  }
  sync_consumers();
  for (;;) {
    // ------------------------------------------------------------ queries --
    // lane (g, t): head g (zeros past G), elements 32 j + 8 t + 0..7
    uint32_t qb[J][4];
    float logit0, logit1;                           // the logits' scale of heads 2t and 2t + 1
    {
      uint32_t raw[J][4];
      const int64_t q0 = work.unit.l * a.q_layer + work.unit.s * a.q_seq +
                         static_cast<int64_t>(work.unit.h * G + g) * a.q_head + 8 * t;
      const bool have = g < G && in_bounds(q0, D - 24, a.ext_q, a.p.status);
      const uint4* qp = reinterpret_cast<const uint4*>(a.q + (have ? q0 : 0));
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint4 w = have ? qp[4 * j] : make_uint4(0, 0, 0, 0);
        raw[j][0] = w.x, raw[j][1] = w.y, raw[j][2] = w.z, raw[j][3] = w.w;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __vmaxu2(m, raw[j][i] & 0x7FFF7FFFu);
      }
      m = max(m & 0xFFFFu, m >> 16);
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
      int k = 14 + 127 - static_cast<int>(m >> 7);  // largest element in [2^14, 2^15)
      k = k > 126 ? 126 : k;
      // (a query that is not finite reaches the rows that there are, and gives NaN
      // if there are any: it is taken as zeros and marked by the sign)
      const bool finite = m < 0x7F80u;
      const float up = pow2(k), logit = finite ? a.c1 * pow2(-k) : -0.f;
      logit0 = __shfl_sync(0xffffffffu, logit, 8 * t);
      logit1 = __shfl_sync(0xffffffffu, logit, 8 * t + 4);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!finite) raw[j][i] = 0u;
          e[2 * i] = __uint_as_float(raw[j][i] << 16) * up;
          e[2 * i + 1] = __uint_as_float(raw[j][i] & 0xFFFF0000u) * up;
        }
        qb[j][0] = pack_half2(e[0], e[4]);
        qb[j][1] = pack_half2(e[1] * 0.0625f, e[5] * 0.0625f);
        qb[j][2] = pack_half2(e[2], e[6]);
        qb[j][3] = pack_half2(e[3] * 0.0625f, e[7] * 0.0625f);
      }
    }
    // heads 2t and 2t + 1: reference (a logit, kSlack below the largest at most),
    // sum over this lane's rows
    float ref[2] = {-FLT_MAX, -FLT_MAX}, den[2] = {0.f, 0.f};
    uint32_t top_scale = 0;                         // what a V scale may reach (bf16 bits, twice; all lanes)
    float room = pow2(kMaxRoom);                    // the power of two that probabilities are taken times
    float acc[2 * J][4];
#pragma unroll
    for (int i = 0; i < 2 * J; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
    // this lane's words of a record, from its start
    const uint8_t *codes = mine + lane * 4 * J, *k_scales = mine + 16 * D + g * 2 * J,
                  *v_scales = mine + 17 * D + t * 4 * J;
    float* const turn = reinterpret_cast<float*>(mine + Sh::kTurnAt);
    float* const turn_to = turn + g * kTurn + 2 * t;
    const float* const turn_from = turn + 2 * t * kTurn + g;
    const int n_end = work.end == x1 ? count : static_cast<int>((work.end - x0 - warp + kWarps - 1) / kWarps);

    // One piece: kPart if its records may hold fewer than 16 rows (eight bits of
    // `both` each).
    const auto piece = [&](auto part_, uint32_t from, int both) {
      constexpr bool kPart = decltype(part_)::value;
      // ----------------------------------------------------------- logits --
      // x: row g, heads 2t and 2t + 1; row g + 8, the same
      float x[kRecs][4];
#pragma unroll
      for (int r = 0; r < kRecs; ++r) {
        uint32_t kw[2][J], ksc[2][J / 2];           // codes; scales of rows g and g + 8
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          load_words<J>(kw[hf], codes + from + r * REC + hf * 4 * D);
          load_words<J / 2>(ksc[hf], k_scales + from + r * REC + hf * (D / 2));
          if (kPart && hf * 8 + g >= ((both >> (8 * r)) & 255)) {   // rows past the end hold anything:
#pragma unroll
            for (int k = 0; k < J / 2; ++k) ksc[hf][k] = k == 0 ? 0x8000u : 0u;   // taken as empty slots
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[r][i] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint32_t w0 = kw[0][j], w1 = kw[1][j], w08 = w0 >> 8, w18 = w1 >> 8;
          const uint32_t a0[4] = {low_codes(w0), low_codes(w1), high_codes(w0), high_codes(w1)};
          const uint32_t a1[4] = {low_codes(w08), low_codes(w18), high_codes(w08), high_codes(w18)};
          float c[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(c, a0, qb[j][0], qb[j][1], c);
          mma_f16(c, a1, qb[j][2], qb[j][3], c);
          const uint32_t u0 = ksc[0][j / 2], u1 = ksc[1][j / 2];
          const float s0 = __uint_as_float((j & 1) ? u0 & 0xFFFF0000u : u0 << 16);
          const float s1 = __uint_as_float((j & 1) ? u1 & 0xFFFF0000u : u1 << 16);
          x[r][0] = fmaf(c[0], s0, x[r][0]);
          x[r][1] = fmaf(c[1], s0, x[r][1]);
          x[r][2] = fmaf(c[2], s1, x[r][2]);
          x[r][3] = fmaf(c[3], s1, x[r][3]);
        }
        // (the sign of a row's first scale marks an empty slot, whose sums are 0)
        const float no0 = (ksc[0][0] & 0x8000u) ? -INFINITY : 0.f, no1 = (ksc[1][0] & 0x8000u) ? -INFINITY : 0.f;
        x[r][0] = fmaf(x[r][0], logit0, no0);
        x[r][1] = fmaf(x[r][1], logit1, no0);
        x[r][2] = fmaf(x[r][2], logit0, no1);
        x[r][3] = fmaf(x[r][3], logit1, no1);
      }
      // ---------------------------------------------------------- softmax --
      uint32_t vsc[kRecs][2][J];                    // V scales of rows 2t and 2t + 1, and of 8 + 2t and 9 + 2t
      uint32_t sc = top_scale;
#pragma unroll
      for (int r = 0; r < kRecs; ++r)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          load_words<J>(vsc[r][hf], v_scales + from + r * REC + hf * (D / 2));
          if (kPart)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (hf * 8 + 2 * t + i >= ((both >> (8 * r)) & 255))
#pragma unroll
                for (int k = 0; k < J / 2; ++k) vsc[r][hf][i * (J / 2) + k] = 0u;
#pragma unroll
          for (int k = 0; k < J; ++k) sc = __vmaxu2(sc, vsc[r][hf][k]);
        }
      const float m0 = fmaxf(fmaxf(x[0][0], x[0][2]), fmaxf(x[1][0], x[1][2]));
      const float m1 = fmaxf(fmaxf(x[0][1], x[0][3]), fmaxf(x[1][1], x[1][3]));
      if (__any_sync(0xffffffffu, m0 - ref[0] > kSlack || m1 - ref[1] > kSlack || sc != top_scale)) {
        // A logit well above the reference, or a V scale of a new power of two:
        // the reference moves up to the largest logit, and the power that
        // probabilities are taken times down (rarely, once a unit is under way),
        // so that probability * scale stays below 2^15.
        uint32_t big = top_scale & 0xFFFFu;
#pragma unroll
        for (int r = 0; r < kRecs; ++r)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int k = 0; k < J; ++k) {           // (NaN scales have no say)
              const uint32_t lo = vsc[r][hf][k] & 0xFFFFu, hi = vsc[r][hf][k] >> 16;
              big = max(big, lo < 0x7F80u ? lo : 0u);
              big = max(big, hi < 0x7F80u ? hi : 0u);
            }
        big = __reduce_max_sync(0xffffffffu, big) | 0x7Fu;
        top_scale = big | (big << 16);
        const int e = 141 - kSlack - static_cast<int>(big >> 7) + 127, fit = min(e, kMaxRoom + 127);
        // (a step of more than 2^-126 leaves sums too large, but far below a new term)
        const float shrink = pow2(max(fit - static_cast<int>(__float_as_uint(room) >> 23), -126));
        room = __uint_as_float(static_cast<uint32_t>(fit) << 23);
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float mx = i == 0 ? m0 : m1;
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          mx = fmaxf(mx, ref[i]);
          f[i] = fast_exp2(ref[i] - mx);
          ref[i] = mx;
          den[i] *= f[i];
          f[i] *= shrink;
        }
#pragma unroll
        for (int i = 0; i < 2 * J; ++i) {
          acc[i][0] *= f[0];
          acc[i][1] *= f[1];
          acc[i][2] *= f[0];
          acc[i][3] *= f[1];
        }
      }
      // row g of heads 2t, 2t + 1 becomes head g of rows 2t, 2t + 1
#pragma unroll
      for (int r = 0; r < kRecs; ++r) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float2 y = __fadd2_rn(make_float2(x[r][2 * hf], x[r][2 * hf + 1]), make_float2(-ref[0], -ref[1]));
          const float2 p = make_float2(fast_exp2(y.x), fast_exp2(y.y));
          den[0] += p.x;
          den[1] += p.y;
          *reinterpret_cast<float2*>(turn_to + (r * kQ4Rows + 8 * hf) * kTurn) = __fmul2_rn(p, make_float2(room, room));
        }
      }
      __syncwarp();
      // ----------------------------------------------------------- values --
#pragma unroll
      for (int r = 0; r < kRecs; ++r) {
        float pr[2][2];
        uint32_t vw[2][J];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          load_words<J>(vw[hf], codes + from + r * REC + 8 * D + hf * 4 * D);
#pragma unroll
          for (int i = 0; i < 2; ++i) pr[hf][i] = turn_from[(r * kQ4Rows + hf * 8 + i) * kTurn];
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          uint32_t bh[2], bl[2];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const uint32_t u0 = vsc[r][hf][j / 2], u1 = vsc[r][hf][J / 2 + j / 2];
            const float y0 = pr[hf][0] * __uint_as_float((j & 1) ? u0 & 0xFFFF0000u : u0 << 16);
            const float y1 = pr[hf][1] * __uint_as_float((j & 1) ? u1 & 0xFFFF0000u : u1 << 16);
            split_half2(y0, y1, &bh[hf], &bl[hf]);
          }
          const uint32_t w0 = vw[0][j], w1 = vw[1][j], w08 = w0 >> 8, w18 = w1 >> 8;
          const uint32_t a0[4] = {low_codes(w0), high_codes(w0), low_codes(w1), high_codes(w1)};
          const uint32_t a1[4] = {low_codes(w08), high_codes(w08), low_codes(w18), high_codes(w18)};
          // (summed on their own and added in fp32: the tensor cores cut a sum's
          // last bits rather than round them, which over 150 records left 1.6e-6
          // of the outputs' size)
          float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
          mma_f16(c0, a0, bl[0], bl[1], c0);
          mma_f16(c1, a1, bl[0], bl[1], c1);
          mma_f16(c0, a0, bh[0], bh[1], c0);
          mma_f16(c1, a1, bh[0], bh[1], c1);
#pragma unroll
          for (int k = 0; k < 4; k += 2) {
            float *s0 = acc[2 * j] + k, *s1 = acc[2 * j + 1] + k;
            const float2 x0 = __fadd2_rn(make_float2(s0[0], s0[1]), make_float2(c0[k], c0[k + 1]));
            const float2 x1 = __fadd2_rn(make_float2(s1[0], s1[1]), make_float2(c1[k], c1[k + 1]));
            s0[0] = x0.x, s0[1] = x0.y;
            s1[0] = x1.x, s1[1] = x1.y;
          }
        }
      }
    };
    for (; n < n_end; ++n) {
      alive = alive && __all_sync(0xffffffffu, mbar_wait(&full[stage], phase, &abort_flag, a.p.status));
      if (!alive) continue;
      const int both = warp_uniform(reinterpret_cast<const int*>(mine + Sh::kRows)[stage]);
      const uint32_t from = Sh::kRing + stage * PIECE;
      if (both == (kQ4Rows | (kQ4Rows << 8)))
        piece(std::false_type{}, from, both);
      else
        piece(std::true_type{}, from, both);
      __syncwarp();                                 // the piece and its probabilities have been read
      if (lane == 0) mbar_arrive(&full[stage] + (Sh::kEmpty - Sh::kFull) / 8);
      if (++stage == S) {
        stage = 0;
        phase ^= 1;
      }
    }

    // ------------------------------------------------- the unit (part) ends --
    // (the means over the warp's rows, whose size is the values' own: a sum, or
    // one with the power of two still on, may lie outside fp32)
    float mean[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) den[i] += __shfl_xor_sync(0xffffffffu, den[i], o);
      if (signbit(i == 0 ? logit0 : logit1) && den[i] != 0.f) den[i] = NAN;
      mean[i] = den[i] == 0.f ? 0.f : pow2(127 - static_cast<int>(__float_as_uint(room) >> 23)) * reciprocal(den[i]);
      if (g == 0) stat[warp][2 * t + i] = make_float2(den[i] == 0.f ? -INFINITY : ref[i], den[i]);
    }
    const Work w = work;
    const bool whole = w.unit.start >= x0 && w.unit.end <= x1;
    const int64_t part = (2ll * blockIdx.x + (w.x == x0 ? 0 : 1)) * G * (D + 2);
    const int64_t out = ((static_cast<int64_t>(w.unit.l) * a.p.b + w.unit.s) * a.p.Hkv + w.unit.h) * G * D;
    const bool write =
        whole ? in_bounds(out, G * D, a.ext_out, a.p.status) : in_bounds(part, G * (D + 2), a.ext_part, a.p.status);
#pragma unroll
    for (int h0 = 0; h0 < kHeads; h0 += 4) {        // four heads at a time
      if (h0 >= G) break;
      if (h0 > 0) sync_consumers();
      if (2 * t >= h0 && 2 * t < h0 + 4) {
        float* y = sums + (warp * 4 + 2 * t - h0) * HEAD + 4 * g;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float *c = acc[2 * j], *d = acc[2 * j + 1];
          const float m0 = mean[0], m1 = mean[1], n0 = m0 * 0.0625f, n1 = m1 * 0.0625f;
          *reinterpret_cast<float4*>(y + 32 * j) = make_float4(c[0] * m0, c[2] * n0, d[0] * m0, d[2] * n0);
          *reinterpret_cast<float4*>(y + HEAD + 32 * j) = make_float4(c[1] * m1, c[3] * n1, d[1] * m1, d[3] * n1);
        }
      }
      sync_consumers();
      for (int i = threadIdx.x; i < 4 * D && h0 + i / D < G && write; i += kThreads) {
        const int hd = h0 + i / D, e = i % D;
        float M = -INFINITY, L = 0.f, o = 0.f, part_of[kWarps];
#pragma unroll
        for (int x = 0; x < kWarps; ++x) M = fmaxf(M, stat[x][hd].x);
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
          const float2 st = stat[x][hd];
          part_of[x] = st.x == -INFINITY ? 0.f : fast_exp2(st.x - M) * st.y;
          L += part_of[x];
        }
        const float by_all = L == 0.f ? 0.f : reciprocal(L);
#pragma unroll
        for (int x = 0; x < kWarps; ++x) o += part_of[x] * by_all * sums[(x * 4 + i / D) * HEAD + e];
        if (whole) {
          a.out[out + hd * D + e] = o;
        } else {
          float* y = a.part + part + hd * (D + 2);
          y[e] = o;
          if (e == 0) {
            y[D] = M;
            y[D + 1] = L;
          }
        }
      }
    }
    if (threadIdx.x == 0 && w.unit.start >= x0) {   // (the CTA that begins a unit)
      const int unit = (w.unit.l * a.p.b + w.unit.s) * a.p.Hkv + w.unit.h;
      if (w.unit.end > x1)
        join[few ? unit : blockIdx.x] =
            make_int4(unit, 2 * blockIdx.x + (w.x == x0 ? 0 : 1),
                      static_cast<int>(divide(w.unit.end - 1, run, &rest_)) - static_cast<int>(blockIdx.x) + 1, 0);
      else if (few)
        join[unit] = make_int4(-1, 0, 0, 0);
    }
    if (threadIdx.x == 0 && share == kShared && w.end == x1 && !(w.unit.start >= x0 && w.unit.end > x1))
      join[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if (w.end == x1) break;
    sync_consumers();                                // the work and the sums have been read
    if (threadIdx.x == 0) {
      next_unit(span(), &work.unit);
      work.x = w.end;
      work.end = work.unit.end < x1 ? work.unit.end : x1;
    }
    sync_consumers();
  }
}

// The parts of a cut unit: part `jn.y`, then the first part of each of the next
// CTAs.  kFew: one CTA a (unit, head), its warps sharing the parts; otherwise
// one CTA a cut unit, which then has few parts, its warps sharing heads and
// parts.  Lanes run over the elements.  (8 units of 57 parts: 13 us with all
// heads in one CTA, 9 with one each, both from cold caches.)  Few means at most
// one unit to four CTAs.  By CTA against by (unit, head), 8192 rows a unit, us for
// the whole call:  8 units: 16.2, 13.3   32: 22.3, 20.6   64: 28.9, 28.2   112:
// 41.9, 41.7   128: 48.7, 48.5   256: 81.8, 83.8.
template <int D, bool kFew>
__global__ void __launch_bounds__(kJoinWarps * 32) q4_join_kernel(const Q4DecodeArgs a) {
  constexpr int E = D / 32;
  constexpr int H = kFew ? 1 : kHeads;              // heads of a CTA
  constexpr int W = kJoinWarps / H;                 // warps of a head
  __shared__ float sums[kJoinWarps][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.G, item = kFew ? blockIdx.x / G : blockIdx.x, h0 = kFew ? blockIdx.x % G : 0;
  wait_for_previous_kernels();
  const int4 jn = join_of(a)[item];
  if (jn.x < 0) return;
  const int hd = h0 + warp / W, first_cta = jn.y / 2;
  const auto part = [&](int i) {
    return a.part + static_cast<int64_t>(i == 0 ? jn.y : 2 * (first_cta + i)) * G * (D + 2) + hd * (D + 2);
  };
  float o[E];
#pragma unroll
  for (int k = 0; k < E; ++k) o[k] = 0.f;
  if (hd < G) {
    // (this warp's first part, on its way while the parts' weights are added: 0.6 us
    // of a short layer's 15.7)
    const int i0 = warp % W;
    float first[E];
#pragma unroll
    for (int k = 0; k < E; ++k) first[k] = i0 < jn.z ? part(i0)[lane + 32 * k] : 0.f;
    // the parts' largest reference and, by it, the sum of all probabilities
    float M = -INFINITY, L = 0.f;
    const auto add = [&](float m, float l) {
      const float to = fmaxf(M, m);
      if (to == -INFINITY) return;
      L = L * fast_exp2(M - to) + l * fast_exp2(m - to);
      M = to;
    };
    for (int i = lane; i < jn.z; i += 32) add(part(i)[D], part(i)[D + 1]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
      const float m = __shfl_xor_sync(0xffffffffu, M, x), l = __shfl_xor_sync(0xffffffffu, L, x);
      add(m, l);
    }
    const float by_all = L == 0.f ? 0.f : reciprocal(L);
    // (parts without a row are zeros; a NaN shows whatever its part's weight)
    const auto weight = [&](const float* p) {
      return p[D] == -INFINITY ? 0.f : fast_exp2(p[D] - M) * p[D + 1] * by_all;
    };
    if (i0 < jn.z) {
      const float f = weight(part(i0));
#pragma unroll
      for (int k = 0; k < E; ++k) o[k] = f * first[k];
    }
#pragma unroll 4
    for (int i = i0 + W; i < jn.z; i += W) {
      const float* p = part(i);
      const float f = weight(p);
#pragma unroll
      for (int k = 0; k < E; ++k) o[k] += f * p[lane + 32 * k];
    }
  }
#pragma unroll
  for (int k = 0; k < E; ++k) sums[warp][lane + 32 * k] = o[k];
  __syncthreads();
  const int64_t out = (static_cast<int64_t>(jn.x) * G + h0) * D;
  const int heads = kFew ? 1 : G;
  if (!in_bounds(out, heads * D, a.ext_out, a.p.status)) return;
  for (int i = threadIdx.x; i < heads * D; i += kJoinWarps * 32) {
    const int h = i / D, e = i % D;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += sums[h * W + w][e];
    a.out[out + i] = v;
  }
}

template <int D>
cudaError_t launch(const Q4DecodeArgs& a, cudaStream_t stream) {
  // (the limit is one for every call: two threads that each set their own would
  // change it under one another)
  constexpr int kLimit = Shape<D>::kLens + (kQ4MaxBatch + 1) * 4;
  static_assert(kLimit <= 226 * 1024, "shared memory of a block");
  cudaError_t e = cudaFuncSetAttribute(q4_decode_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLimit);
  if (e != cudaSuccess) return e;
  const int64_t units = static_cast<int64_t>(a.p.L) * a.p.b * a.p.Hkv;
  const int64_t pieces = (static_cast<int64_t>(a.p.max_pages) * a.p.page_rows + kPieceRows - 1) / kPieceRows;
  auto* main_kernel = q4_decode_kernel<D>;
  if (pieces <= kWholePieces)
    return launch_early(main_kernel, static_cast<unsigned>(units), kBlock, Shape<D>::kLens + 8, stream, 1, a,
                        int{kOneUnit});
  const int smem = Shape<D>::kLens + (a.p.b + 1) * 4;
  const bool few = 4 * units <= a.ctas;
  auto* few_kernel = q4_join_kernel<D, true>;
  auto* join_kernel = q4_join_kernel<D, false>;
  e = launch_early(main_kernel, a.ctas, kBlock, smem, stream, 1, a, int{few ? kFewUnits : kShared});
  if (e != cudaSuccess) return e;
  if (few) return launch_early(few_kernel, static_cast<unsigned>(units) * a.G, kJoinWarps * 32, 0, stream, 1, a);
  return launch_early(join_kernel, a.ctas, kJoinWarps * 32, 0, stream, 1, a);
}

}  // namespace

cudaError_t launch_q4_decode(const Q4DecodeArgs& a, cudaStream_t stream) {
  return a.p.d == 128 ? launch<128>(a, stream) : launch<64>(a, stream);
}

}  // namespace rolekv
