// Attention of drafted nodes over the paged cache: each of a sequence's N nodes sees its P cached
// tokens and, of the nodes cached behind them, those whose bits its mask sets.
//
// Lengths are read on the GPU, so the launch divides the work itself.  A KV head's N G (node, head)
// rows are cut into tiles of M = 32 kWaves rows, an item is a tile over all P + N keys, and a step
// is 32 keys of an item.  With U units in all, one a step and item_cost before each item's first,
// workgroup w takes those of the units [w q, (w + 1) q) in the items' order that are steps, q =
// ceil(U / workgroups): some whole items, and at most a part of one before and of one behind them.
// Parts are float32 results, normalised, with their log-sum-exps in slots 2 w (an item begun by
// another workgroup) and 2 w + 1 (one that it begins and does not end), and a record tells the merge
// how many workgroups' slots hold the item.  Neighbouring ranges run on one XCD, so that tiles of the
// same keys share its L2.
//
// A step's K and V tiles, two pages, are copied from memory straight into an LDS ring (16 bytes a lane,
// the tiles as stored) some steps ahead, across the ends of items, and shared by the waves.  Wave w holds
// 32 of the tile's rows as the columns of its products, on v_mfma_f32_32x32x16_bf16:
//   S^T[32 keys x 32 rows] = K Q^T: 8 products over the 128 channels; lane (key m, half h) reads K
//     granule (2 c + h) 16 + m % 16 of page m / 16 and gets the scores of keys 8 (r / 4) + 4 h + r % 4
//     (r = 0 .. 15) for its row;
//   O^T[128 channels x 32 rows] += V^T P^T: per page 4 products; a lane's probabilities of a page are
//     its operand as they come out of the scores, V granule 128 h + d the other.
// Softmax runs online in base 2 with the running maximum set on an item's first step and moved only
// when a lane's sum of 16 probabilities exceeds 2^kTau, for the wave's 32 rows together: a row's last
// bits depend on its neighbours'.  Probabilities enter the products as bf16, off by at most 2^-8 of
// each, their sum is taken in float32 before.
//
// Steps that reach past the cached tokens are masked: a row's 32 bits of them are its mask's, shifted.
// There the values may be those of nodes that a row does not see, or nothing; where any is not
// finite, a product of a zero probability would be NaN, and the step takes finite values only
// and adds the infinities and NaNs of seen nodes one by one (rare).
//
// What bounds it.  Up to 128 rows a KV head the reads: four requests of 123,000 tokens, 2.02 GB,
// 320 us, 6.3 TB/s (a plain streaming read 7.1); 32 sequences of 4,000 tokens, 0.53 GB, 92 us with
// 16 rows, 5.7 TB/s, of which some 9 are the time until the first copies land, and 122 with 128 rows,
// whose scores and probabilities take as long as the copies.  256 rows (32 sequences of 8,192 tokens,
// 64 nodes, 4 heads to a KV head): 292-298 us after a fill of other memory, 344 a pass in a row of
// them, 800-940 TFLOP/s.  There the matrix cores and the reads of LDS: a wave's 32 rows take all of a
// step's 16 KiB from it, so the eight waves 128 KiB, 1,024 cycles at 128 bytes each, and the products
// of a SIMD's two waves take 1,024 too.  The next step's scores among this step's products took wide
// trees from 411 to 333 us; a higher wave priority there than at probabilities takes them from 303 to
// 290 a pass.  Non-temporal copies, whose lines displace nothing: 92 us instead of 169 with 16 rows,
// 163 instead of 200 with 256, after a fill of other memory.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "drafts.h"
#include "internal.h"

namespace libra {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kStepKeys = 32;
constexpr int kTau = 8;  // a sum's exponent in base 2 from which the running maximum moves
constexpr float kSumTau = float(1 << kTau);
constexpr int kMaskWords = LIBRA_MAX_MASK_WORDS;
constexpr int kPartBlock = 32 * kDim / 4;  // 32 rows of a part, in fours of floats
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Workgroups of the launch: all that run at once, by their LDS: one of eight waves and 128 KiB to a CU,
// two of four waves and 64 KiB.
constexpr int kCus = 256;
constexpr int groups_of(int waves) { return kCus * 8 / waves; }

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 x) { return __builtin_bit_cast(bf16x8, x); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ constexpr int acc_row(int r, int h) { return 8 * (r / 4) + 4 * h + (r % 4); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x)))) | uint64_t(uint32_t(uniform(int(x >> 32)))) << 32);
}
template <int kCount>
__device__ __forceinline__ void wait_loads() {  // all but the last kCount vector-memory operations
  __builtin_amdgcn_s_waitcnt((kCount & 15) | (kCount >> 4) << 14 | 0x0F70);
}

// What the merge gets to know of an item that workgroup w begins and does not end.
struct alignas(32) Split {
  int32_t parts;  // 0: there is none
  int32_t row0, nodes, g, tile;
};

struct TreeArgs {
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const uint16_t* q;
  const uint32_t* mask;
  const int32_t* prior;
  const int32_t* starts;
  const int32_t* table;
  uint16_t* out;
  float* lse;
  float* part_o;
  float* part_lse;
  Split* splits;  // of each workgroup
  int64_t stride;
  uint32_t last_page;
  int rows, most;  // query rows, tokens that a row of the block table can hold
  int batch, hkv, hq, group, mask_words;
  int item_cost;  // units
  float sl2;
};

// A sequence's sizes, kept inside the rows and the block table whatever the caller's memory holds.
struct Seq {
  int prior, nodes, row0, len, steps, tiles;
};
template <int kRows>
__device__ __forceinline__ Seq make_seq(const TreeArgs& A, int prior, int start, int end) {
  Seq s;
  s.row0 = min(max(start, 0), A.rows);
  s.nodes = min(max(end, s.row0), A.rows) - s.row0;
  s.prior = min(max(prior, 0), A.most);
  s.len = int(min(uint32_t(s.prior) + uint32_t(s.nodes), uint32_t(A.most)));
  s.steps = (s.len + kStepKeys - 1) / kStepKeys;
  s.tiles = (s.nodes * A.group + kRows - 1) / kRows;  // rows * hq fits 32 bits
  return s;
}

// Lane l holds the lengths of sequence first + l, loaded at once: the sequences of a range are then
// found without a chain of loads.
template <int kRows>
struct Window {
  int first, prior, start, end;
  __device__ __forceinline__ void load(const TreeArgs& A, int from, int lane) {
    first = from;
    const int b = min(from + lane, A.batch - 1);
    prior = A.prior[b], start = A.starts[b], end = A.starts[b + 1];
  }
  // This lane's sequence's items, one a tile and KV head, and their steps.
  __device__ __forceinline__ void count(const TreeArgs& A, int lane, int64_t& items, int64_t& steps) const {
    const Seq s = make_seq<kRows>(A, prior, start, end);
    items = first + lane < A.batch && s.steps > 0 ? int64_t(s.tiles) * A.hkv : 0;
    steps = items * s.steps;
  }
  __device__ __forceinline__ Seq get(const TreeArgs& A, int b, int lane) {
    if (b >= first + 64) load(A, b, lane);
    const int l = b - first;
    return make_seq<kRows>(A, __builtin_amdgcn_readlane(prior, l), __builtin_amdgcn_readlane(start, l),
                           __builtin_amdgcn_readlane(end, l));
  }
};

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int n = 32; n; n >>= 1) x += __shfl_xor(x, n);
  return uniform64(x);
}

// A place in the launch's steps.
template <int kRows>
struct Cursor {
  Window<kRows> window;
  Seq seq;
  int b, g, tile, step;
  // To the workgroup's first step; returns how many it has (0: none).  each: the ranges' size.
  __device__ __forceinline__ int start(const TreeArgs& A, int w, int groups, int lane, int64_t& each) {
    int64_t items, steps, total = 0, total_steps = 0;
    for (int b0 = 0; b0 < A.batch; b0 += 64) {
      window.load(A, b0, lane);
      window.count(A, lane, items, steps);
      total += wave_sum(steps + A.item_cost * items);
    }
    each = (total + groups - 1) / groups;
    const int64_t begin = w * each, end = min(begin + each, total);
    if (begin >= total) return 0;
    // Steps before a place in the ranges' units: of an item, A.item_cost units and then its steps.
    int64_t before = 0, steps_before = 0, first_step = -1;
    for (int b0 = 0; b0 < A.batch; b0 += 64) {
      if (window.first != b0) window.load(A, b0, lane);
      window.count(A, lane, items, steps);
      int64_t upto = steps + A.item_cost * items, upto_steps = steps;
      const int64_t cost = upto;
#pragma unroll
      for (int n = 1; n < 64; n <<= 1) {
        const int64_t y = __shfl_up(upto, n), z = __shfl_up(upto_steps, n);
        if (lane >= n) upto += y, upto_steps += z;
      }
      // Where `unit` lies in this turn's sequences: the sequence, the item in it, the step in that.
      auto locate = [&](int64_t unit, int& at_b, int& at_item, int& at_step) -> int64_t {
        const int l = __builtin_ctzll(__ballot(before + upto > unit));
        at_b = uniform(b0 + l);
        seq = window.get(A, at_b, lane);
        const int64_t in_seq = unit - before - uniform64(__shfl(upto - cost, l));
        const int item_units = seq.steps + A.item_cost;
        at_item = uniform(int(in_seq / item_units));
        at_step = max(uniform(int(in_seq - int64_t(at_item) * item_units)) - A.item_cost, 0);
        return steps_before + uniform64(__shfl(upto_steps - steps, l)) + int64_t(at_item) * seq.steps + at_step;
      };
      const int64_t here = before + uniform64(__shfl(upto, 63));
      if (end < here && end >= before) {  // begin lies in this turn too, or in one before
        int b1, item1, step1;
        total_steps = locate(end, b1, item1, step1);
      } else if (end == here) {
        total_steps = steps_before + uniform64(__shfl(upto_steps, 63));
      }
      if (first_step < 0 && begin < here) {
        int item;
        first_step = locate(begin, b, item, step);
        g = uniform(item / seq.tiles);
        tile = item - g * seq.tiles;
      }
      if (end <= here) break;
      before = here;
      steps_before += uniform64(__shfl(upto_steps, 63));
    }
    // The window may have gone on to the range's end.
    if (b < window.first) window.load(A, b / 64 * 64, lane);
    seq = window.get(A, b, lane);
    return int(total_steps - first_step);
  }
  // To the next sequence that has nodes.
  __device__ __forceinline__ void next_seq(const TreeArgs& A, int lane) {
    g = tile = step = 0;
    do {
      ++b;
      seq = window.get(A, b, lane);
    } while (seq.tiles == 0 && b + 1 < A.batch);
  }
  // To the first step of the next item; not past the launch's last one.
  __device__ __forceinline__ void next_item(const TreeArgs& A, int lane) {
    step = 0;
    if (++tile < seq.tiles) return;
    tile = 0;
    if (++g < A.hkv) return;
    next_seq(A, lane);
  }
};

// The rows of a wave: their running maximum and sum, and the unnormalised output, transposed: lane
// (col, hh) holds channels 32 cb + 8 e + 4 hh .. + 3 of row col.
struct Rows {
  f32x16 acc[4];
  float m, l;
  __device__ __forceinline__ void clear() {
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[cb][r] = 0.f;
  }
};

// A step's probabilities from its scores, against the running maximum.  While a row has seen no
// finite score the offset is the largest float: scores of -inf give 0, and the first finite one
// infinity, which moves the maximum, as any sum above 2^kTau does.
__device__ __forceinline__ void soften(Rows& R, const f32x16& sc, float sl2, bf16x8 (&pr)[2]) {
  float p[16], ps;
  auto take = [&]() {
    const float neg_m = R.m == -INFINITY ? FLT_MAX : -R.m;
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], sl2, neg_m));
    const float t0 = (p[0] + p[1]) + (p[2] + p[3]), t1 = (p[4] + p[5]) + (p[6] + p[7]);
    const float t2 = (p[8] + p[9]) + (p[10] + p[11]), t3 = (p[12] + p[13]) + (p[14] + p[15]);
    ps = (t0 + t1) + (t2 + t3);
  };
  take();
  if (__ballot(!(ps <= kSumTau))) {
    float mloc = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mloc = fmaxf(mloc, sc[r]);
    float mc = fmaxf(mloc * sl2, R.m);
    mc = fmaxf(mc, __shfl_xor(mc, 32));
    const float alpha = R.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(R.m - mc);
    R.l *= alpha;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) R.acc[cb] *= alpha;
    R.m = mc;
    take();
  }
  R.l += ps;
  pr[0] = as_bf16x8(make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                               pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
  pr[1] = as_bf16x8(make_uint4(pack_bf16x2(p[8], p[9]), pack_bf16x2(p[10], p[11]),
                               pack_bf16x2(p[12], p[13]), pack_bf16x2(p[14], p[15])));
}

// Which of a step's keys the row sees (bit i: key key0 + i), in a step that reaches past the cached
// tokens.  bits: the row's mask words in LDS.
__device__ __forceinline__ uint32_t seen_keys(const TreeArgs& A, const Seq& s, const uint32_t* bits, int node,
                                              int key0) {
  uint32_t sees;
  const int d = key0 - s.prior;  // > -32: the first key's node
  if (!A.mask) {
    const int lim = node - d;
    sees = lim >= 31 ? ~0u : lim < 0 ? 0u : (2u << lim) - 1;
  } else if (d < 0) {
    sees = bits[0] << -d | ((1u << -d) - 1);
  } else {
    const int i = d >> 5, sh = d & 31;
    const uint32_t w0 = i < A.mask_words ? bits[i] : 0;
    const uint32_t w1 = i + 1 < A.mask_words ? bits[i + 1] : 0;
    sees = uint32_t((uint64_t(w1) << 32 | w0) >> sh);
  }
  const int left = s.len - key0;
  if (left < 32) sees &= (1u << left) - 1;
  return node < s.nodes ? sees : 0;
}
__device__ __forceinline__ void mask_scores(uint32_t sees, int hh, f32x16& sc) {
  sees >>= 4 * hh;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (!(sees >> acc_row(r, 0) & 1)) sc[r] = -INFINITY;
}

// The products of a step's values, v[4 j + cb] being page j's of channel block cb.
__device__ __forceinline__ void add_values(Rows& R, const uint4 (&v)[8], const bf16x8 (&pr)[2]) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    R.acc[c & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[c]), pr[c >> 2], R.acc[c & 3], 0, 0, 0);
}

// Sets the top bit of each half whose bf16 is infinite or NaN (and other bits).
__device__ __forceinline__ uint32_t special_bits(uint32_t x) { return (x & 0x7F807F80u) + 0x00800080u; }

// Zeroes values in slots past the end, `valid` keys from the step's first; whether any that is left
// is not finite.
__device__ __forceinline__ bool trim_values(uint4 (&v)[8], int valid, int hh) {
  uint32_t special = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int s0 = j * kPage + 8 * (e / 2) + 4 * hh + 2 * (e % 2);
      const uint32_t keep = (s0 < valid ? 0x0000FFFFu : 0u) | (s0 + 1 < valid ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        uint32_t& x = reinterpret_cast<uint32_t*>(&v[4 * j + cb])[e];
        x &= keep;
        special |= special_bits(x);
      }
    }
  return __ballot((special & 0x80008000u) != 0) != 0;
}

// Where some values of a masked step are not finite, a product with a probability of 0 would be NaN:
// they are added one by one to the rows that see them (slow, and rare), and the products take
// zeros in their place.  tile0, tile1: the two pages' V tiles, in LDS.
__device__ __forceinline__ void finite_values(uint4 (&v)[8]) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t& x = reinterpret_cast<uint32_t*>(&v[c])[e];
      x &= ~((special_bits(x) >> 15 & 0x00010001u) * 0xFFFFu);
    }
}
template <class Tile>
__device__ __forceinline__ void add_special_values(Rows& R, uint32_t sees, int hh, Tile tile0, Tile tile1) {
#pragma unroll 1
  for (int key = 0; key < kStepKeys; ++key) {
    const bool seen = sees >> key & 1;
    const int slot = key & (kPage - 1);
    const Tile t = (key < kPage ? tile0 : tile1) + 1024 * (slot >> 2 & 1) + 32 * hh + 4 * (slot >> 3) + (slot & 3);
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t x = t[8 * (32 * cb + 8 * (r / 4) + r % 4)];
        R.acc[cb][r] += seen && (x & 0x7F80u) == 0x7F80u ? __uint_as_float(x << 16) : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);  // few registers, rather than many loads at once
    }
  }
}

// The row's query as the score products' operands, and its mask words.
__device__ __forceinline__ void load_query(const TreeArgs& A, const Seq& s, int g, int node, int head, int hh,
                                           bf16x8 (&qop)[8], uint32_t* bits) {
  const bool ok = node < s.nodes;
  const uint4* qrow = reinterpret_cast<const uint4*>(
      A.q + (size_t(s.row0 + (ok ? node : 0)) * A.hq + size_t(g) * A.group + head) * kDim);
#pragma unroll
  for (int c = 0; c < 8; ++c) qop[c] = as_bf16x8(ok ? qrow[2 * c + hh] : make_uint4(0, 0, 0, 0));
  if (A.mask)
    for (int i = hh; i < A.mask_words; i += 2)
      bits[i] = ok ? A.mask[size_t(s.row0 + node) * A.mask_words + i] : 0;
}

// One int per lane straight into LDS, lane after lane.  The s_nop: a load to LDS may read an m0 that the
// instruction right before it writes too early; one wait state is needed, which the compiler puts
// between its own instructions, but not inside an asm block.
__device__ __forceinline__ void copy_lds_dword(const int32_t* src, int32_t* dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(uniform(int(reinterpret_cast<uintptr_t>(dst)))), "v"(src)
               : "memory", "m0");
}
__device__ __forceinline__ void wave_sync() {  // LDS operations of one wave complete in order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A tile's waves share each step's K and V through LDS.  Eight waves meet every two steps (a pass of
// 256 rows over 32 x 8,192 tokens 344 us, 365 every step), four every step, as two steps would take
// two more stages.
template <int kWaves>
struct Ring {
  static constexpr int kStages = kWaves;
  static constexpr int kCopies = 16 / kWaves;  // of 1 KiB, per wave and step
  static constexpr int kUnit = kWaves / 4;     // steps between barriers
  // What a unit reads, and the scores a step ahead, is copied before it begins.
  static_assert(kStages >= 2 * kUnit + 1 && kCopies <= 4);
};

template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void tree_ring_kernel(TreeArgs A) {
  constexpr int kRows = 32 * kWaves;
  constexpr int kStages = Ring<kWaves>::kStages;
  constexpr int kCopies = Ring<kWaves>::kCopies;
  constexpr int kUnit = Ring<kWaves>::kUnit;
  __shared__ __align__(16) uint4 ring[kStages][4][256];  // K of the step's two pages, V of them
  __shared__ uint32_t bits[kRows][kMaskWords + 1];
  __shared__ int32_t ids[kWaves][2][3][64];  // of two turns of 64 steps: a step's page ids and KV head
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int G = A.group;

  // Neighbouring ranges on one XCD: workgroup w runs on XCD w % 8.
  const int per_xcd = int(gridDim.x) / kNumXcds;
  const int w = int(blockIdx.x) % kNumXcds * per_xcd + int(blockIdx.x) / kNumXcds;
  Cursor<kRows> at;
  int64_t each;
  const int n_steps = uniform(at.start(A, w, int(gridDim.x), lane, each));
  if (tid == 0) A.splits[w].parts = 0;  // unless an item is begun and not ended, below
  if (n_steps == 0) return;

  // What the copies need of each step, page ids and KV head, 64 steps at a time: lane l finds
  // step l's place among the sequences and copies its two ids into LDS, asynchronously like the tiles,
  // 64 steps ahead, so that no step waits for them.
  Cursor<kRows> fill = at;
  int filled = 0;
  auto fill_ids = [&]() {
    int32_t(&to)[3][64] = ids[wave][filled >> 6 & 1];
    const int32_t *id0 = A.table, *id1 = A.table;
    int head = 0, done = 0;
    const int want = min(n_steps - filled, 64);
    while (true) {  // the sequences of these steps
      const Seq& s = fill.seq;
      const int64_t left = (int64_t(A.hkv - fill.g) * s.tiles - fill.tile) * s.steps - fill.step;
      const int take = int(min(left, int64_t(want - done)));
      const int x = lane - done;
      if (x >= 0 && x < take) {
        const uint32_t item = uint32_t(fill.step + x) / uint32_t(s.steps);
        const int step = fill.step + x - int(item) * s.steps;
        head = fill.g + int((uint32_t(fill.tile) + item) / uint32_t(s.tiles));
        const int32_t* row = A.table + fill.b * A.stride;
        id0 = row + 2 * step;
        id1 = row + min(2 * step + 1, (s.len - 1) / kPage);
      }
      done += take;
      if (done < want) {
        fill.next_seq(A, lane);
        continue;
      }
      const uint32_t items = uint32_t(fill.step + take) / uint32_t(s.steps);
      fill.step += take - int(items) * s.steps;
      const uint32_t tile = uint32_t(fill.tile) + items;
      fill.g += int(tile / uint32_t(s.tiles));
      fill.tile = int(tile % uint32_t(s.tiles));
      if (fill.g == A.hkv && filled + want < n_steps) fill.next_seq(A, lane);
      break;
    }
    copy_lds_dword(id0, &to[0][0]);
    copy_lds_dword(id1, &to[1][0]);
    to[2][lane] = head;
    filled += 64;
  };
  // A wave copies 1 KiB pieces of one of the step's tiles K 0, K 1, V 0, V 1.  Lane l holds the tile's
  // offset of step l of the current turn.
  const uint32_t page_bytes = uint32_t(A.hkv) * kTileBytes, lane_bytes = uint32_t(lane) * 16;
  const int piece0 = wave * kCopies, my_tile = piece0 / 4;
  const uint64_t my_cache = reinterpret_cast<uint64_t>(my_tile < 2 ? A.k_cache : A.v_cache) + piece0 % 4 * 1024;
  uint64_t off = 0;
  int copied = 0;
  auto copy_step = [&]() {
    if ((copied & 63) == 0) {
      // A turn's ids landed long ago; the next turn's then take the place of the last's.
      const int32_t(&from)[3][64] = ids[wave][copied >> 6 & 1];
      off = uint64_t(min(uint32_t(from[my_tile & 1][lane]), A.last_page)) * page_bytes +
            uint32_t(from[2][lane]) * kTileBytes;
      if (copied > 0 && filled < n_steps) fill_ids();
    }
    const uint64_t at_page = uint64_t(uint32_t(__builtin_amdgcn_readlane(int(off), copied & 63))) |
                             uint64_t(uint32_t(__builtin_amdgcn_readlane(int(off >> 32), copied & 63))) << 32;
    const int stage = uniform(int(reinterpret_cast<uintptr_t>(&ring[copied % kStages][0][0])));
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                   :
                   : "s"(stage + (piece0 + c) * 1024), "v"(lane_bytes), "s"(my_cache + at_page + c * 1024)
                   : "memory", "m0");
    }
    ++copied;
  };
  // Waits until all but the last `steps` steps' copies have landed, for every wave.
  auto wait_steps = [&](int steps) {
    switch (min(steps, kStages - 1)) {
      case 0: wait_loads<0>(); break;
      case 1: wait_loads<kCopies>(); break;
      case 2: wait_loads<2 * kCopies>(); break;
      case 3: wait_loads<3 * kCopies>(); break;
      case 4: wait_loads<4 * kCopies>(); break;
      case 5: wait_loads<5 * kCopies>(); break;
      case 6: wait_loads<6 * kCopies>(); break;
      default: wait_loads<7 * kCopies>(); break;
    }
    __syncthreads();
  };
  // Before step n (every kUnit steps): the copies of the steps until the next time have landed, and
  // of the one whose scores are taken ahead; all waves are done with the steps before, and
  // their stages are filled again.
  int n = 0;
  auto open_step = [&]() {
    if (n % kUnit) return;
    wait_steps(max(copied - n - kUnit - 1, 0));
    const int until = min(n + kStages, n_steps);
    while (copied < until) copy_step();
  };
  fill_ids();
  wait_loads<0>();
  wave_sync();
  if (filled < n_steps) fill_ids();
#pragma unroll 1
  while (copied < min(kStages - kUnit, n_steps)) copy_step();

  bf16x8 qop[8];
  Rows R;
  auto load_keys = [&](uint4(&k)[8], int n) {
    const uint4(&stage)[4][256] = ring[n % kStages];
#pragma unroll
    for (int c = 0; c < 8; ++c) k[c] = stage[col >> 4][(2 * c + hh) * 16 + (col & 15)];
  };
  auto score = [&](const uint4(&k)[8]) {
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[c]), qop[c], sc, 0, 0, 0);
    return sc;
  };
  auto load_value = [&](int n, int c) { return ring[n % kStages][2 + (c >> 2)][128 * hh + 32 * (c & 3) + col]; };
  // The wave's row of this lane in the cursor's item.
  auto row_of = [&](int& node, int& head) {
    const int r = at.tile * kRows + 32 * wave + col;
    node = r / G, head = r - node * G;
  };
  int node, head;
  uint32_t* const my_bits = bits[32 * wave + col];
  row_of(node, head);
  load_query(A, at.seq, at.g, node, head, hh, qop, my_bits);
  while (true) {  // the range's parts of items
    const Seq s = at.seq;
    const int g = at.g, tile = at.tile, step0 = at.step, step1 = min(s.steps, step0 + n_steps - n);
    // A wave without rows in the tile only copies and keeps step.
    const bool idle = tile * kRows + 32 * wave >= s.nodes * G;
    R.clear();
    wave_sync();
    int step = step0;
    // Steps over cached tokens alone, which every row sees.
    const int plain = min(s.prior / kStepKeys, step1 - 1);
    if (!idle && step < plain) {
      uint4 k[8];
      open_step();
      load_keys(k, n);
      f32x16 sc = score(k);
      while (true) {
        bf16x8 pr[2];
        load_keys(k, n + 1);
        soften(R, sc, A.sl2, pr);
        // The next step's scores, a chain of products, among this step's values' independent ones.  A
        // wave at its products goes before the other one of its SIMD, which may take its
        // probabilities meanwhile.
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[c]), qop[c], sc, 0, 0, 0);
          R.acc[c & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(load_value(n, c)), pr[c >> 2],
                                                                 R.acc[c & 3], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        ++step, ++n;
        if (step == plain) break;
        open_step();
      }
    }
    for (; step < step1; ++step, ++n) {
      open_step();
      if (idle) continue;
      uint4 k[8], v[8];
      load_keys(k, n);
      f32x16 sc = score(k);
      const int key0 = step * kStepKeys;
      uint32_t sees = ~0u;
      if (key0 + kStepKeys > s.prior) {
        sees = seen_keys(A, s, my_bits, node, key0);
        mask_scores(sees, hh, sc);
      }
      bf16x8 pr[2];
      soften(R, sc, A.sl2, pr);
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] = load_value(n, c);
      if (trim_values(v, s.len - key0, hh) && key0 + kStepKeys > s.prior) {
        finite_values(v);
        const uint4(&stage)[4][256] = ring[n % kStages];
        add_special_values(R, sees, hh, reinterpret_cast<const uint16_t*>(stage[2]),
                           reinterpret_cast<const uint16_t*>(stage[3]));
      }
      add_values(R, v, pr);
    }
    // The next part's queries are on their way before this part's results.
    const int row_node = node, row_head = head;
    if (n < n_steps) {
      at.next_item(A, lane);
      row_of(node, head);
      load_query(A, at.seq, at.g, node, head, hh, qop, my_bits);
    }
    // Row col's sum over both lane halves.
    const float ls = R.l + __shfl_xor(R.l, 32);
    const float inv = ls > 0.f ? 1.f / ls : ls == 0.f ? 0.f : ls;  // a NaN stays
    if (step0 == 0 && step1 == s.steps) {
      const size_t orow = size_t(s.row0 + row_node) * A.hq + size_t(g) * G + row_head;
      uint4* const o = reinterpret_cast<uint4*>(A.out + orow * kDim);
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          // The row's lanes exchange halves, so that each has eight channels: granule e or e + 1.
          uint32_t x[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const auto r = __builtin_amdgcn_permlane32_swap(
                pack_bf16x2(R.acc[cb][4 * e + 2 * i] * inv, R.acc[cb][4 * e + 2 * i + 1] * inv),
                pack_bf16x2(R.acc[cb][4 * e + 4 + 2 * i] * inv, R.acc[cb][4 * e + 5 + 2 * i] * inv), false, false);
            x[i] = r[0], x[2 + i] = r[1];
          }
          if (row_node < s.nodes) o[4 * cb + e + hh] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      if (row_node < s.nodes && A.lse && hh == 0) A.lse[orow] = ls == 0.f ? -INFINITY : (R.m + log2f(ls)) * kLn2;
    } else if (row_node < s.nodes) {
      // A part, as the lanes hold it: four channels of a lane after those of the lane before.
      const size_t block = (size_t(2) * w + (step0 == 0 ? 1 : 0)) * kWaves + wave;
      f32x4* const o = reinterpret_cast<f32x4*>(A.part_o) + block * kPartBlock + lane;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[(4 * cb + e) * 64] = f32x4{R.acc[cb][4 * e] * inv, R.acc[cb][4 * e + 1] * inv, R.acc[cb][4 * e + 2] * inv,
                                       R.acc[cb][4 * e + 3] * inv};
      if (hh == 0) A.part_lse[block * 32 + col] = ls == 0.f ? -INFINITY : R.m + log2f(ls);
    }
    if (step1 < s.steps && step0 == 0 && tid == 0) {
      // The item's other parts are those of the workgroups after this one.
      A.splits[w] = {int((s.steps - step1 + each - 1) / each) + 1, s.row0, s.nodes, g, tile};
    }
    if (n == n_steps) return;
  }
}

// Joins the parts of the items that workgroups of the attention began and did not end.  Workgroup
// (x, y) takes kMergeGroups / kPerRow rows of the tile of workgroup x's item; kPerRow groups of 16
// threads, eight channels each, fold a row's parts.  Where items have many parts, most records are
// empty, and x counts the others: the workgroup finds its own among all of them.
constexpr int kMergeThreads = 256;
constexpr int kMergeGroups = kMergeThreads / 16;
static_assert(groups_of(4) <= 2 * kMergeThreads, "the merge looks at two records a thread");

// The x-th workgroup with a split item, or -1.
__device__ __forceinline__ int find_split(const TreeArgs& A, int groups, int x) {
  __shared__ int counts[2][kMergeThreads / 64], found;
  const int tid = threadIdx.x;
  if (tid == 0) found = -1;
  uint64_t has[2];  // of records 256 i + 64 wave ..
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = kMergeThreads * i + tid;
    has[i] = __ballot(at < groups && A.splits[at].parts != 0);
    if ((tid & 63) == 0) counts[i][tid >> 6] = __popcll(has[i]);
  }
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int v = 0; v < kMergeThreads / 64; ++v) {
      if (v == tid >> 6 && has[i] >> (tid & 63) & 1 &&
          before + __popcll(has[i] & ((uint64_t(1) << (tid & 63)) - 1)) == x)
        found = kMergeThreads * i + tid;
      before += counts[i][v];
    }
  __syncthreads();
  return found;
}

template <int kPerRow>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(TreeArgs A, int groups, int tile_rows) {
  constexpr int kBatch = kPerRow == 1 ? 2 : 4;  // parts that a group loads at a time
  const int w = kPerRow == 1 ? int(blockIdx.x) : find_split(A, groups, blockIdx.x);
  if (w < 0) return;
  const Split s = A.splits[w];
  const int n = min(s.parts, groups - w);  // of lengths that changed meanwhile, too, within the workspace
  if (n <= 0) return;
  // Neighbouring lanes take neighbouring rows, whose parts lie together; t: eight channels.
  constexpr int kBlockRows = kMergeGroups / kPerRow;
  const int tid = threadIdx.x, t = tid / kBlockRows % 16, k = tid / (16 * kBlockRows);
  const int in_tile = int(blockIdx.y) * kBlockRows + tid % kBlockRows;
  const int r = s.tile * tile_rows + in_tile;
  const int node = r / A.group, head = r - node * A.group;
  const bool live = node < s.nodes;
  if (kPerRow == 1 && !live) return;
  float M = -INFINITY, sum = 0.f, acc[8] = {};
  auto fold = [&](float Mk, float wk, const float (&xk)[8]) {
    // A part without a key of the row adds nothing, whatever else it holds; a NaN makes a NaN.
    const float Mn = fmaxf(M, Mk);
    const float a = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
    const float c = Mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(Mk - Mn);
    sum = sum * a + wk * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = (a == 0.f ? 0.f : acc[e] * a) + (c == 0.f ? 0.f : xk[e] * c);
    M = Mn;
  };
  for (int j0 = k * kBatch; j0 < n; j0 += kPerRow * kBatch) {
    float lj[kBatch];
    f32x4 lo[kBatch], hi[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      lj[j] = -INFINITY;
      lo[j] = hi[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live && j0 + j < n) {
        const size_t slot = j0 + j == 0 ? size_t(2) * w + 1 : size_t(2) * (w + j0 + j);
        lj[j] = A.part_lse[slot * tile_rows + in_tile];
        const f32x4* o = reinterpret_cast<const f32x4*>(A.part_o) + (slot * tile_rows + in_tile) / 32 * kPartBlock +
                         t * 64 + in_tile % 32;
        lo[j] = o[0], hi[j] = o[32];
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float x[8] = {lo[j][0], lo[j][1], lo[j][2], lo[j][3], hi[j][0], hi[j][1], hi[j][2], hi[j][3]};
      fold(lj[j], 1.f, x);
    }
  }
  if constexpr (kPerRow > 1) {
    __shared__ float shared[kMergeThreads][11];
    float* mine = shared[tid];
    mine[0] = M, mine[1] = sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) mine[2 + e] = acc[e];
    __syncthreads();
    if (k > 0) return;
    for (int o = 1; o < kPerRow; ++o) {
      const float* other = shared[tid + o * 16 * kBlockRows];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = other[2 + e];
      fold(other[0], other[1], x);
    }
  }
  if (live) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t orow = size_t(s.row0 + node) * A.hq + size_t(s.g) * A.group + head;
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *reinterpret_cast<uint4*>(A.out + orow * kDim + 8 * t) = make_uint4(o[0], o[1], o[2], o[3]);
    if (A.lse && t == 0) A.lse[orow] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
  }
}

// Waves of a workgroup, 32 rows each; waves without rows only copy.  Four where an average sequence
// has 65 to 128 rows a KV head, eight otherwise.  A pass over 32 sequences of 3,000-5,000 tokens and 8
// KV heads, with four and with eight waves: 32 rows 98 and 99 us, 64 rows 110 and 109, 128 rows 125 and
// 136, 132 rows 200 and 150, 256 rows 231 and 185; trees of a 7B-class step, 35 to 112 rows, 125-129
// and 126; one sequence of 16,000 tokens, whose parts are fewer with eight, 38 and 28.  The mean tells
// nothing of a batch's largest trees: one of more than 128 rows has two tiles of four waves, which both
// read its keys and values.  64 requests of a 7B-class step with 1-24 nodes of 8 heads 162 and 154 us,
// 1-32 of 7 heads 176 and 158, 1-32 of 8 heads 180 and 162.
int64_t mean_rows(int64_t rows, int32_t batch, int32_t group) {
  return (rows + std::max(batch, 1) - 1) / std::max(batch, 1) * group;
}
int waves_of(int64_t rows, int32_t batch, int32_t group) {
  const int64_t mean = mean_rows(rows, batch, group);
  return mean > 64 && mean <= 128 ? 4 : 8;
}

// What an item costs besides its steps (queries, masked steps, results), in steps: ranges that span
// many short items otherwise end last.  A pass (attention and merge) at 6, 8, 10 and 12: 256 rows,
// requests of 4,096 tokens at the median 276, 274, 269 and 269 us, others of such lengths 283, 278, 276 and
// 276, 160 rows 223, 221, 219 and 220; trees of a 7B-class step 124, 124, 125 and 125, small trees 13.5
// at 6 and 13.9 at 9, 64 requests of 50-600 tokens 33.1 and 34.5.
int item_cost(int64_t rows, int32_t batch, int32_t group) {
  return mean_rows(rows, batch, group) > 128 ? 10 : 6;
}

TreeArgs tree_args(const KvLayout& L, const TreeCall& c, int waves) {
  TreeArgs A{};
  A.k_cache = static_cast<const uint16_t*>(L.desc.k_cache);
  A.v_cache = static_cast<const uint16_t*>(L.desc.v_cache);
  A.q = static_cast<const uint16_t*>(c.q);
  A.mask = c.mask, A.mask_words = c.mask_words;
  A.prior = c.prior, A.starts = c.starts, A.table = c.table, A.stride = c.stride;
  A.out = static_cast<uint16_t*>(c.out);
  A.lse = c.lse;
  const size_t part_rows = size_t(2) * groups_of(waves) * 32 * waves;
  A.part_o = static_cast<float*>(c.ws);
  A.part_lse = A.part_o + part_rows * kDim;
  A.splits = reinterpret_cast<Split*>(A.part_lse + part_rows);
  A.rows = int(c.rows);
  A.most = int(std::min<int64_t>(c.stride * kPage, INT32_MAX - 64));
  A.last_page = uint32_t(std::min<int64_t>(L.desc.num_pages - 1, INT32_MAX));
  A.item_cost = item_cost(c.rows, c.batch, c.hq / L.desc.num_kv_heads);
  A.batch = c.batch, A.hkv = L.desc.num_kv_heads, A.hq = c.hq, A.group = c.hq / A.hkv;
  A.sl2 = c.scale * kLog2e;
  return A;
}

}  // namespace

// One size for both forms, so that a workspace for the largest step is enough for every smaller one:
// their parts take the same bytes (groups_of(waves) * waves is fixed), the records those of more groups.
size_t tree_workspace() {
  constexpr size_t part_rows = size_t(2) * groups_of(8) * 32 * 8;
  static_assert(part_rows == size_t(2) * groups_of(4) * 32 * 4 && groups_of(4) > groups_of(8));
  return part_rows * (kDim + 1) * sizeof(float) + groups_of(4) * sizeof(Split);
}

hipError_t launch_tree(const KvLayout& L, const TreeCall& c, hipStream_t s) {
  const int waves = waves_of(c.rows, c.batch, c.hq / L.desc.num_kv_heads);
  const TreeArgs A = tree_args(L, c, waves);
  const dim3 grid{unsigned(groups_of(waves))}, block{unsigned(64 * waves)};
  if (waves == 4) hipLaunchKernelGGL(tree_ring_kernel<4>, grid, block, 0, s, A);
  else hipLaunchKernelGGL(tree_ring_kernel<8>, grid, block, 0, s, A);
  return hipGetLastError();
}

hipError_t launch_tree_merge(const KvLayout& L, const TreeCall& c, hipStream_t s) {
  const int waves = waves_of(c.rows, c.batch, c.hq / L.desc.num_kv_heads);
  const TreeArgs A = tree_args(L, c, waves);
  const int rows = 32 * waves, groups = groups_of(waves);
  // Items, at most, and with them the parts of one, about.
  const int64_t items = A.hkv * (int64_t(c.batch) + c.rows * A.group / rows);
  const int live = int(std::min<int64_t>(rows, c.rows * A.group));  // of a tile, at most
  auto launch = [&](auto kernel, int64_t x, int per_row) {
    const int y = (live * per_row + kMergeGroups - 1) / kMergeGroups;
    hipLaunchKernelGGL(kernel, dim3(unsigned(x), unsigned(y)), dim3(kMergeThreads), 0, s, A, groups, rows);
    return hipGetLastError();
  };
  // Groups of 16 threads to a row: 1, 4 and 16 took for 256 items of 256 rows 17, 37 and 179 us (with
  // some 4 of two events), 16 items 12, 9 and 17, 8 items 19, 10 and 13, one 107, 30 and 23.  The number
  // of items does not tell where one has most of the parts: with a request of 131,072 tokens among 63 of
  // 512-4,096 and 1, 2, 4 and 8 KV heads the merge takes 31, 60, 35 and 23 us, the attention 38, 64, 122
  // and 231.
  if (groups <= 4 * items) return launch(tree_merge_kernel<1>, groups, 1);
  if (groups <= 32 * items) return launch(tree_merge_kernel<4>, std::min<int64_t>(items, groups), 4);
  return launch(tree_merge_kernel<16>, std::min<int64_t>(items, groups), 16);
}

}  // namespace libra
