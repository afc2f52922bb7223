// Attention of drafted nodes over the paged cache: each of a sequence's N nodes sees its P cached
// tokens and, of the nodes cached behind them, those whose bits its mask sets.
//
// Lengths are read on the GPU, so the launch divides the work itself.  A KV head's N G (node, head)
// rows are cut into tiles of M = 32 kWaves rows, an item is a tile over all P + N keys, and a step
// is 32 keys of an item.  With S steps in all, workgroup w takes steps [w q, (w + 1) q) of the
// items in order, q = max(ceil(S / workgroups), kMinSteps): some whole items, and at most a part
// of one before and of one behind them.  Parts are float32 results, normalised, with their
// log-sum-exps in slots 2 w (an item begun by another workgroup) and 2 w + 1 (one that it begins and
// does not end); the merge finds an item's slots by the same arithmetic.  Neighbouring ranges run on
// one XCD, so that tiles of the same keys share its L2.
//
// A step's K and V tiles, two pages, are copied from memory straight into a four-stage LDS ring
// (global_load_lds_dwordx4: 16 bytes a lane, the tiles as stored) three steps ahead, across the
// ends of items, and shared by the waves.  Wave w holds 32 of the tile's rows as the columns of
// its products, on v_mfma_f32_32x32x16_bf16:
//   S^T[32 keys x 32 rows] = K Q^T: 8 products over the 128 channels; lane (key m, half h) reads K
//     granule (2 c + h) 16 + m % 16 of page m / 16 and gets the scores of keys 8 (r / 4) + 4 h + r % 4
//     (r = 0 .. 15) for its row;
//   O^T[128 channels x 32 rows] += V^T P^T: per page 4 products; a lane's probabilities of a page are
//     its operand as they come out of the scores, V granule 128 h + d the other.
// Softmax runs online in base 2 with the running maximum set on an item's first step and moved only
// when a lane's sum of 16 probabilities exceeds 2^kTau.  Probabilities enter the products as bf16,
// off by at most 2^-8 of each, their sum is taken in float32 before.
//
// Steps that reach past the cached tokens are masked: a row's 32 bits of them are its mask's, shifted.
// There the values may be those of nodes that a row does not see, or nothing; where any is not
// finite, a product of a zero probability would be NaN, and the step takes finite values only
// and adds the infinities and NaNs of seen nodes after (rare).
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
// Uniform reads of data that no launch here writes go through the scalar cache, whose counter is
// another than the copies'.
typedef const int32_t __attribute__((address_space(4))) * ScalarInts;

constexpr int kStepKeys = 32;
constexpr int kStages = 4;
constexpr int kMinSteps = 4;
constexpr int kTau = 8;
constexpr float kSumTau = float(1 << kTau);
constexpr int kMaskWords = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Workgroups of the launch: all that run at once.
constexpr int kCus = 256;
constexpr int groups_of(int waves) { return waves == 8 ? kCus : 2 * kCus; }

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
  int64_t stride;
  int64_t rows;
  uint32_t last_page;
  int batch, hkv, hq, group, mask_words;
  float sl2;
};

// A sequence's sizes, kept inside the rows and the block table whatever the caller's memory holds.
struct Seq {
  int prior, nodes, row0, len, steps, tiles;
  // The steps of all its items: one a tile and KV head.
  __device__ __forceinline__ int64_t cost(const TreeArgs& A) const { return int64_t(tiles) * A.hkv * steps; }
};
template <int kRows, class Ints>
__device__ __forceinline__ Seq load_seq(const TreeArgs& A, Ints prior, Ints starts, int b) {
  Seq s;
  const int64_t r0 = min(max(int64_t(starts[b]), int64_t(0)), A.rows);
  const int64_t r1 = min(max(int64_t(starts[b + 1]), r0), A.rows);
  s.row0 = int(r0), s.nodes = int(r1 - r0);
  const int64_t most = min(A.stride * kPage, int64_t(INT32_MAX) - 64);
  s.prior = int(min(int64_t(max(prior[b], 0)), most));
  s.len = int(min(int64_t(s.prior) + s.nodes, most));
  s.steps = (s.len + kStepKeys - 1) / kStepKeys;
  s.tiles = (s.nodes * A.group + kRows - 1) / kRows;  // rows * hq fits 32 bits
  return s;
}

// The launch's division: total steps, and steps per workgroup.
template <int kRows>
__device__ __forceinline__ int64_t total_steps(const TreeArgs& A, int lane) {
  int64_t sum = 0;
  for (int b = lane; b < A.batch; b += 64) sum += load_seq<kRows>(A, A.prior, A.starts, b).cost(A);
#pragma unroll
  for (int n = 32; n; n >>= 1) sum += __shfl_xor(sum, n);
  return uniform64(sum);
}
__device__ __forceinline__ int64_t steps_each(int64_t total, int groups) {
  return max((total + groups - 1) / groups, int64_t(kMinSteps));
}

// A place in the launch's steps.
template <int kRows>
struct Cursor {
  Seq seq;
  int b, g, tile, step;
  __device__ __forceinline__ void load(const TreeArgs& A) {
    seq = load_seq<kRows>(A, (ScalarInts)A.prior, (ScalarInts)A.starts, b);
  }
  // The sequence that holds step `at`, which is below the total.
  __device__ __forceinline__ void seek(const TreeArgs& A, int64_t at, int lane) {
    int64_t before = 0;
    for (int b0 = 0;; b0 += 64) {
      const int i = b0 + lane;
      const int64_t cost = i < A.batch ? load_seq<kRows>(A, A.prior, A.starts, i).cost(A) : 0;
      int64_t upto = cost;
#pragma unroll
      for (int n = 1; n < 64; n <<= 1) {
        const int64_t y = __shfl_up(upto, n);
        if (lane >= n) upto += y;
      }
      const uint64_t beyond = __ballot(before + upto > at);
      if (beyond || b0 + 64 >= A.batch) {
        const int l = beyond ? __builtin_ctzll(beyond) : 0;
        b = uniform(b0 + l);
        load(A);
        const int64_t in_seq = at - uniform64(before + __shfl(upto - cost, l));
        const int item = uniform(int(in_seq / seq.steps));
        step = uniform(int(in_seq - int64_t(item) * seq.steps));
        g = uniform(item / seq.tiles);
        tile = item - g * seq.tiles;
        return;
      }
      before += uniform64(__shfl(upto, 63));
    }
  }
  // To the next step; not past the launch's last one.
  __device__ __forceinline__ void advance(const TreeArgs& A) {
    if (++step < seq.steps) return;
    step = 0;
    if (++tile < seq.tiles) return;
    tile = 0;
    if (++g < A.hkv) return;
    g = 0;
    do {
      ++b;
      load(A);
    } while (seq.tiles == 0 && b + 1 < A.batch);
  }
};

template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(kWaves >= 4 ? 2 : 1, 2)))
void tree_kernel(TreeArgs A) {
  constexpr int kRows = 32 * kWaves;
  constexpr int kCopies = 16 / kWaves;  // of 1 KiB, per wave and step
  __shared__ __align__(16) uint4 ring[kStages][4][256];  // K of the step's two pages, V of them
  __shared__ uint32_t bits[kWaves][32][kMaskWords + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int G = A.group;

  // Neighbouring ranges on one XCD: workgroup w runs on XCD w % 8.
  const int per_xcd = int(gridDim.x) / kNumXcds;
  const int w = int(blockIdx.x) % kNumXcds * per_xcd + int(blockIdx.x) / kNumXcds;
  const int64_t total = total_steps<kRows>(A, lane);
  const int64_t each = steps_each(total, int(gridDim.x));
  const int64_t begin = w * each;
  if (begin >= total) return;
  const int n_steps = int(min(each, total - begin));

  Cursor<kRows> at, ahead;
  at.seek(A, begin, lane);
  ahead = at;
  const uint32_t page_bytes = uint32_t(A.hkv) * kTileBytes;
  // The page ids of the step that is copied next, loaded a step earlier.
  int id[2];
  auto load_ids = [&]() {
    const ScalarInts row = (ScalarInts)A.table + int64_t(ahead.b) * A.stride;
    const int p = 2 * ahead.step, last = (ahead.seq.len - 1) / kPage;
    id[0] = row[p];
    id[1] = row[min(p + 1, last)];
  };
  // This wave's part of a step: 1 KiB pieces of the tiles K 0, K 1, V 0, V 1.
  int copied = 0;
  auto copy_step = [&]() {
    uint64_t off[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
      off[p] = uint64_t(min(uint32_t(id[p]), A.last_page)) * page_bytes + uint32_t(ahead.g) * kTileBytes;
    uint4(&stage)[4][256] = ring[copied & (kStages - 1)];
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int piece = wave * kCopies + c, tile = piece >> 2, part = piece & 3;
      const char* src = reinterpret_cast<const char*>(tile < 2 ? A.k_cache : A.v_cache) +
                        off[tile & 1] + part * 1024 + lane * 16;
      const uint32_t dst = uint32_t(reinterpret_cast<uintptr_t>(&stage[tile][part * 64]));
      asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off"
                   :
                   : "s"(dst), "v"(src)
                   : "memory", "m0");
    }
    if (++copied < n_steps) {
      ahead.advance(A);
      load_ids();
    }
  };
  load_ids();
#pragma unroll 1
  for (int i = 0; i < kStages - 1 && copied < n_steps; ++i) copy_step();
  if (n_steps >= kStages - 1) wait_loads<(kStages - 2) * kCopies>();
  else wait_loads<0>();
  __syncthreads();

  bf16x8 qop[8];
  f32x16 acc[4];
  float m = -INFINITY, l = 0.f;
  int node = 0, head = 0, first_step = 0;
  bool ok = false;
#pragma unroll 1
  for (int n = 0; n < n_steps; ++n) {
    if (copied < n_steps) copy_step();
    const Seq& s = at.seq;
    const int g = at.g;
    const bool starts = n == 0 || at.step == 0;
    if (starts) {
      const int r = at.tile * kRows + 32 * wave + col;
      node = r / G, head = r - node * G;
      ok = node < s.nodes;
      first_step = at.step;
      const uint4* qrow = reinterpret_cast<const uint4*>(
          A.q + (size_t(s.row0 + (ok ? node : 0)) * A.hq + size_t(g) * G + head) * kDim);
#pragma unroll
      for (int c = 0; c < 8; ++c) qop[c] = as_bf16x8(ok ? qrow[2 * c + hh] : make_uint4(0, 0, 0, 0));
      if (A.mask)
        for (int i = hh; i < A.mask_words; i += 2)
          bits[wave][col][i] = ok ? A.mask[size_t(s.row0 + node) * A.mask_words + i] : 0;
      m = -INFINITY, l = 0.f;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2) acc[cb][r2] = 0.f;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const uint4(&stage)[4][256] = ring[n & (kStages - 1)];
    const int key0 = at.step * kStepKeys;
    const bool masked = key0 + kStepKeys > s.prior;  // uniform

    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          as_bf16x8(stage[col >> 4][(2 * c + hh) * 16 + (col & 15)]), qop[c], sc, 0, 0, 0);
    if (masked) {
      // Bit i: the row sees key key0 + i.
      uint32_t sees;
      const int d = key0 - s.prior;  // > -32: the first key's node
      if (!A.mask) {
        const int lim = node - d;
        sees = lim >= 31 ? ~0u : lim < 0 ? 0u : (2u << lim) - 1;
      } else if (d < 0) {
        sees = bits[wave][col][0] << -d | ((1u << -d) - 1);
      } else {
        const int i = d >> 5, sh = d & 31;
        const uint32_t w0 = i < A.mask_words ? bits[wave][col][i] : 0;
        const uint32_t w1 = i + 1 < A.mask_words ? bits[wave][col][i + 1] : 0;
        sees = uint32_t((uint64_t(w1) << 32 | w0) >> sh);
      }
      const int left = s.len - key0;
      if (left < 32) sees &= (1u << left) - 1;
      if (!ok) sees = 0;
      sees >>= 4 * hh;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(sees >> acc_row(r, 0) & 1)) sc[r] = -INFINITY;
    }
    auto rescale = [&]() {
      float mloc = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mloc = fmaxf(mloc, sc[r]);
      float mc = fmaxf(mloc * A.sl2, m);
      mc = fmaxf(mc, __shfl_xor(mc, 32));
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mc);
      l *= alpha;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) acc[cb] *= alpha;
      m = mc;
    };
    if (starts) rescale();
    // While a row has seen no finite score, the offset is the largest float: scores of -inf give 0,
    // and the first finite one infinity, which moves the maximum.
    float p[16], ps;
    auto take = [&]() {
      const float neg_m = m == -INFINITY ? FLT_MAX : -m;
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], A.sl2, neg_m));
      const float t0 = (p[0] + p[1]) + (p[2] + p[3]), t1 = (p[4] + p[5]) + (p[6] + p[7]);
      const float t2 = (p[8] + p[9]) + (p[10] + p[11]), t3 = (p[12] + p[13]) + (p[14] + p[15]);
      ps = (t0 + t1) + (t2 + t3);
    };
    take();
    if (__ballot(!(ps <= kSumTau))) {
      rescale();
      take();
    }
    l += ps;
    const bf16x8 pr[2] = {
        as_bf16x8(make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]),
                             pack_bf16x2(p[6], p[7]))),
        as_bf16x8(make_uint4(pack_bf16x2(p[8], p[9]), pack_bf16x2(p[10], p[11]),
                             pack_bf16x2(p[12], p[13]), pack_bf16x2(p[14], p[15])))};
    if (!masked) {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        acc[c & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(stage[2 + (c >> 2)][128 * hh + 32 * (c & 3) + col]), pr[c >> 2], acc[c & 3], 0, 0, 0);
    } else {
      // Slots past the end hold anything: zero.
      uint32_t keep[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int valid = s.len - key0 - j * kPage;
          const int s0 = 8 * (e / 2) + 4 * hh + 2 * (e % 2);
          keep[j][e] = (s0 < valid ? 0x0000FFFFu : 0u) | (s0 + 1 < valid ? 0xFFFF0000u : 0u);
        }
      auto value = [&](int cb, int j) {
        uint4 v = stage[2 + j][128 * hh + 32 * cb + col];
        v.x &= keep[j][0], v.y &= keep[j][1], v.z &= keep[j][2], v.w &= keep[j][3];
        return v;
      };
      auto has_special = [](uint32_t x) { return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u; };
#pragma unroll 1
      for (int cb2 = 0; cb2 < 4; ++cb2) {
        uint4 v[2];
        bool special = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          v[j] = value(cb2, j);
          special |= has_special(v[j].x) || has_special(v[j].y) || has_special(v[j].z) || has_special(v[j].w);
        }
        const bool any = __ballot(special) != 0;
        const uint4 raw[2] = {v[0], v[1]};
        if (any) {
          auto finite = [](uint32_t x) {
            return ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) |
                   ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
          };
#pragma unroll
          for (int j = 0; j < 2; ++j)
            v[j] = make_uint4(finite(v[j].x), finite(v[j].y), finite(v[j].z), finite(v[j].w));
        }
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          if (cb != cb2) continue;
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[j]), pr[j], acc[cb], 0, 0, 0);
          if (!any) continue;
          // The same products with 1 in the places of +inf, of -inf and of NaN: above 0 where the row
          // sees one.
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {
            const uint32_t lo = kind == 1 ? 0xFF80u : 0x7F80u;
            auto ones = [&](uint32_t x) {
              uint32_t o = 0;
#pragma unroll
              for (int half = 0; half < 32; half += 16) {
                const uint32_t e = x >> half & 0xFFFF;
                if (kind == 2 ? (e & 0x7FFF) > 0x7F80u : e == lo) o |= 0x3F80u << half;
              }
              return o;
            };
            f32x16 seen;
#pragma unroll
            for (int r = 0; r < 16; ++r) seen[r] = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
              seen = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  as_bf16x8(make_uint4(ones(raw[j].x), ones(raw[j].y), ones(raw[j].z), ones(raw[j].w))),
                  pr[j], seen, 0, 0, 0);
            const float put = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (seen[r] > 0.f) acc[cb][r] += put;
          }
        }
      }
    }

    const bool ends = at.step + 1 == s.steps;
    if (ends || n + 1 == n_steps) {
      // Row col's sum over both lane halves; a lane holds channels 32 cb + 8 e + 4 hh .. + 3.
      const float ls = l + __shfl_xor(l, 32);
      const float inv = ls > 0.f ? 1.f / ls : ls == 0.f ? 0.f : ls;  // a NaN stays
      if (first_step == 0 && ends) {
        if (ok) {
          const size_t orow = size_t(s.row0 + node) * A.hq + size_t(g) * G + head;
          uint16_t* o = A.out + orow * kDim + 4 * hh;
#pragma unroll
          for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<uint2*>(o + 32 * cb + 8 * e) =
                  make_uint2(pack_bf16x2(acc[cb][4 * e] * inv, acc[cb][4 * e + 1] * inv),
                             pack_bf16x2(acc[cb][4 * e + 2] * inv, acc[cb][4 * e + 3] * inv));
          if (A.lse && hh == 0) A.lse[orow] = ls == 0.f ? -INFINITY : (m + log2f(ls)) * kLn2;
        }
      } else {
        const size_t slot = size_t(2) * w + (first_step == 0 ? 1 : 0);
        const size_t prow = slot * kRows + 32 * wave + col;
        if (ok) {
          float* o = A.part_o + prow * kDim + 4 * hh;
#pragma unroll
          for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<f32x4*>(o + 32 * cb + 8 * e) =
                  f32x4{acc[cb][4 * e] * inv, acc[cb][4 * e + 1] * inv, acc[cb][4 * e + 2] * inv,
                        acc[cb][4 * e + 3] * inv};
          if (hh == 0) A.part_lse[prow] = ls == 0.f ? -INFINITY : m + log2f(ls);
        }
      }
    }
    if (n + 1 < n_steps) {
      at.advance(A);
      // Step n + 1's copies have landed; those of the two after it may be in flight.
      if (n + kStages - 1 < n_steps) wait_loads<(kStages - 2) * kCopies>();
      else wait_loads<0>();
      __syncthreads();
    }
  }
}

// Joins the parts of split items.  A workgroup takes a node's heads, `heads` of them at a time from
// blockIdx.y; 16 threads, eight channels each, fold an eighth part or all of a head's, as many
// groups to a head as its parts need.
constexpr int kMergeThreads = 256;
constexpr int kMergeGroups = kMergeThreads / 16;
constexpr int kMergeBatch = 4;

template <int kRows>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(TreeArgs A, int groups) {
  __shared__ int64_t found[kMergeThreads / 64][3];
  __shared__ __align__(16) float shared[kMergeGroups][16][12];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  // The row's sequence, the steps before it, and all steps.
  int64_t seqs = 0, before = 0, total = 0;
  for (int b = tid; b < A.batch; b += kMergeThreads) {
    const int64_t cost = load_seq<kRows>(A, A.prior, A.starts, b).cost(A);
    total += cost;
    if (A.starts[b + 1] <= row) ++seqs, before += cost;
  }
#pragma unroll
  for (int n = 32; n; n >>= 1) {
    seqs += __shfl_xor(seqs, n);
    before += __shfl_xor(before, n);
    total += __shfl_xor(total, n);
  }
  if (lane == 0) found[wave][0] = seqs, found[wave][1] = before, found[wave][2] = total;
  __syncthreads();
  seqs = before = total = 0;
#pragma unroll
  for (int w = 0; w < kMergeThreads / 64; ++w) seqs += found[w][0], before += found[w][1], total += found[w][2];
  if (seqs >= A.batch) return;  // padding
  const int b = int(seqs);
  const Seq s = load_seq<kRows>(A, A.prior, A.starts, b);
  // (Starts that do not ascend could put the sequence anywhere.)
  if (row < s.row0 || row >= s.row0 + s.nodes || before + s.cost(A) > total) return;
  const int64_t each = steps_each(total, groups);
  const int node = int(row - s.row0);
  // An item has at most this many parts; every group of a head folds kMergeBatch of them at a time.
  const int64_t most = (s.steps + each - 2) / each + 1;
  const int per_head = most <= kMergeBatch ? 1 : most <= 4 * kMergeBatch ? 4 : kMergeGroups;
  const int at_once = kMergeGroups / per_head;
  const int grp = tid >> 4, t = tid & 15, k = grp % per_head;
  for (int h0 = int(blockIdx.y) * at_once; h0 < A.hq; h0 += int(gridDim.y) * at_once) {
    const int h = h0 + grp / per_head;
    int64_t w0 = 0, w1 = 0;
    int in_tile = 0;
    if (h < A.hq) {
      const int g = h / A.group;
      const int r = node * A.group + (h - g * A.group);
      const int64_t first = before + (int64_t(g) * s.tiles + r / kRows) * s.steps;
      in_tile = r % kRows;
      w0 = first / each, w1 = (first + s.steps - 1) / each;
    }
    const int n = w0 == w1 ? 0 : int(w1 - w0) + 1;
    float M = -INFINITY, sum = 0.f, acc[8] = {};
    auto fold = [&](float Mk, float wk, const float (&xk)[8]) {
      // A NaN moves no maximum, but makes both factors' sums NaN.
      const float Mn = fmaxf(M, Mk);
      const float a = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
      const float c = Mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(Mk - Mn);
      sum = sum * a + wk * c;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = (a == 0.f ? 0.f : acc[i] * a) + (c == 0.f ? 0.f : xk[i] * c);
      M = Mn;
    };
    for (int j0 = k * kMergeBatch; j0 < n; j0 += per_head * kMergeBatch) {
      float lj[kMergeBatch], x[kMergeBatch][8];
#pragma unroll
      for (int j = 0; j < kMergeBatch; ++j) {
        lj[j] = -INFINITY;
        if (j0 + j < n) {
          const size_t slot = j0 + j == 0 ? size_t(2) * w0 + 1 : size_t(2) * (w0 + j0 + j);
          lj[j] = A.part_lse[slot * kRows + in_tile];
          const f32x4* o = reinterpret_cast<const f32x4*>(A.part_o + (slot * kRows + in_tile) * kDim + 8 * t);
          const f32x4 lo = o[0], hi = o[1];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[j][i] = lo[i], x[j][4 + i] = hi[i];
        }
      }
#pragma unroll
      for (int j = 0; j < kMergeBatch; ++j)
        if (j0 + j < n) fold(lj[j], 1.f, x[j]);
    }
    if (per_head > 1) {
      float* mine = shared[grp][t];
      mine[0] = M, mine[1] = sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) mine[2 + i] = acc[i];
      __syncthreads();
      if (k == 0)
        for (int o = 1; o < per_head; ++o) {
          const float* other = shared[grp + o][t];
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = other[2 + i];
          fold(other[0], other[1], x);
        }
      __syncthreads();
    }
    if (k == 0 && n > 0) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const size_t orow = size_t(row) * A.hq + h;
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
      *reinterpret_cast<uint4*>(A.out + orow * kDim + 8 * t) = make_uint4(o[0], o[1], o[2], o[3]);
      if (A.lse && t == 0) A.lse[orow] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
    }
  }
}

// Waves of a workgroup, 32 rows each: enough for the rows of an average sequence's KV head.
int waves_of(int64_t rows, int32_t batch, int32_t group) {
  const int64_t mean = (rows + std::max(batch, 1) - 1) / std::max(batch, 1) * group;
  return mean <= 32 ? 1 : mean <= 64 ? 2 : mean <= 128 ? 4 : 8;
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
  A.rows = c.rows;
  A.last_page = uint32_t(std::min<int64_t>(L.desc.num_pages - 1, INT32_MAX));
  A.batch = c.batch, A.hkv = L.desc.num_kv_heads, A.hq = c.hq, A.group = c.hq / A.hkv;
  A.sl2 = c.scale * kLog2e;
  return A;
}

}  // namespace

size_t tree_workspace(int64_t rows, int32_t batch, int32_t hq, int32_t hkv) {
  const int waves = waves_of(rows, batch, hq / hkv);
  return size_t(2) * groups_of(waves) * 32 * waves * (kDim + 1) * sizeof(float);
}

hipError_t launch_tree(const KvLayout& L, const TreeCall& c, hipStream_t s) {
  const int waves = waves_of(c.rows, c.batch, c.hq / L.desc.num_kv_heads);
  const TreeArgs A = tree_args(L, c, waves);
  const dim3 grid{unsigned(groups_of(waves))}, block{unsigned(64 * waves)};
  switch (waves) {
    case 1: hipLaunchKernelGGL(tree_kernel<1>, grid, block, 0, s, A); break;
    case 2: hipLaunchKernelGGL(tree_kernel<2>, grid, block, 0, s, A); break;
    case 4: hipLaunchKernelGGL(tree_kernel<4>, grid, block, 0, s, A); break;
    default: hipLaunchKernelGGL(tree_kernel<8>, grid, block, 0, s, A); break;
  }
  return hipGetLastError();
}

hipError_t launch_tree_merge(const KvLayout& L, const TreeCall& c, hipStream_t s) {
  const int waves = waves_of(c.rows, c.batch, c.hq / L.desc.num_kv_heads);
  const TreeArgs A = tree_args(L, c, waves);
  const int groups = groups_of(waves);
  // Few rows: their heads over more workgroups.
  const unsigned y = unsigned(std::clamp<int64_t>(2048 / c.rows, 1, c.hq));
  const dim3 grid{unsigned(c.rows), y}, block{unsigned(kMergeThreads)};
  switch (waves) {
    case 1: hipLaunchKernelGGL(tree_merge_kernel<32>, grid, block, 0, s, A, groups); break;
    case 2: hipLaunchKernelGGL(tree_merge_kernel<64>, grid, block, 0, s, A, groups); break;
    case 4: hipLaunchKernelGGL(tree_merge_kernel<128>, grid, block, 0, s, A, groups); break;
    default: hipLaunchKernelGGL(tree_merge_kernel<256>, grid, block, 0, s, A, groups); break;
  }
  return hipGetLastError();
}

}  // namespace libra
