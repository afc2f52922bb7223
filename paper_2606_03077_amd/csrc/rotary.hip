// Rotary positions of dense rows, and the cache append that turns keys on the way.
//
// Both are bound by HBM (each value is read and written once), or by the launch for few rows.  A
// thread turns four pairs, whose cosines and sines (about 26 instructions each) it computes once
// for up to four heads; a table of them would be read instead.  40,960 rows of 40 heads (bf16,
// 839 MB) take 137 us, 6.1 TB/s; their append with 8 KV heads 214 us, 5.5 TB/s; a copy of as
// much runs at 4.9-5.4 TB/s on the same card.  16 rows of 28 heads: 3.0 us, an append of 64
// rows 4.8 us.
//
// An append whose R is no multiple of 8 (kAnyPairs) is bound by its vector work instead: the
// long append takes 609 us at R = 20 in half pairing, 537 interleaved.  Each head works out its
// rows' cosines and sines anew, and in half pairing a granule's partners are eight loads of two
// bytes.
//
// Heads may be normalised before they are turned (kNorm, norm_*): the sum of squares is a reduction
// over the lanes that hold the head, so a value is still read and written once.  16,381 rows of 40
// query and 8 key heads (bf16): alone 76 us, 5.3 TB/s; on their way into the cache 106 us, 4.5 TB/s,
// where the V tiles' transposition costs LDS conflicts besides; 16 rows 6 us, a chain of loads.  An
// append whose R is no multiple of 8 is bound by its vector work (cosines of every head and channel,
// weights one at a time): 267 us at R = 20 in either pairing.
#include <algorithm>
#include <type_traits>

#include "drafts.h"
#include "row_types.h"

namespace libra {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = kMaxRotaryDim / 2;

// Rows x heads to turn, for both forms below.
template <class T>
struct RowsArgs {
  const typename T::Elem* x;
  typename T::Elem* out;
  int64_t x_row, x_head, out_row, out_head;
  const int32_t* positions;
  const int64_t* slots;  // rows whose slot lies outside [0, slot_end) are left out (null: none)
  int64_t slot_end;
  int64_t rows;
  int heads, dim;
  int backward;
  // The wide form's block: per_row = per_head * head_slots threads take a row, each one of its
  // eight-channel pieces in up to kHeads heads, head_slots apart; y_blocks blocks share a row.
  int per_head, head_slots, per_row, block_rows, y_blocks;
};

template <class T>
__device__ __forceinline__ bool skipped(const RowsArgs<T>& A, int64_t row) {
  return A.slots && uint64_t(A.slots[row]) >= uint64_t(A.slot_end);
}

// Two quads of a head normalised over its `lanes` threads' quads, and turned if they are.
template <class T, bool kInter>
__device__ __forceinline__ void norm_quads(typename T::Quad& a, typename T::Quad& b,
                                           const float (&wa)[4], const float (&wb)[4], int lanes,
                                           int dim, float eps, bool turned, const float2 (&cs)[4]) {
  float f[4], g[4], y[4], z[4], squares = 0.f;
  T::unpack(a, f);
  T::unpack(b, g);
#pragma unroll
  for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(f[e], f[e], squares);
#pragma unroll
  for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(g[e], g[e], squares);
  const float r = norm_scale(group_sum(squares, lanes), dim, eps);
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = f[e] * r * wa[e], g[e] = g[e] * r * wb[e];
  if (turned) {
    turn_values<kInter>(f, g, cs, y, z);
    a = T::pack(y), b = T::pack(z);
  } else {
    a = T::pack(f), b = T::pack(g);
  }
}

constexpr int64_t kStreamBytes = int64_t(128) << 20;  // written by a call whose writes go past

// What goes past the caches: nothing, the reads (each value is read once), or both.
enum Streaming : int { kCached, kReads, kReadsWrites };

// Wide form: R and the head size are multiples of 8, rows are aligned for four channels at a
// time.  A thread owns two quads of a head (4 pairs, or 8 copied channels), computes their
// cosines and sines once, and turns them in up to kHeads heads.
// kNorm: the heads are normalised first (their size is a power of two then, so that a head's
// threads are an aligned group of lanes, of which all take part or none).
template <class T, bool kInter, int kHeads, Streaming kStream, bool kNorm = false, class Rot>
__device__ __forceinline__ void turn_rows_wide(const Rot& rot, const RowsArgs<T>& A, int64_t bx,
                                               int by, [[maybe_unused]] const HeadNorm& norm = {}) {
  using Quad = typename T::Quad;
  const int t = threadIdx.x;
  const int r = t / A.per_row, in_row = t - r * A.per_row;
  const int h0 = in_row / A.per_head, j = in_row - h0 * A.per_head;
  const int64_t row = bx * A.block_rows + r;
  if (r >= A.block_rows || row >= A.rows || skipped(A, row)) return;
  const int R8 = rot.rdim / 8;
  const bool turned = j < R8;
  if (!kNorm && !turned && A.x == A.out) return;
  const int2 qd = quads_of<T, kInter>(j, R8, A.per_head);
  const int head0 = by * A.head_slots * kHeads + h0;
  const typename T::Elem* x = A.x + row * A.x_row;
  typename T::Elem* out = A.out + row * A.out_row;
  Quad a[kHeads], b[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = head0 + i * A.head_slots;
    if (h < A.heads) {
      a[i] = load_quad<kStream != kCached>(reinterpret_cast<const Quad*>(x + h * A.x_head + 4 * qd.x));
      b[i] = load_quad<kStream != kCached>(reinterpret_cast<const Quad*>(x + h * A.x_head + 4 * qd.y));
    }
  }
  [[maybe_unused]] float wa[4], wb[4];
  if constexpr (kNorm) {
    norm_weights(norm, 4 * qd.x, wa);
    norm_weights(norm, 4 * qd.y, wb);
  }
  float2 cs[4];
  if (turned) {
    const int32_t pos = A.positions[row];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cs[i] = rotary_cos_sin(rot.turn[pair_of<kInter>(qd, j, i)], pos, rot.amplitude);
      if (A.backward) cs[i].y = -cs[i].y;
    }
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = head0 + i * A.head_slots;
    if (h < A.heads) {
      if constexpr (kNorm) norm_quads<T, kInter>(a[i], b[i], wa, wb, A.per_head, A.dim, norm.eps, turned, cs);
      else if (turned) turn_quads<T, kInter>(a[i], b[i], cs);
      store_quad<kStream == kReadsWrites>(reinterpret_cast<Quad*>(out + h * A.out_head + 4 * qd.x), a[i]);
      store_quad<kStream == kReadsWrites>(reinterpret_cast<Quad*>(out + h * A.out_head + 4 * qd.y), b[i]);
    }
  }
}

// Narrow form: any even R, any alignment.  A thread owns one pair (or one copied channel) of
// a row, in every kNarrowHeads heads of its block row.
constexpr int kNarrowHeads = 8;
template <class T, class Rot>
__device__ __forceinline__ void turn_rows_narrow(const Rot& rot, const RowsArgs<T>& A, int64_t bx,
                                                 int by) {
  const int half = rot.rdim / 2;
  const int items = A.dim - half;
  const int64_t idx = bx * kThreads + threadIdx.x;
  const int64_t row = idx / items;
  const int j = int(idx - row * items);
  if (row >= A.rows || skipped(A, row)) return;
  const typename T::Elem* x = A.x + row * A.x_row;
  typename T::Elem* out = A.out + row * A.out_row;
  const int h0 = by * kNarrowHeads;
  const bool turned = j < half;
  if (!turned && A.x == A.out) return;
  const int d1 = !turned ? j + half : rot.interleaved ? 2 * j : j;
  const int d2 = !turned ? d1 : rot.interleaved ? 2 * j + 1 : j + half;
  typename T::Elem e1[kNarrowHeads], e2[kNarrowHeads];
#pragma unroll
  for (int i = 0; i < kNarrowHeads; ++i) {
    const int64_t h = min(h0 + i, A.heads - 1);
    e1[i] = x[h * A.x_head + d1];
    e2[i] = x[h * A.x_head + d2];
  }
  float2 cs = make_float2(1.f, 0.f);
  if (turned) cs = rotary_cos_sin(rot.turn[j], A.positions[row], rot.amplitude);
  if (A.backward) cs.y = -cs.y;
#pragma unroll
  for (int i = 0; i < kNarrowHeads; ++i) {
    const int64_t h = h0 + i;
    if (h >= A.heads) break;
    const float x1 = T::get(e1[i]), x2 = T::get(e2[i]);
    out[h * A.out_head + d1] = turned ? T::put(turn_first(x1, x2, cs)) : e1[i];
    if (turned) out[h * A.out_head + d2] = T::put(turn_second(x1, x2, cs));
  }
}

template <class T, bool kInter, int kHeads, Streaming kStream>
__global__ __launch_bounds__(kThreads) void rotary_wide_kernel(RotaryArgs<kMaxPairs> rot,
                                                               RowsArgs<T> A) {
  turn_rows_wide<T, kInter, kHeads, kStream>(rot, A, blockIdx.x, blockIdx.y);
}
template <class T>
__global__ __launch_bounds__(kThreads) void rotary_narrow_kernel(RotaryArgs<kMaxPairs> rot,
                                                                 RowsArgs<T> A) {
  turn_rows_narrow(rot, A, blockIdx.x, blockIdx.y);
}

// Queries' rows, then keys', both normalised: q_blocks blocks for the first.
template <class T, bool kInter, int kHeads, Streaming kStream>
__global__ __launch_bounds__(kThreads) void norm_rotary_wide_kernel(RotaryArgs<kMaxPairs> rot, RowsArgs<T> Q,
                                                                    RowsArgs<T> K, RowNorms norms, int q_blocks) {
  const int i = int(blockIdx.x);
  if (i < q_blocks)
    turn_rows_wide<T, kInter, kHeads, kStream, true>(rot, Q, i / Q.y_blocks, i % Q.y_blocks, norms.q);
  else
    turn_rows_wide<T, kInter, kHeads, kStream, true>(rot, K, (i - q_blocks) / K.y_blocks, (i - q_blocks) % K.y_blocks, norms.k);
}

// Any head size, R, alignment: a wave per head.  Its values go through LDS, where a channel finds
// its partner; all are read before one is written, so in place is fine.
template <class T>
__device__ __forceinline__ void norm_rows_any(const RotaryArgs<kMaxPairs>& rot, const RowsArgs<T>& A,
                                              int64_t vector, const HeadNorm& norm, float* u) {
  const int lane = threadIdx.x & 63;
  const int64_t row = vector / A.heads;
  const int h = int(vector - row * A.heads);
  if (row >= A.rows) return;
  const typename T::Elem* x = A.x + row * A.x_row + h * A.x_head;
  for (int d = lane; d < A.dim; d += 64) u[d] = T::get(x[d]);
  auto wave_sync = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  wave_sync();
  float squares = 0.f;  // eight channels a lane, as the cache append adds them
#pragma unroll
  for (int e = 0; e < kMaxRotaryHead / 64; ++e)
    if (8 * lane + e < A.dim) squares = __builtin_fmaf(u[8 * lane + e], u[8 * lane + e], squares);
  const float r = norm_scale(group_sum(squares, 64), A.dim, norm.eps);
  wave_sync();
  for (int d = lane; d < A.dim; d += 64) u[d] = u[d] * r * norm_weight(norm, d);
  wave_sync();
  const int32_t pos = A.positions[row];
  typename T::Elem* out = A.out + row * A.out_row + h * A.out_head;
  for (int d = lane; d < A.dim; d += 64) {
    float y = u[d];
    if (d < rot.rdim) {
      const bool first = rot.interleaved ? !(d & 1) : d < rot.rdim / 2;
      const int o = rot.interleaved ? d ^ 1 : first ? d + rot.rdim / 2 : d - rot.rdim / 2;
      const float2 cs = rotary_cos_sin(rot.turn[rot.interleaved ? d / 2 : first ? d : o], pos, rot.amplitude);
      y = first ? turn_first(y, u[o], cs) : turn_second(u[o], y, cs);
    }
    out[d] = T::put(y);
  }
}
template <class T>
__global__ __launch_bounds__(kThreads) void norm_rotary_any_kernel(RotaryArgs<kMaxPairs> rot, RowsArgs<T> Q,
                                                                   RowsArgs<T> K, RowNorms norms, int q_blocks) {
  __shared__ float u[kThreads / 64][kMaxRotaryHead];
  const int wave = threadIdx.x >> 6, i = int(blockIdx.x);
  const int64_t at = i < q_blocks ? i : i - q_blocks;
  norm_rows_any<T>(rot, i < q_blocks ? Q : K, at * (kThreads / 64) + wave, i < q_blocks ? norms.q : norms.k, u[wave]);
}

constexpr int64_t kMaxBlocks = int64_t(1) << 22;  // per launch: 2^30 threads

// How rows x heads are cut: the form, heads per thread, rows per block.
template <class T>
struct RowsPlan {
  RowsArgs<T> args;
  bool wide, many, lines, stream;
  int threads;
  // Blocks along x for `rows` rows, and the rows that n of them take.
  int64_t blocks(int64_t rows) const {
    return wide ? (rows + args.block_rows - 1) / args.block_rows
                : (rows * items() + kThreads - 1) / kThreads;
  }
  int64_t rows_of(int64_t n) const { return wide ? n * args.block_rows : n * kThreads / items(); }
  int64_t items() const { return args.dim - half; }
  int half;
};

// many: whether threads take several heads (-1: by the rule below).
template <class T>
RowsPlan<T> plan_rows(const Rotary& r, const RotaryRows& a, int many = -1) {
  RowsPlan<T> p{};
  RowsArgs<T>& A = p.args;
  A.x = static_cast<const typename T::Elem*>(a.x);
  A.out = static_cast<typename T::Elem*>(a.out);
  A.x_row = a.x_row, A.x_head = a.x_head, A.out_row = a.out_row, A.out_head = a.out_head;
  A.positions = a.positions;
  A.rows = a.rows;
  A.heads = a.heads, A.dim = r.head_dim;
  A.backward = a.backward;
  A.per_head = r.head_dim / 8;
  const size_t quad = sizeof(typename T::Quad);
  p.wide = r.rotary_dim % 8 == 0 && r.head_dim % 8 == 0 &&
           (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) % quad == 0 &&
           ((a.x_row | a.x_head | a.out_row | a.out_head) & 3) == 0;
  // Four heads to a thread share its cosines and sines, which pays once the chip is full and a
  // row has heads enough: 40,960 rows of 40 heads (bf16) 168 us against 197 with one head each
  // and 177 with two, of 28 heads 125 (143, 123); but 1,024 rows of 28 heads 9.0 us against 8.6,
  // 16 rows 6.4 against 6.1, 40,960 rows of 8 heads 46 against 45 (cold caches, launch included).
  p.many = many >= 0 ? many != 0 : a.heads >= 16 && a.rows * a.heads * A.per_head >= int64_t(2560) * kThreads;
  // Nothing goes past the caches where an instruction covers half lines (128 bytes), as half
  // pairing of 64 16-bit channels does: 40,960 rows of 40 heads 168 us so, 151 through them.
  p.lines = (r.pairing == LIBRA_ROTARY_INTERLEAVED && quad == 8) ||
            r.rotary_dim / 2 * sizeof(typename T::Elem) % 128 == 0;
  // More than the last-level cache (256 MiB) would hold of both sides: the result goes past it
  // too.  Turned and then copied, 16,384 rows of 40 heads (160 MiB a side) take 111 us so, 125
  // through the caches, 40,960 rows 290 and 303; but 8,192 rows (80 MiB) 58 and 54.
  p.stream = p.many && p.lines &&
             a.rows * a.heads * r.head_dim * int64_t(sizeof(typename T::Elem)) >= kStreamBytes;
  const int per_thread = p.many ? 4 : 1;
  p.threads = kThreads;
  A.y_blocks = (a.heads + kNarrowHeads - 1) / kNarrowHeads;
  p.half = r.rotary_dim / 2;
  if (p.wide) {
    // As few blocks to a row as its heads need, with even shares.
    const int most = kThreads / A.per_head * per_thread;
    A.y_blocks = (a.heads + most - 1) / most;
    A.head_slots = (a.heads + A.y_blocks * per_thread - 1) / (A.y_blocks * per_thread);
    A.per_row = A.head_slots * A.per_head;
    A.block_rows = kThreads / A.per_row;
    p.threads = A.per_row * A.block_rows;
  }
  return p;
}

template <class T>
hipError_t apply(const Rotary& r, const RotaryRows& a, hipStream_t s) {
  const RowsPlan<T> p = plan_rows<T>(r, a);
  const RotaryArgs<kMaxPairs> rot = rotary_args<kMaxPairs>(r);
  const int64_t step = p.rows_of(kMaxBlocks);
  for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
    RowsArgs<T> A = p.args;
    A.rows = std::min(step, a.rows - r0);
    A.x += r0 * a.x_row;
    A.out += r0 * a.out_row;
    A.positions += r0;
    const dim3 grid(unsigned(p.blocks(A.rows)), unsigned(A.y_blocks));
    const bool inter = r.pairing == LIBRA_ROTARY_INTERLEAVED;
    auto wide_form = [&](auto pairing) {
      constexpr bool kInter = decltype(pairing)::value;
      return !p.many    ? rotary_wide_kernel<T, kInter, 1, kCached>
             : p.stream ? rotary_wide_kernel<T, kInter, 4, kReadsWrites>
             : p.lines  ? rotary_wide_kernel<T, kInter, 4, kReads>
                        : rotary_wide_kernel<T, kInter, 4, kCached>;
    };
    auto k = !p.wide ? rotary_narrow_kernel<T>
             : inter ? wide_form(std::true_type{})
                     : wide_form(std::false_type{});
    hipLaunchKernelGGL(k, grid, dim3(unsigned(p.threads)), 0, s, rot, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Queries and keys in one launch (a tensor without heads takes no blocks).
template <class T>
hipError_t apply_norm(const Rotary& r, const RotaryRows& q, const RotaryRows& k, const RowNorms& norms,
                      hipStream_t s) {
  const int dim = r.head_dim, heads = q.heads + k.heads;
  // Four heads to a thread as for the turn alone (plan_rows), over both tensors' heads.
  const bool many = heads >= 16 && q.rows * heads * (dim / 8) >= int64_t(2560) * kThreads;
  // A tensor without heads is planned as the other, and gets no blocks.
  const RowsPlan<T> pq = plan_rows<T>(r, q.heads ? q : k, many), pk = plan_rows<T>(r, k.heads ? k : q, many);
  const bool wide = (dim & (dim - 1)) == 0 && pq.wide && pk.wide;
  const bool inter = r.pairing == LIBRA_ROTARY_INTERLEAVED;
  const bool lines = pq.lines;
  const bool stream = many && lines && q.rows * heads * dim * int64_t(sizeof(typename T::Elem)) >= kStreamBytes;
  auto wide_form = [&](auto pairing) {
    constexpr bool kInter = decltype(pairing)::value;
    return !many    ? norm_rotary_wide_kernel<T, kInter, 1, kCached>
           : stream ? norm_rotary_wide_kernel<T, kInter, 4, kReadsWrites>
           : lines  ? norm_rotary_wide_kernel<T, kInter, 4, kReads>
                    : norm_rotary_wide_kernel<T, kInter, 4, kCached>;
  };
  auto form = !wide ? norm_rotary_any_kernel<T> : inter ? wide_form(std::true_type{}) : wide_form(std::false_type{});
  const RotaryArgs<kMaxPairs> rot = rotary_args<kMaxPairs>(r);
  auto blocks = [&](const RowsPlan<T>& p, int of, int64_t rows) -> int64_t {
    if (!of) return 0;
    return wide ? p.blocks(rows) * p.args.y_blocks : (rows * p.args.heads + kThreads / 64 - 1) / (kThreads / 64);
  };
  // Both tensors' blocks of a launch stay in 32 bits: a row has at most 2 * 65,535 heads.
  const int64_t step = std::max<int64_t>(1, kMaxBlocks * (kThreads / 64) / heads);
  for (int64_t r0 = 0; r0 < q.rows; r0 += step) {
    RowsArgs<T> A[2] = {pq.args, pk.args};
    for (RowsArgs<T>& a : A) {
      a.rows = std::min(step, q.rows - r0);
      a.x += r0 * a.x_row;
      a.out += r0 * a.out_row;
      a.positions += r0;
    }
    const int64_t nq = blocks(pq, q.heads, A[0].rows), nk = blocks(pk, k.heads, A[0].rows);
    hipLaunchKernelGGL(form, dim3(unsigned(nq + nk)), dim3(kThreads), 0, s, rot, A[0], A[1], norms, int(nq));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// --- cache append ------------------------------------------------------------------------

struct WriteArgs {
  uint16_t* k_cache;
  uint16_t* v_cache;
  const uint16_t* k_new;
  const uint16_t* v_new;
  int64_t k_row, v_row;
  const int32_t* positions;
  int hkv;
  // by slots
  const int64_t* slots;
  int64_t slot_end;
  int64_t rows;
  int64_t first_block;  // of 16 rows
  int kv_blocks;        // blocks of this launch that write the cache; the others turn queries
  // by an append plan's records
  const int32_t* writes;
  const int32_t* bt;
  int64_t bt_stride;
};
using Rot = RotaryArgs<kRotaryPairs>;  // rdim 0: keys are copied

// How a key is turned: quads in half or interleaved pairing (R a multiple of 8; copies are
// interleaved quads of which none turns), or granules whose pairs may lie anywhere.
enum KeyForm : int { kHalfQuads, kInterQuads, kAnyPairs };

// What thread j of a row's 16 holds of it, for one KV head: eight channels of the key (two
// quads; not used by kAnyPairs, which reads them when it turns them) and of the value.
struct NewPiece {
  uint2 a, b;
  uint4 v;
  int32_t pos;
};

template <int kForm>
__device__ __forceinline__ NewPiece load_piece(const WriteArgs& A, const Rot& rot, int64_t row,
                                               int g, int j) {
  NewPiece p;
  const uint16_t* k = A.k_new + row * A.k_row + g * kDim;
  if constexpr (kForm != kAnyPairs) {
    const int2 qd = quads_of<Bf16, kForm == kInterQuads>(j, rot.rdim / 8, kDim / 8);
    p.a = *reinterpret_cast<const uint2*>(k + 4 * qd.x);
    p.b = *reinterpret_cast<const uint2*>(k + 4 * qd.y);
  }
  p.v = *reinterpret_cast<const uint4*>(A.v_new + row * A.v_row + g * kDim + 8 * j);
  p.pos = rot.rdim && A.positions ? A.positions[row] : 0;
  return p;
}

// Granule j of a bf16 row whose pairs may lie anywhere.  The 16 threads of a row, in one wave,
// share the row's cosines and sines through cs; all of them read before any of them writes.
__device__ __forceinline__ uint4 turn_any_granule(const Rot& rot, const uint16_t* row, int j,
                                                  int32_t pos, float2* cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4 * j + i < rot.rdim / 2)
      cs[4 * j + i] = rotary_cos_sin(rot.turn[4 * j + i], pos, rot.amplitude);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int gi[1] = {j};
  Granules<1> in;
  uint4 out[1], none[1];
  load_granules(in, row, gi, rot.rdim, rot.interleaved);
  turn_granules<1, false>(in, gi, cs, rot.rdim, rot.interleaved, out, none);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return out[0];
}

// Granule j of a row that is normalised before it is turned, its pairs anywhere; u: the row.
__device__ __forceinline__ uint4 norm_any_granule(const Rot& rot, const uint16_t* row, int j, int32_t pos,
                                                  const HeadNorm& norm, float* u) {
  const uint4 x = *reinterpret_cast<const uint4*>(row + 8 * j);
  float f[4], g[4], squares = 0.f;
  Bf16::unpack(make_uint2(x.x, x.y), f);
  Bf16::unpack(make_uint2(x.z, x.w), g);
#pragma unroll
  for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(f[e], f[e], squares);
#pragma unroll
  for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(g[e], g[e], squares);
  const float r = norm_scale(group_sum(squares, kDim / 8), kDim, norm.eps);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    u[8 * j + e] = f[e] * r * norm_weight(norm, 8 * j + e);
    u[8 * j + 4 + e] = g[e] * r * norm_weight(norm, 8 * j + 4 + e);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float y[8];
  const int half = rot.rdim / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = 8 * j + e;
    y[e] = u[d];
    if (d < rot.rdim) {
      const bool first = rot.interleaved ? !(d & 1) : d < half;
      const int o = rot.interleaved ? d ^ 1 : first ? d + half : d - half;
      const float2 cs = rotary_cos_sin(rot.turn[rot.interleaved ? d / 2 : first ? d : o], pos, rot.amplitude);
      y[e] = first ? turn_first(y[e], u[o], cs) : turn_second(u[o], y[e], cs);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return make_uint4(rotary_pack_bf16(y[0], y[1]), rotary_pack_bf16(y[2], y[3]),
                    rotary_pack_bf16(y[4], y[5]), rotary_pack_bf16(y[6], y[7]));
}

// 16 rows of one query head, any pairs.
__device__ __forceinline__ void norm_queries_any(const Rot& rot, const RowsArgs<Bf16>& A, int64_t bx,
                                                 int head, const HeadNorm& norm, float (*u)[kDim]) {
  const int s = threadIdx.x >> 4, j = threadIdx.x & 15;
  const int64_t row = bx * kPage + s;
  if (row >= A.rows || skipped(A, row)) return;
  const uint4 y = norm_any_granule(rot, A.x + row * A.x_row + int64_t(head) * kDim, j, A.positions[row], norm, u[s]);
  *reinterpret_cast<uint4*>(A.out + row * A.out_row + int64_t(head) * kDim + 8 * j) = y;
}
__device__ __forceinline__ void turn_queries_any(const Rot& rot, const RowsArgs<Bf16>& A, int64_t bx,
                                                 int head, float2 (*cs)[kRotaryPairs]) {
  const int s = threadIdx.x >> 4, j = threadIdx.x & 15;
  const int64_t row = bx * kPage + s;
  if (row >= A.rows || skipped(A, row)) return;
  const uint4 y = turn_any_granule(rot, A.x + row * A.x_row + int64_t(head) * kDim, j, A.positions[row], cs[s]);
  *reinterpret_cast<uint4*>(A.out + row * A.out_row + int64_t(head) * kDim + 8 * j) = y;
}

// Turns the piece's key (normalised first if kNorm: all 16 threads of the row take part) and stores
// it to slot s of the K tile.  cs: the row's part of LDS (kAnyPairs).
template <int kForm, bool kNorm = false>
__device__ __forceinline__ void store_key(const WriteArgs& A, const Rot& rot, const NewPiece& p,
                                          int64_t row, int g, int j, int s, uint16_t* tile,
                                          float2* cs, [[maybe_unused]] const HeadNorm& norm = {}) {
  if constexpr (kForm == kAnyPairs && kNorm) {
    *reinterpret_cast<uint4*>(tile + k_off(s, 8 * j)) = norm_any_granule(
        rot, A.k_new + row * A.k_row + g * kDim, j, p.pos, norm, reinterpret_cast<float*>(cs));
  } else if constexpr (kForm == kAnyPairs) {
    *reinterpret_cast<uint4*>(tile + k_off(s, 8 * j)) =
        turn_any_granule(rot, A.k_new + row * A.k_row + g * kDim, j, p.pos, cs);
  } else {
    constexpr bool kInter = kForm == kInterQuads;
    const int2 qd = quads_of<Bf16, kInter>(j, rot.rdim / 8, kDim / 8);
    uint2 a = p.a, b = p.b;
    const bool turned = j < rot.rdim / 8;
    float2 t[4];
    if (turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t[i] = rotary_cos_sin(rot.turn[pair_of<kInter>(qd, j, i)], p.pos, rot.amplitude);
    }
    if constexpr (kNorm) {
      float wa[4], wb[4];
      norm_weights(norm, 4 * qd.x, wa);
      norm_weights(norm, 4 * qd.y, wb);
      norm_quads<Bf16, kInter>(a, b, wa, wb, kDim / 8, kDim, norm.eps, turned, t);
    } else if (turned) {
      turn_quads<Bf16, kInter>(a, b, t);
    }
    *reinterpret_cast<uint2*>(tile + k_off(s, 4 * qd.x)) = a;
    *reinterpret_cast<uint2*>(tile + k_off(s, 4 * qd.y)) = b;
  }
}

// Blocks below kv_blocks: new rows [16 i, 16 i + 16) of one KV head.  Rows with consecutive
// slots of one page form a run; the block writes the runs that begin among its rows, so a long
// chunk's blocks write whole pages wherever its pages begin.  Whole pages go through LDS (V
// tiles are transposed), single rows straight to their slots.  The other blocks turn queries.
struct NoNorms {
  HeadNorm q, k;  // not read
};
template <int kForm, int kHeads, Streaming kStream, class Norms = NoNorms>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(Rot rot, WriteArgs A,
                                                             RowsArgs<Bf16> Q, Norms norms) {
  constexpr bool kNorm = std::is_same_v<Norms, RowNorms>;
  static_assert(sizeof(float2[kRotaryPairs]) == sizeof(float[kDim]), "a row of either in LDS");
  __shared__ __align__(16) uint16_t vt[kTileElems];
  __shared__ __align__(16) float2 cs[kForm == kAnyPairs ? kPage : 1][kRotaryPairs];
  if (int(blockIdx.x) >= A.kv_blocks) {
    const int i = int(blockIdx.x) - A.kv_blocks;
    const int bx = i / Q.y_blocks;
    if constexpr (kForm == kAnyPairs && kNorm)
      norm_queries_any(rot, Q, bx, i - bx * Q.y_blocks, norms.q, reinterpret_cast<float(*)[kDim]>(cs));
    else if constexpr (kForm == kAnyPairs)
      turn_queries_any(rot, Q, bx, i - bx * Q.y_blocks, cs);
    else
      turn_rows_wide<Bf16, kForm == kInterQuads, kHeads, kStream, kNorm>(rot, Q, bx, i - bx * Q.y_blocks, norms.q);
    return;
  }
  const int blk = int(blockIdx.x) / A.hkv, g = int(blockIdx.x) - blk * A.hkv;
  const int64_t r0 = (A.first_block + blk) * kPage;
  const int t = threadIdx.x, lane = t & 63;
  const int s = t >> 4, j = t & 15;
  // Lane l looks at row r0 - 1 + l.
  const int64_t seen = r0 - 1 + lane;
  int64_t slot = -1;
  if (seen >= 0 && seen < A.rows && lane < 48) slot = A.slots[seen];
  if (uint64_t(slot) >= uint64_t(A.slot_end)) slot = -1;
  const int64_t before = __shfl_up(slot, 1);
  const bool leads = slot < 0 || (slot & 15) == 0 || before != slot - 1;
  const uint64_t leaders = __ballot(leads) >> 1;  // bit i: row r0 + i
  const int a = __builtin_ctzll(leaders);
  if (a >= kPage) return;
  const int e = kPage + __builtin_ctzll(leaders >> kPage);
  const int64_t first = __shfl(slot, a + 1);
  const bool whole = e - a == kPage && first >= 0 &&
                     __popcll((leaders >> a) & ((uint64_t(1) << kPage) - 1)) == 1;
  if (whole) {
    const int64_t row = r0 + a + s;
    const size_t base = (size_t(first >> 4) * A.hkv + g) * kTileElems;
    const NewPiece p = load_piece<kForm>(A, rot, row, g, j);
    v_scatter8(vt, s, 8 * j, p.v);
    store_key<kForm, kNorm>(A, rot, p, row, g, j, s, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0], norms.k);
    __syncthreads();
    *reinterpret_cast<uint4*>(A.v_cache + base + t * 8) = *reinterpret_cast<const uint4*>(vt + t * 8);
    return;
  }
  for (int i = a + s; i - s < e; i += kPage) {
    const int64_t at = __shfl(slot, i + 1);
    if (i >= e || at < 0) continue;
    const int64_t row = r0 + i;
    const size_t base = (size_t(at >> 4) * A.hkv + g) * kTileElems;
    const int sl = int(at & 15);
    const NewPiece p = load_piece<kForm>(A, rot, row, g, j);
    v_scatter8(A.v_cache + base, sl, 8 * j, p.v);
    store_key<kForm, kNorm>(A, rot, p, row, g, j, sl, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0], norms.k);
  }
}

// Block (w, g): record w of an append plan's write table, as cache_write_kernel.
template <int kForm>
__global__ __launch_bounds__(kThreads) void cache_write_rotary_kernel(Rot rot, WriteArgs A) {
  __shared__ __align__(16) uint16_t vt[kTileElems];
  __shared__ __align__(16) float2 cs[kForm == kAnyPairs ? kPage : 1][kRotaryPairs];
  const int32_t* w = A.writes + size_t(blockIdx.x) * kWriteInts;
  const int g = blockIdx.y;
  const int b = w[W_B], pg = w[W_PAGE], s0 = w[W_SLOT0], s1 = w[W_SLOT1];
  const int t = threadIdx.x;
  const int s = t >> 4, j = t & 15;
  const int from = min(max(s, s0), s1 - 1);  // a new slot: the loads then need no mask
  const int64_t row = int64_t(w[W_ROW]) + from - s0;
  NewPiece p = load_piece<kForm>(A, rot, row, g, j);
  if (!A.positions) p.pos = pg * kPage + from;
  const int64_t page = A.bt[int64_t(b) * A.bt_stride + pg];
  const size_t base = (size_t(page) * A.hkv + g) * kTileElems;
  if (s1 - s0 < kPage) {  // uniform over the block
    if (s != from) return;
    v_scatter8(A.v_cache + base, s, 8 * j, p.v);
    store_key<kForm>(A, rot, p, row, g, j, s, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0]);
    return;
  }
  v_scatter8(vt, s, 8 * j, p.v);
  store_key<kForm>(A, rot, p, row, g, j, s, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0]);
  __syncthreads();
  *reinterpret_cast<uint4*>(A.v_cache + base + t * 8) = *reinterpret_cast<const uint4*>(vt + t * 8);
}

WriteArgs write_args(const KvLayout& L, const NewRows& n) {
  WriteArgs A{};
  A.k_cache = static_cast<uint16_t*>(L.desc.k_cache);
  A.v_cache = static_cast<uint16_t*>(L.desc.v_cache);
  A.k_new = static_cast<const uint16_t*>(n.k);
  A.v_new = static_cast<const uint16_t*>(n.v);
  A.k_row = n.k_row, A.v_row = n.v_row;
  A.positions = n.positions;
  A.hkv = L.desc.num_kv_heads;
  return A;
}

KeyForm key_form(const Rotary* r) {
  if (!r) return kInterQuads;
  if (r->rotary_dim % 8) return kAnyPairs;
  return r->pairing == LIBRA_ROTARY_INTERLEAVED ? kInterQuads : kHalfQuads;
}

}  // namespace

hipError_t launch_rotary(const Rotary& r, const RotaryRows& a, hipStream_t s) {
  switch (a.dtype) {
    case LIBRA_DTYPE_BF16: return apply<Bf16>(r, a, s);
    case LIBRA_DTYPE_FP16: return apply<Fp16>(r, a, s);
    default: return apply<Fp32>(r, a, s);
  }
}

namespace {

template <class Norms>
hipError_t append_rows(const KvLayout& L, const NewRows& n, const int64_t* slots, int64_t rows,
                       int32_t hq, void* q_out, const Norms& norms, hipStream_t s) {
  Rot rot{};
  if (n.rotary) rot = rotary_args<kRotaryPairs>(*n.rotary);
  const KeyForm form = key_form(n.rotary);
  RowsPlan<Bf16> q{};
  if (hq > 0)
    q = plan_rows<Bf16>(*n.rotary, {n.q, q_out, n.q_row, kDim, int64_t(hq) * kDim, kDim, n.positions,
                                    rows, hq, LIBRA_DTYPE_BF16, false});
  if (form == kAnyPairs && hq > 0) {  // blocks of 16 rows of a head
    q.wide = true, q.many = false;
    q.args.block_rows = kPage;
    q.args.y_blocks = hq;
  }
  // The cache's rows take their share of the caches too.
  q.stream = q.many && q.lines && rows * (hq + 2 * L.desc.num_kv_heads) * kDim * 2 >= kStreamBytes;
  auto quads = [&](auto key_form) {
    constexpr int kForm = decltype(key_form)::value;
    return !q.many    ? kv_append_kernel<kForm, 1, kCached, Norms>
           : q.stream ? kv_append_kernel<kForm, 4, kReadsWrites, Norms>
                      : kv_append_kernel<kForm, 4, kCached, Norms>;
  };
  auto k = form == kAnyPairs     ? kv_append_kernel<kAnyPairs, 1, kCached, Norms>
           : form == kInterQuads ? quads(std::integral_constant<int, kInterQuads>{})
                                 : quads(std::integral_constant<int, kHalfQuads>{});
  // Rows that one launch takes: at most kMaxBlocks blocks of either kind.
  WriteArgs A = write_args(L, n);
  A.slots = slots;
  A.slot_end = L.desc.num_pages * kPage;
  A.rows = rows;
  int64_t step = kMaxBlocks / A.hkv * kPage;
  if (hq > 0) step = std::max<int64_t>(kPage, std::min(step, q.rows_of(kMaxBlocks / q.args.y_blocks)) / kPage * kPage);
  for (int64_t r0 = 0; r0 < rows; r0 += step) {
    const int64_t n_rows = std::min(step, rows - r0);
    A.first_block = r0 / kPage;
    A.kv_blocks = int((n_rows + kPage - 1) / kPage * A.hkv);
    RowsArgs<Bf16> Q = q.args;
    int64_t blocks = A.kv_blocks;
    if (hq > 0) {
      Q.rows = n_rows;
      Q.x += r0 * Q.x_row;
      Q.out += r0 * Q.out_row;
      Q.positions += r0;
      Q.slots = slots + r0;
      Q.slot_end = A.slot_end;
      blocks += q.blocks(n_rows) * Q.y_blocks;
    }
    hipLaunchKernelGGL(k, dim3(unsigned(blocks)), dim3(kThreads), 0, s, rot, A, Q, norms);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_kv_append(const KvLayout& L, const NewRows& n, const int64_t* slots,
                            int64_t rows, int32_t hq, void* q_out, hipStream_t s) {
  return append_rows(L, n, slots, rows, hq, q_out, NoNorms{}, s);
}

hipError_t launch_kv_append_norm(const KvLayout& L, const NewRows& n, const RowNorms& norms, const int64_t* slots,
                                 int64_t rows, int32_t hq, void* q_out, hipStream_t s) {
  return append_rows(L, n, slots, rows, hq, q_out, norms, s);
}

hipError_t launch_norm_rotary(const Rotary& r, const RotaryRows& q, const RotaryRows& k, const RowNorms& norms,
                              hipStream_t s) {
  switch (q.dtype) {
    case LIBRA_DTYPE_BF16: return apply_norm<Bf16>(r, q, k, norms, s);
    case LIBRA_DTYPE_FP16: return apply_norm<Fp16>(r, q, k, norms, s);
    default: return apply_norm<Fp32>(r, q, k, norms, s);
  }
}

hipError_t launch_cache_write_rotary(const KvLayout& L, const Plan& P, const void* ws,
                                     const NewRows& n, const int32_t* bt, int32_t stride,
                                     hipStream_t s) {
  const int tiles = P.info.n_write_tiles;
  if (tiles == 0) return hipSuccess;
  WriteArgs A = write_args(L, n);
  A.writes = reinterpret_cast<const int32_t*>(static_cast<const char*>(ws) + P.off_writes);
  A.bt = bt;
  A.bt_stride = stride;
  const KeyForm form = key_form(n.rotary);
  auto k = form == kAnyPairs     ? cache_write_rotary_kernel<kAnyPairs>
           : form == kInterQuads ? cache_write_rotary_kernel<kInterQuads>
                                 : cache_write_rotary_kernel<kHalfQuads>;
  hipLaunchKernelGGL(k, dim3(unsigned(tiles), unsigned(A.hkv)), dim3(kThreads), 0, s,
                     rotary_args<kRotaryPairs>(*n.rotary), A);
  return hipGetLastError();
}

}  // namespace libra
