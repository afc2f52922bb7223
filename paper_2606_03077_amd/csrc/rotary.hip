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
#include <algorithm>
#include <type_traits>

#include "rotary_calls.h"

namespace libra {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = kMaxRotaryDim / 2;

// Element types: four channels as loaded, to and from float32 (rounded to nearest even).
struct Bf16 {
  using Elem = uint16_t;
  using Quad = uint2;
  static __device__ __forceinline__ float get(Elem e) { return bf16_to_f32(e); }
  static __device__ __forceinline__ Elem put(float f) { return Elem(rotary_pack_bf16(f, f)); }
  static __device__ __forceinline__ void unpack(Quad q, float (&f)[4]) {
    f[0] = bf16_to_f32(q.x & 0xFFFF), f[1] = bf16_to_f32(q.x >> 16);
    f[2] = bf16_to_f32(q.y & 0xFFFF), f[3] = bf16_to_f32(q.y >> 16);
  }
  static __device__ __forceinline__ Quad pack(const float (&f)[4]) {
    return make_uint2(rotary_pack_bf16(f[0], f[1]), rotary_pack_bf16(f[2], f[3]));
  }
};
struct Fp16 {
  using Elem = uint16_t;
  using Quad = uint2;
  static __device__ __forceinline__ float get(Elem e) {
    return float(__builtin_bit_cast(_Float16, e));
  }
  static __device__ __forceinline__ Elem put(float f) {
    return __builtin_bit_cast(Elem, _Float16(f));
  }
  static __device__ __forceinline__ void unpack(Quad q, float (&f)[4]) {
    f[0] = get(Elem(q.x)), f[1] = get(Elem(q.x >> 16));
    f[2] = get(Elem(q.y)), f[3] = get(Elem(q.y >> 16));
  }
  static __device__ __forceinline__ Quad pack(const float (&f)[4]) {
    return make_uint2(put(f[0]) | uint32_t(put(f[1])) << 16, put(f[2]) | uint32_t(put(f[3])) << 16);
  }
};
struct Fp32 {
  using Elem = float;
  using Quad = float4;
  static __device__ __forceinline__ float get(Elem e) { return e; }
  static __device__ __forceinline__ Elem put(float f) { return f; }
  static __device__ __forceinline__ void unpack(Quad q, float (&f)[4]) {
    f[0] = q.x, f[1] = q.y, f[2] = q.z, f[3] = q.w;
  }
  static __device__ __forceinline__ Quad pack(const float (&f)[4]) {
    return make_float4(f[0], f[1], f[2], f[3]);
  }
};

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

// Four pairs in two quads, which is what a thread turns: half pairing takes channel e of both
// quads as a pair, interleaved pairing two neighbours of one.
template <class T, bool kInter>
__device__ __forceinline__ void turn_quads(typename T::Quad& a, typename T::Quad& b,
                                           const float2 (&cs)[4]) {
  float f[4], g[4], y[4], z[4];
  T::unpack(a, f);
  T::unpack(b, g);
  if (kInter) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      y[2 * e] = turn_first(f[2 * e], f[2 * e + 1], cs[e]);
      y[2 * e + 1] = turn_second(f[2 * e], f[2 * e + 1], cs[e]);
      z[2 * e] = turn_first(g[2 * e], g[2 * e + 1], cs[2 + e]);
      z[2 * e + 1] = turn_second(g[2 * e], g[2 * e + 1], cs[2 + e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = turn_first(f[e], g[e], cs[e]);
      z[e] = turn_second(f[e], g[e], cs[e]);
    }
  }
  a = T::pack(y);
  b = T::pack(z);
}

// The quads of piece j of a head of `pieces`, turned ones while j < R / 8, copied ones after.
// Neighbouring threads take neighbouring quads, so that an instruction covers whole lines; two
// quads of 8 bytes that are neighbours themselves make one access of 16.
template <class T, bool kInter>
__device__ __forceinline__ int2 quads_of(int j, int R8, int pieces) {
  if (kInter && sizeof(typename T::Quad) == 8) return make_int2(2 * j, 2 * j + 1);
  return j < R8 ? make_int2(j, j + R8) : make_int2(j + R8, j + pieces);
}

// Pair i of the four that a turned piece's quads hold.
template <bool kInter>
__device__ __forceinline__ int pair_of(int2 quads, int j, int i) {
  return !kInter ? 4 * j + i : i < 2 ? 2 * quads.x + i : 2 * quads.y + i - 2;
}

template <bool kPastCaches, class Quad>
__device__ __forceinline__ Quad load_quad(const Quad* p) {
  typedef uint32_t V __attribute__((ext_vector_type(sizeof(Quad) / 4)));
  if constexpr (kPastCaches)
    return __builtin_bit_cast(Quad, __builtin_nontemporal_load(reinterpret_cast<const V*>(p)));
  else
    return *p;
}
template <bool kPastCaches, class Quad>
__device__ __forceinline__ void store_quad(Quad* p, Quad v) {
  typedef uint32_t V __attribute__((ext_vector_type(sizeof(Quad) / 4)));
  if constexpr (kPastCaches)
    __builtin_nontemporal_store(__builtin_bit_cast(V, v), reinterpret_cast<V*>(p));
  else
    *p = v;
}

constexpr int64_t kStreamBytes = int64_t(128) << 20;  // written by a call whose writes go past

// What goes past the caches: nothing, the reads (each value is read once), or both.
enum Streaming : int { kCached, kReads, kReadsWrites };

// Wide form: R and the head size are multiples of 8, rows are aligned for four channels at a
// time.  A thread owns two quads of a head (4 pairs, or 8 copied channels), computes their
// cosines and sines once, and turns them in up to kHeads heads.
template <class T, bool kInter, int kHeads, Streaming kStream, class Rot>
__device__ __forceinline__ void turn_rows_wide(const Rot& rot, const RowsArgs<T>& A, int64_t bx,
                                               int by) {
  using Quad = typename T::Quad;
  const int t = threadIdx.x;
  const int r = t / A.per_row, in_row = t - r * A.per_row;
  const int h0 = in_row / A.per_head, j = in_row - h0 * A.per_head;
  const int64_t row = bx * A.block_rows + r;
  if (r >= A.block_rows || row >= A.rows || skipped(A, row)) return;
  const int R8 = rot.rdim / 8;
  const bool turned = j < R8;
  if (!turned && A.x == A.out) return;
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
      if (turned) turn_quads<T, kInter>(a[i], b[i], cs);
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

template <class T>
RowsPlan<T> plan_rows(const Rotary& r, const RotaryRows& a) {
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
  p.many = a.heads >= 16 && a.rows * a.heads * A.per_head >= int64_t(2560) * kThreads;
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

// Element offsets inside a tile (kv_layout.hip has the layout).
__device__ __forceinline__ int k_off(int s, int d) { return ((d >> 3) * 16 + s) * 8 + (d & 7); }
__device__ __forceinline__ int v_off(int s, int d) {
  return (128 * ((s >> 2) & 1) + d) * 8 + (s >> 3) * 4 + (s & 3);
}
__device__ __forceinline__ void v_scatter8(uint16_t* tile, int s, int d0, uint4 val) {
  const uint32_t w[4] = {val.x, val.y, val.z, val.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) tile[v_off(s, d0 + i)] = uint16_t(w[i / 2] >> (16 * (i & 1)));
}

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

// 16 rows of one query head, any pairs.
__device__ __forceinline__ void turn_queries_any(const Rot& rot, const RowsArgs<Bf16>& A, int64_t bx,
                                                 int head, float2 (*cs)[kRotaryPairs]) {
  const int s = threadIdx.x >> 4, j = threadIdx.x & 15;
  const int64_t row = bx * kPage + s;
  if (row >= A.rows || skipped(A, row)) return;
  const uint4 y = turn_any_granule(rot, A.x + row * A.x_row + int64_t(head) * kDim, j, A.positions[row], cs[s]);
  *reinterpret_cast<uint4*>(A.out + row * A.out_row + int64_t(head) * kDim + 8 * j) = y;
}

// Turns the piece's key and stores it to slot s of the K tile.
template <int kForm>
__device__ __forceinline__ void store_key(const WriteArgs& A, const Rot& rot, const NewPiece& p,
                                          int64_t row, int g, int j, int s, uint16_t* tile,
                                          float2* cs) {
  if constexpr (kForm == kAnyPairs) {
    *reinterpret_cast<uint4*>(tile + k_off(s, 8 * j)) =
        turn_any_granule(rot, A.k_new + row * A.k_row + g * kDim, j, p.pos, cs);
  } else {
    constexpr bool kInter = kForm == kInterQuads;
    const int2 qd = quads_of<Bf16, kInter>(j, rot.rdim / 8, kDim / 8);
    uint2 a = p.a, b = p.b;
    if (j < rot.rdim / 8) {
      float2 t[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t[i] = rotary_cos_sin(rot.turn[pair_of<kInter>(qd, j, i)], p.pos, rot.amplitude);
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
template <int kForm, int kHeads, Streaming kStream>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(Rot rot, WriteArgs A,
                                                             RowsArgs<Bf16> Q) {
  __shared__ __align__(16) uint16_t vt[kTileElems];
  __shared__ __align__(16) float2 cs[kForm == kAnyPairs ? kPage : 1][kRotaryPairs];
  if (int(blockIdx.x) >= A.kv_blocks) {
    const int i = int(blockIdx.x) - A.kv_blocks;
    const int bx = i / Q.y_blocks;
    if constexpr (kForm == kAnyPairs)
      turn_queries_any(rot, Q, bx, i - bx * Q.y_blocks, cs);
    else
      turn_rows_wide<Bf16, kForm == kInterQuads, kHeads, kStream>(rot, Q, bx, i - bx * Q.y_blocks);
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
    store_key<kForm>(A, rot, p, row, g, j, s, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0]);
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
    store_key<kForm>(A, rot, p, row, g, j, sl, A.k_cache + base, cs[kForm == kAnyPairs ? s : 0]);
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

hipError_t launch_kv_append(const KvLayout& L, const NewRows& n, const int64_t* slots,
                            int64_t rows, int32_t hq, void* q_out, hipStream_t s) {
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
    return !q.many    ? kv_append_kernel<kForm, 1, kCached>
           : q.stream ? kv_append_kernel<kForm, 4, kReadsWrites>
                      : kv_append_kernel<kForm, 4, kCached>;
  };
  auto k = form == kAnyPairs     ? kv_append_kernel<kAnyPairs, 1, kCached>
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
    hipLaunchKernelGGL(k, dim3(unsigned(blocks)), dim3(kThreads), 0, s, rot, A, Q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
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
