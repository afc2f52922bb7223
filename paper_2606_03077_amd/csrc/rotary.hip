// Rotary positions of dense rows, and the cache append that turns keys on the way.
#include <algorithm>

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

template <class T>
struct ApplyArgs {
  RotaryArgs<kMaxPairs> rot;
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
  // eight-channel pieces in kHeads heads, head_slots apart.
  int per_head, head_slots, per_row, block_rows;
};

// Sign of the sine: the gradient turns back.
template <class Args>
__device__ __forceinline__ float2 cos_sin_of(const Args& A, int j, int32_t pos) {
  float2 cs = rotary_cos_sin(A.rot.turn[j], pos, A.rot.amplitude);
  if (A.backward) cs.y = -cs.y;
  return cs;
}

template <class Args>
__device__ __forceinline__ bool skipped(const Args& A, int64_t row) {
  return A.slots && uint64_t(A.slots[row]) >= uint64_t(A.slot_end);
}

// Wide form: R and the head size are multiples of 8, rows are aligned for four channels at a
// time.  A thread owns two quads of a head (4 pairs, or 8 copied channels), computes their
// cosines and sines once, and turns them in up to kHeads heads.
template <class T, bool kInter, int kHeads>
__global__ __launch_bounds__(kThreads) void rotary_wide_kernel(ApplyArgs<T> A) {
  using Quad = typename T::Quad;
  const int t = threadIdx.x;
  const int r = t / A.per_row, in_row = t - r * A.per_row;
  const int h0 = in_row / A.per_head, j = in_row - h0 * A.per_head;
  const int64_t row = int64_t(blockIdx.x) * A.block_rows + r;
  if (r >= A.block_rows || row >= A.rows || skipped(A, row)) return;
  const int R8 = A.rot.rdim / 8;
  const bool turned = j < R8;
  if (!turned && A.x == A.out) return;
  const int qa = kInter || !turned ? 2 * j : j, qb = kInter || !turned ? 2 * j + 1 : j + R8;
  const int head0 = blockIdx.y * A.head_slots * kHeads + h0;
  const typename T::Elem* x = A.x + row * A.x_row;
  typename T::Elem* out = A.out + row * A.out_row;
  Quad a[kHeads], b[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = head0 + i * A.head_slots;
    if (h < A.heads) {
      a[i] = *reinterpret_cast<const Quad*>(x + h * A.x_head + 4 * qa);
      b[i] = *reinterpret_cast<const Quad*>(x + h * A.x_head + 4 * qb);
    }
  }
  float2 cs[4];
  if (turned) {
    const int32_t pos = A.positions[row];
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = cos_sin_of(A, 4 * j + i, pos);
  }
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = head0 + i * A.head_slots;
    if (h < A.heads) {
      if (turned) {
        float f[4], g[4], y[4], z[4];
        T::unpack(a[i], f);
        T::unpack(b[i], g);
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
        a[i] = T::pack(y);
        b[i] = T::pack(z);
      }
      *reinterpret_cast<Quad*>(out + h * A.out_head + 4 * qa) = a[i];
      *reinterpret_cast<Quad*>(out + h * A.out_head + 4 * qb) = b[i];
    }
  }
}

// Narrow form: any even R, any alignment.  A thread owns one pair (or one copied channel) of
// a row, in every kNarrowHeads heads of its block row.
constexpr int kNarrowHeads = 8;
template <class T>
__global__ __launch_bounds__(kThreads) void rotary_narrow_kernel(ApplyArgs<T> A) {
  const int half = A.rot.rdim / 2;
  const int items = A.dim - half;
  const int64_t idx = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = idx / items;
  const int j = int(idx - row * items);
  if (row >= A.rows || skipped(A, row)) return;
  const typename T::Elem* x = A.x + row * A.x_row;
  typename T::Elem* out = A.out + row * A.out_row;
  const int h0 = blockIdx.y * kNarrowHeads, h1 = min(A.heads, h0 + kNarrowHeads);
  if (j >= half) {
    if (A.x == A.out) return;
    const int d = j + half;
    for (int h = h0; h < h1; ++h) out[h * A.out_head + d] = x[h * A.x_head + d];
    return;
  }
  const int d1 = A.rot.interleaved ? 2 * j : j, d2 = A.rot.interleaved ? 2 * j + 1 : j + half;
  const float2 cs = cos_sin_of(A, j, A.positions[row]);
  for (int h = h0; h < h1; ++h) {
    const float x1 = T::get(x[h * A.x_head + d1]), x2 = T::get(x[h * A.x_head + d2]);
    out[h * A.out_head + d1] = T::put(turn_first(x1, x2, cs));
    out[h * A.out_head + d2] = T::put(turn_second(x1, x2, cs));
  }
}

constexpr int64_t kMaxBlocks = int64_t(1) << 22;  // per launch: 2^30 threads

template <class T>
hipError_t apply(const Rotary& r, const RotaryRows& a, const int64_t* slots, int64_t slot_end,
                 hipStream_t s) {
  using Elem = typename T::Elem;
  ApplyArgs<T> A;
  A.rot = rotary_args<kMaxPairs>(r);
  A.x_row = a.x_row, A.x_head = a.x_head, A.out_row = a.out_row, A.out_head = a.out_head;
  A.slot_end = slot_end;
  A.heads = a.heads, A.dim = r.head_dim;
  A.backward = a.backward;
  A.per_head = r.head_dim / 8;
  const size_t quad = sizeof(typename T::Quad);
  const bool wide = r.rotary_dim % 8 == 0 && r.head_dim % 8 == 0 &&
                    (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) % quad == 0 &&
                    ((a.x_row | a.x_head | a.out_row | a.out_head) & 3) == 0;
  const bool many = a.rows * a.heads * A.per_head >= int64_t(4) * 2048 * kThreads;
  const int per_thread = many ? 4 : 1;
  if (wide) {
    A.head_slots = std::min<int>((a.heads + per_thread - 1) / per_thread, kThreads / A.per_head);
    A.per_row = A.head_slots * A.per_head;
    A.block_rows = kThreads / A.per_row;
  }
  const int items = r.head_dim - r.rotary_dim / 2;
  const int64_t rows_per_launch = wide ? kMaxBlocks * A.block_rows : kMaxBlocks * kThreads / items;
  for (int64_t r0 = 0; r0 < a.rows; r0 += rows_per_launch) {
    A.rows = std::min(rows_per_launch, a.rows - r0);
    A.x = static_cast<const Elem*>(a.x) + r0 * a.x_row;
    A.out = static_cast<Elem*>(a.out) + r0 * a.out_row;
    A.positions = a.positions + r0;
    A.slots = slots ? slots + r0 : nullptr;
    if (wide) {
      const int per_block = A.head_slots * per_thread;
      const dim3 grid(unsigned((A.rows + A.block_rows - 1) / A.block_rows),
                      unsigned((a.heads + per_block - 1) / per_block));
      const bool inter = r.pairing == LIBRA_ROTARY_INTERLEAVED;
      auto k = many ? (inter ? rotary_wide_kernel<T, true, 4> : rotary_wide_kernel<T, false, 4>)
                    : (inter ? rotary_wide_kernel<T, true, 1> : rotary_wide_kernel<T, false, 1>);
      hipLaunchKernelGGL(k, grid, dim3(unsigned(A.per_row * A.block_rows)), 0, s, A);
    } else {
      const dim3 grid(unsigned((A.rows * items + kThreads - 1) / kThreads),
                      unsigned((a.heads + kNarrowHeads - 1) / kNarrowHeads));
      hipLaunchKernelGGL(rotary_narrow_kernel<T>, grid, dim3(kThreads), 0, s, A);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// --- cache append ------------------------------------------------------------------------

struct WriteArgs {
  RotaryArgs<kRotaryPairs> rot;  // rdim 0: keys are copied
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
  // by an append plan's records
  const int32_t* writes;
  const int32_t* bt;
  int64_t bt_stride;
};

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

// Granule j (8 channels) of row `row`'s key of head g, turned.  The 16 threads of a row, in
// one wave, share the row's cosines and sines through cs.
__device__ __forceinline__ uint4 key_granule(const WriteArgs& A, int64_t row, int g, int j,
                                             int32_t pos, float2* cs) {
  const uint16_t* k = A.k_new + row * A.k_row + g * kDim;
  if (A.rot.rdim == 0) return *reinterpret_cast<const uint4*>(k + 8 * j);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4 * j + i < A.rot.rdim / 2)
      cs[4 * j + i] = rotary_cos_sin(A.rot.turn[4 * j + i], pos, A.rot.amplitude);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return turned_granule<false>(k, j, cs, A.rot.rdim, A.rot.interleaved).hi;
}

// Block (i, g): new rows [16 i, 16 i + 16) of KV head g.  Rows with consecutive slots of one
// page form a run; the block writes the runs that begin among its rows, so a long chunk's
// blocks write whole pages wherever its pages begin.  Whole pages go through LDS (V tiles are
// transposed), single rows straight to their slots.
__global__ __launch_bounds__(kThreads) void kv_append_kernel(WriteArgs A, int64_t block0) {
  __shared__ __align__(16) uint16_t vt[kTileElems];
  __shared__ __align__(16) float2 cs[kPage][kRotaryPairs];
  const int g = blockIdx.y;
  const int64_t r0 = (block0 + blockIdx.x) * kPage;
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
    const uint4 v = *reinterpret_cast<const uint4*>(A.v_new + row * A.v_row + g * kDim + 8 * j);
    const int32_t pos = A.rot.rdim ? A.positions[row] : 0;
    const uint4 k = key_granule(A, row, g, j, pos, cs[s]);
    *reinterpret_cast<uint4*>(A.k_cache + base + k_off(s, 8 * j)) = k;
    v_scatter8(vt, s, 8 * j, v);
    __syncthreads();
    *reinterpret_cast<uint4*>(A.v_cache + base + t * 8) = *reinterpret_cast<const uint4*>(vt + t * 8);
    return;
  }
  for (int i = a + s; i - s < e; i += kPage) {
    const int64_t at = __shfl(slot, i + 1 < 64 ? i + 1 : 63);
    if (i >= e || at < 0) continue;
    const int64_t row = r0 + i;
    const size_t base = (size_t(at >> 4) * A.hkv + g) * kTileElems;
    const int sl = int(at & 15);
    const uint4 v = *reinterpret_cast<const uint4*>(A.v_new + row * A.v_row + g * kDim + 8 * j);
    const int32_t pos = A.rot.rdim ? A.positions[row] : 0;
    const uint4 k = key_granule(A, row, g, j, pos, cs[s]);
    *reinterpret_cast<uint4*>(A.k_cache + base + k_off(sl, 8 * j)) = k;
    v_scatter8(A.v_cache + base, sl, 8 * j, v);
  }
}

// Block (w, g): record w of an append plan's write table, as cache_write_kernel.
__global__ __launch_bounds__(kThreads) void cache_write_rotary_kernel(WriteArgs A) {
  __shared__ __align__(16) uint16_t vt[kTileElems];
  __shared__ __align__(16) float2 cs[kPage][kRotaryPairs];
  const int32_t* w = A.writes + size_t(blockIdx.x) * kWriteInts;
  const int g = blockIdx.y;
  const int b = w[W_B], pg = w[W_PAGE], s0 = w[W_SLOT0], s1 = w[W_SLOT1];
  const int t = threadIdx.x;
  const int s = t >> 4, j = t & 15;
  const int from = min(max(s, s0), s1 - 1);  // a new slot: the loads then need no mask
  const int64_t row = int64_t(w[W_ROW]) + from - s0;
  const uint4 v = *reinterpret_cast<const uint4*>(A.v_new + row * A.v_row + g * kDim + 8 * j);
  const int64_t page = A.bt[int64_t(b) * A.bt_stride + pg];
  const int32_t pos = A.positions ? A.positions[row] : pg * kPage + from;
  const uint4 k = key_granule(A, row, g, j, pos, cs[s]);
  const size_t base = (size_t(page) * A.hkv + g) * kTileElems;
  if (s1 - s0 < kPage) {  // uniform over the block
    if (s == from) {
      *reinterpret_cast<uint4*>(A.k_cache + base + k_off(s, 8 * j)) = k;
      v_scatter8(A.v_cache + base, s, 8 * j, v);
    }
    return;
  }
  *reinterpret_cast<uint4*>(A.k_cache + base + k_off(s, 8 * j)) = k;
  v_scatter8(vt, s, 8 * j, v);
  __syncthreads();
  *reinterpret_cast<uint4*>(A.v_cache + base + t * 8) = *reinterpret_cast<const uint4*>(vt + t * 8);
}

WriteArgs write_args(const KvLayout& L, const NewRows& n) {
  WriteArgs A{};
  if (n.rotary) A.rot = rotary_args<kRotaryPairs>(*n.rotary);
  A.k_cache = static_cast<uint16_t*>(L.desc.k_cache);
  A.v_cache = static_cast<uint16_t*>(L.desc.v_cache);
  A.k_new = static_cast<const uint16_t*>(n.k);
  A.v_new = static_cast<const uint16_t*>(n.v);
  A.k_row = n.k_row, A.v_row = n.v_row;
  A.positions = n.positions;
  A.hkv = L.desc.num_kv_heads;
  return A;
}

}  // namespace

hipError_t launch_rotary(const Rotary& r, const RotaryRows& a, hipStream_t s) {
  switch (a.dtype) {
    case LIBRA_DTYPE_BF16: return apply<Bf16>(r, a, nullptr, 0, s);
    case LIBRA_DTYPE_FP16: return apply<Fp16>(r, a, nullptr, 0, s);
    default: return apply<Fp32>(r, a, nullptr, 0, s);
  }
}

hipError_t launch_kv_append(const KvLayout& L, const NewRows& n, const int64_t* slots,
                            int64_t rows, int32_t hq, void* q_out, hipStream_t s) {
  WriteArgs A = write_args(L, n);
  A.slots = slots;
  A.slot_end = L.desc.num_pages * kPage;
  A.rows = rows;
  const int64_t blocks = (rows + kPage - 1) / kPage;
  for (int64_t b0 = 0; b0 < blocks; b0 += kMaxBlocks) {
    const int64_t n_blocks = std::min(kMaxBlocks, blocks - b0);
    hipLaunchKernelGGL(kv_append_kernel, dim3(unsigned(n_blocks), unsigned(A.hkv)),
                       dim3(kThreads), 0, s, A, b0);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (hq == 0) return hipSuccess;
  const RotaryRows a{n.q, q_out, n.q_row, kDim, int64_t(hq) * kDim, kDim, n.positions, rows, hq,
                     LIBRA_DTYPE_BF16, false};
  return apply<Bf16>(*n.rotary, a, slots, A.slot_end, s);
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
  hipLaunchKernelGGL(cache_write_rotary_kernel, dim3(unsigned(tiles), unsigned(A.hkv)),
                     dim3(kThreads), 0, s, A);
  return hipGetLastError();
}

}  // namespace libra
