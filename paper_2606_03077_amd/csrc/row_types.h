// Element types, quads of channels and cache-tile offsets shared by the kernels that take rows
// of heads (rotary.hip, norm.hip, kv_map.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "drafts.h"
#include "rotary.h"

namespace libra {

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

// Four pairs in two quads, which is what a thread turns: half pairing takes channel e of both
// quads as a pair, interleaved pairing two neighbours of one.
template <bool kInter>
__device__ __forceinline__ void turn_values(const float (&f)[4], const float (&g)[4],
                                            const float2 (&cs)[4], float (&y)[4], float (&z)[4]) {
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
}
template <class T, bool kInter>
__device__ __forceinline__ void turn_quads(typename T::Quad& a, typename T::Quad& b,
                                           const float2 (&cs)[4]) {
  float f[4], g[4], y[4], z[4];
  T::unpack(a, f);
  T::unpack(b, g);
  turn_values<kInter>(f, g, cs, y, z);
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

// --- norms of heads ------------------------------------------------------------------------

// n = x / sqrt(mean(x^2) + eps), u = w n: all in float32, the same operations in every kernel, so
// that all paths give the same bits.
__device__ __forceinline__ float norm_weight(const HeadNorm& n, int d) {
  if (n.weight_dtype == LIBRA_DTYPE_FP32) return static_cast<const float*>(n.weight)[d];
  const uint16_t e = static_cast<const uint16_t*>(n.weight)[d];
  return n.weight_dtype == LIBRA_DTYPE_BF16 ? Bf16::get(e) : Fp16::get(e);
}

// Weights of channels d .. d + 3; in one load where that is aligned (norm.quads).
__device__ __forceinline__ void norm_weights(const HeadNorm& n, int d, float (&w)[4]) {
  if (!n.quads) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = norm_weight(n, d + e);
  } else if (n.weight_dtype == LIBRA_DTYPE_FP32) {
    Fp32::unpack(*reinterpret_cast<const float4*>(static_cast<const float*>(n.weight) + d), w);
  } else {
    const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(n.weight) + d);
    if (n.weight_dtype == LIBRA_DTYPE_BF16) Bf16::unpack(q, w);
    else Fp16::unpack(q, w);
  }
}

__device__ __forceinline__ float norm_scale(float squares, int dim, float eps) {
  const float v = squares / float(dim) + eps;
  const float r = __builtin_amdgcn_rsqf(v);
  // One Newton step: v_rsq_f32 is good to one unit in the last place only.  0 and infinity, whose
  // steps are NaN, stay.
  const float s = __builtin_fmaf(0.5f * r, __builtin_fmaf(-v * r, r, 1.f), r);
  return s == s ? s : r;
}

template <int kCtrl>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                           0, __builtin_bit_cast(int, x), kCtrl, 0xF, 0xF, true));
}
// The sum over aligned groups of `lanes` lanes (a power of two, the same in all), in each of them,
// and the same bits in each: both sides of every step add the same two numbers.
__device__ __forceinline__ float group_sum(float x, int lanes) {
  if (lanes > 1) x = dpp_add<0xB1>(x);    // lanes i and i ^ 1
  if (lanes > 2) x = dpp_add<0x4E>(x);    // i ^ 2
  if (lanes > 4) x = dpp_add<0x141>(x);   // the halves of 8 lanes, mirrored
  if (lanes > 8) x = dpp_add<0x140>(x);   // of 16
  if (lanes > 16) x += __shfl_xor(x, 16);
  if (lanes > 32) x += __shfl_xor(x, 32);
  return x;
}

}  // namespace libra
