// Rotary positions: the handle, what kernels get of it, and the rotation on the device.
//
// The first R channels of a head are R / 2 pairs (x1, x2); pair j of a row at position p is
// turned by the angle p theta_j and scaled by the amplitude A:
//   y1 = A (x1 cos - x2 sin),  y2 = A (x2 cos + x1 sin);
// the gradient's pass takes -sin (the transpose).  Half pairing: channels (j, j + R / 2);
// interleaved: (2 j, 2 j + 1).  Channels from R on are copied.
//
// Angles are kept in turns, as 64-bit fixed point: turn_j = theta_j / 2 pi mod 1 in units of
// 2^-64, and p turn_j mod 2^64 is the angle mod one turn, exact but for turn_j's own rounding
// (p 2^-65 turns), whatever the position; float32 angles lose 2^-24 p theta.  The fraction's
// top 32 bits give the quadrant and an angle in [-pi / 4, pi / 4] for the sine's and cosine's
// Taylor polynomials (truncated below 2e-9; with float32 rounding within 1.2e-7).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "tables.h"

namespace libra {

constexpr int kMaxRotaryDim = 256;       // channels that may rotate
constexpr int kMaxRotaryHead = 512;      // channels per head of libra_rotary_apply
constexpr int kRotaryPairs = kDim / 2;   // pairs of a cached head

struct Rotary {
  int32_t head_dim = 0, rotary_dim = 0, pairing = 0;
  float amplitude = 1.f;
  uint64_t turn[kMaxRotaryDim / 2] = {};
  double theta[kMaxRotaryDim / 2] = {};
};

// Kernel arguments: the turns of up to kPairs pairs.
template <int kPairs>
struct RotaryArgs {
  uint64_t turn[kPairs];
  float amplitude;
  int32_t rdim;         // R
  int32_t interleaved;  // pairing
};

template <int kPairs>
inline RotaryArgs<kPairs> rotary_args(const Rotary& r) {
  RotaryArgs<kPairs> a{};
  for (int j = 0; j < r.rotary_dim / 2 && j < kPairs; ++j) a.turn[j] = r.turn[j];
  a.amplitude = r.amplitude;
  a.rdim = r.rotary_dim;
  a.interleaved = r.pairing == LIBRA_ROTARY_INTERLEAVED;
  return a;
}

#ifdef __HIPCC__

// (cos, sin) of p turn / 2^64 turns, times the amplitude.
__device__ __forceinline__ float2 rotary_cos_sin(uint64_t turn, int32_t pos, float amplitude) {
  const uint32_t u = uint32_t((turn * uint64_t(int64_t(pos))) >> 32);
  const uint32_t quad = (u + 0x20000000u) >> 30;                  // nearest quarter turn, mod 4
  const float y = float(int32_t(u - (quad << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = y * y;
  float s = __builtin_fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f);
  s = __builtin_fmaf(z, s, 8.3333333333e-3f);
  s = __builtin_fmaf(z, s, -1.6666666667e-1f);
  s = __builtin_fmaf(y * z, s, y);
  float c = __builtin_fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);
  c = __builtin_fmaf(z, c, -1.3888888889e-3f);
  c = __builtin_fmaf(z, c, 4.1666666667e-2f);
  c = __builtin_fmaf(z, c, -0.5f);
  c = __builtin_fmaf(z, c, 1.f);
  const bool odd = quad & 1;
  const uint32_t cn = __float_as_uint((odd ? s : c) * amplitude) ^ (((quad + 1) << 30) & 0x80000000u);
  const uint32_t sn = __float_as_uint((odd ? c : s) * amplitude) ^ ((quad << 30) & 0x80000000u);
  return make_float2(__uint_as_float(cn), __uint_as_float(sn));
}

// The two halves of a turned pair.  One rounding each besides the product's, the same in
// every kernel, so that all paths give the same bits.
__device__ __forceinline__ float turn_first(float x1, float x2, float2 cs) {
  return __builtin_fmaf(x1, cs.x, -(x2 * cs.y));
}
__device__ __forceinline__ float turn_second(float x1, float x2, float2 cs) {
  return __builtin_fmaf(x2, cs.x, x1 * cs.y);
}

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }

// Two floats to bf16 (round to nearest even) in one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t rotary_pack_bf16(float lo, float hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
}

// Eight turned channels: as bf16 (nearest), and what that leaves of the float32 values, as
// bf16 again (both together hold 16 bits).  Nothing is left of copied channels, of values
// that are not finite, or of those beyond bf16's range.
struct TurnedGranule {
  uint4 hi, lo;
};

template <bool kLow>
__device__ __forceinline__ void split_pair(float y0, float y1, bool turned0, bool turned1,
                                           uint32_t raw, uint32_t& hi, uint32_t& lo) {
  const uint32_t h = rotary_pack_bf16(y0, y1);
  const uint32_t keep = (turned0 ? 0u : 0x0000FFFFu) | (turned1 ? 0u : 0xFFFF0000u);
  hi = (raw & keep) | (h & ~keep);
  if constexpr (kLow) {
    const float h0 = bf16_to_f32(h & 0xFFFF), h1 = bf16_to_f32(h >> 16);
    const float l0 = turned0 && __builtin_isfinite(h0) ? y0 - h0 : 0.f;
    const float l1 = turned1 && __builtin_isfinite(h1) ? y1 - h1 : 0.f;
    lo = rotary_pack_bf16(l0, l1);
  } else {
    lo = 0;
  }
}

// Granule gi (channels 8 gi .. + 7) of a bf16 row of 128 channels, turned (lo only if kLow).
// cs: the row's (cos, sin) by pair.  Reads the partner channels from the row too.
template <bool kLow>
__device__ __forceinline__ TurnedGranule turned_granule(const uint16_t* row, int gi,
                                                        const float2* cs, int rdim,
                                                        int interleaved) {
  const int d0 = 8 * gi;
  const uint4 raw = *reinterpret_cast<const uint4*>(row + d0);
  if (d0 >= rdim) return {raw, make_uint4(0, 0, 0, 0)};
  const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t hi[4], lo[4];
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = cs[4 * gi + i];  // past the last pair: not used
      const float x1 = bf16_to_f32(rw[i] & 0xFFFF), x2 = bf16_to_f32(rw[i] >> 16);
      const bool turned = d0 + 2 * i < rdim;
      split_pair<kLow>(turn_first(x1, x2, t), turn_second(x1, x2, t), turned, turned, rw[i], hi[i],
                       lo[i]);
    }
  } else {
    const int h = rdim / 2;
    uint32_t pw[4];  // the partners, two in a word
    if ((h & 7) == 0) {
      const uint4 p = *reinterpret_cast<const uint4*>(row + (d0 < h ? d0 + h : d0 - h));
      pw[0] = p.x, pw[1] = p.y, pw[2] = p.z, pw[3] = p.w;
    } else {
      auto partner = [&](int d) -> uint32_t { return row[d < h ? d + h : d < rdim ? d - h : d]; };
#pragma unroll
      for (int i = 0; i < 4; ++i) pw[i] = partner(d0 + 2 * i) | partner(d0 + 2 * i + 1) << 16;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = d0 + 2 * i + e;
        const bool first = d < h;
        const float2 t = cs[first ? d : d < rdim ? d - h : 0];
        const float x = bf16_to_f32((rw[i] >> (16 * e)) & 0xFFFF);
        const float o = bf16_to_f32((pw[i] >> (16 * e)) & 0xFFFF);
        y[e] = first ? turn_first(x, o, t) : turn_second(o, x, t);
      }
      const int d = d0 + 2 * i;
      split_pair<kLow>(y[0], y[1], d < rdim, d + 1 < rdim, rw[i], hi[i], lo[i]);
    }
  }
  return {make_uint4(hi[0], hi[1], hi[2], hi[3]), make_uint4(lo[0], lo[1], lo[2], lo[3])};
}

#endif  // __HIPCC__

}  // namespace libra
