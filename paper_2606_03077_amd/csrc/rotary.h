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
// (p 2^-65 turns), whatever the position and the frequency; float32 angles lose 2^-24 p theta.
// theta_j itself is a given double, or computed in long double (64 bits).  The fraction's
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

// Granules (8 channels) of a bf16 row of 128 channels and their channels' partners in the
// pairs, loaded together so that their latencies overlap.
template <int N>
struct Granules {
  uint4 own[N], partner[N];
};

// Whether a granule's partners are a granule too (or the granule itself).
__device__ __forceinline__ bool granules_pair(int rdim, int interleaved) {
  return (rdim & (interleaved ? 7 : 15)) == 0;
}

template <int N>
__device__ __forceinline__ void load_granules(Granules<N>& in, const uint16_t* row,
                                              const int (&gi)[N], int rdim, int interleaved) {
#pragma unroll
  for (int i = 0; i < N; ++i) in.own[i] = *reinterpret_cast<const uint4*>(row + 8 * gi[i]);
  const int h = rdim / 2;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint4 w = in.own[i];
      in.partner[i] = make_uint4(w.x >> 16 | w.x << 16, w.y >> 16 | w.y << 16,
                                 w.z >> 16 | w.z << 16, w.w >> 16 | w.w << 16);
    }
  } else if (granules_pair(rdim, interleaved)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = 8 * gi[i];
      in.partner[i] =
          *reinterpret_cast<const uint4*>(row + (d < h ? d + h : d < rdim ? d - h : d));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      in.partner[i] = in.own[i];
      if (8 * gi[i] >= rdim) continue;
      auto at = [&](int e) -> uint32_t {
        const int d = 8 * gi[i] + e;
        return row[d < h ? d + h : d < rdim ? d - h : d];
      };
      in.partner[i] = make_uint4(at(0) | at(1) << 16, at(2) | at(3) << 16, at(4) | at(5) << 16,
                                 at(6) | at(7) << 16);
    }
  }
}

// Turns the granules: hi is bf16 (nearest), lo (if kLow) what that leaves of the float32
// values, as bf16 again, so that both together hold 16 bits.  Nothing is left of copied
// channels and of values that bf16 makes infinite or NaN.  cs: the row's (cos, sin) by pair.
template <int N, bool kLow, bool kPaired>
__device__ __forceinline__ void turn_granules_as(const Granules<N>& in, const int (&gi)[N],
                                                 const float2* cs, int rdim, int interleaved,
                                                 uint4 (&hi)[N], uint4 (&lo)[N]) {
  const int h = rdim / 2;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int d0 = 8 * gi[i];
    const uint32_t own[4] = {in.own[i].x, in.own[i].y, in.own[i].z, in.own[i].w};
    const uint32_t oth[4] = {in.partner[i].x, in.partner[i].y, in.partner[i].z, in.partner[i].w};
    uint32_t ho[4], lw[4];
    // Past the last pair: any entry, its result is not used.
    const int base = d0 >= rdim ? 0 : interleaved ? d0 / 2 : d0 < h ? d0 : d0 - h;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float y[2], left[2];
      bool turned[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = d0 + 2 * w + e;
        turned[e] = d < rdim;
        float2 t;
        bool first;
        if constexpr (kPaired) {
          t = cs[base + ((2 * w + e) >> interleaved)];
          first = interleaved ? e == 0 : d0 < h;
        } else {
          t = cs[!turned[e] ? 0 : interleaved ? d / 2 : d < h ? d : d - h];
          first = interleaved ? e == 0 : d < h;
        }
        const float x = bf16_to_f32((own[w] >> (16 * e)) & 0xFFFF);
        const float o = bf16_to_f32((oth[w] >> (16 * e)) & 0xFFFF);
        y[e] = __builtin_fmaf(x, t.x, o * (first ? -t.y : t.y));  // as turn_first / turn_second
      }
      const uint32_t b = rotary_pack_bf16(y[0], y[1]);
      const uint32_t keep = (turned[0] ? 0u : 0x0000FFFFu) | (turned[1] ? 0u : 0xFFFF0000u);
      ho[w] = (own[w] & keep) | (b & ~keep);
      if constexpr (kLow) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float r = bf16_to_f32((b >> (16 * e)) & 0xFFFF);
          left[e] = turned[e] && __builtin_isfinite(r) ? y[e] - r : 0.f;
        }
        lw[w] = rotary_pack_bf16(left[0], left[1]);
      }
    }
    hi[i] = make_uint4(ho[0], ho[1], ho[2], ho[3]);
    if constexpr (kLow) lo[i] = make_uint4(lw[0], lw[1], lw[2], lw[3]);
  }
}

template <int N, bool kLow>
__device__ __forceinline__ void turn_granules(const Granules<N>& in, const int (&gi)[N],
                                              const float2* cs, int rdim, int interleaved,
                                              uint4 (&hi)[N], uint4 (&lo)[N]) {
  // rdim may differ between lanes where it is 0 (copies) or the row's.
  if (granules_pair(rdim, interleaved))
    turn_granules_as<N, kLow, true>(in, gi, cs, rdim, interleaved, hi, lo);
  else
    turn_granules_as<N, kLow, false>(in, gi, cs, rdim, interleaved, hi, lo);
}

#endif  // __HIPCC__

}  // namespace libra
