// The gradient's pass of norms with rotary positions.  With u = w n, n = x r, r = 1 / sqrt(mean(x^2)
// + eps) and y = R u (R the turn times the amplitude):
//   du = R^T dy,  dw = sum over rows and heads of du n,
//   dx = r (w du - n mean(w du n)) = r (w du - x r^2 mean(w du x)).
// x^2 and w du x are summed over a head together, so x and dy are read once and dx written once:
// bound by HBM.  Where the second sum leaves float32's range (heads whose squares do, so that n is 0,
// or gradients of 1e19 and more) that of w du n takes its place.  A workgroup takes rows in turns and
// keeps its part of dw in registers, eight channels a thread; the parts go to the workspace, and a
// second launch adds them in a fixed order.
//
// 16,381 rows of 40 query and 8 key heads (bf16, 604 MB): 124-128 us, 4.7-4.9 TB/s (streams of two reads
// to a write reach 6.3), and 5 for the second launch, which is a chain of a launch, one round of loads
// and a reduction.  Four heads' loads at once took the first launch from 164 us to 118, 1,024 threads to
// 16 channels the second from 22 to 8.
#include <algorithm>
#include <type_traits>

#include "drafts.h"
#include "row_types.h"

namespace libra {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = kMaxRotaryDim / 2;
// Workgroups of one tensor: with both, four to a CU, which run at once.  With 256, 512 and 1,024 of them
// the whole pass (40 / 8 heads of bf16) took 29.4, 27.3 and 30.9 us at 1,021 rows, 78, 65 and 67 at
// 4,093, 259, 201 and 199 at 16,381; 1,024 divided by the tensors' heads 30, 72 and 222.
constexpr int kMaxParts = 512;
// Bytes of dx from which nothing goes through the caches.  40 / 8 heads of bf16 between copies that
// write x and dy and read dx, all three, past and through the caches: 2,003 rows (25 MB) 94 and 92
// us, 4,093 150 and 150, 8,191 298 and 308, 10,007 353 and 366; with cold caches 36 and 45 a launch at
// 4,093 rows, 61 and 78 at 8,191.
constexpr int64_t kPastBytes = int64_t(32) << 20;

template <class T>
struct BackArgs {
  const typename T::Elem* x;
  const typename T::Elem* dy;
  typename T::Elem* dx;
  int64_t x_row, x_head, dy_row, dy_head, dx_row, dx_head;
  HeadNorm norm;
  float* parts;  // [blocks][dim]
  int heads, blocks;
  int head_slots, block_rows;  // wide form: heads and rows that a workgroup takes at once
};
struct BackCall {
  const int32_t* positions;
  int64_t rows;
  int dim;
};

// Wide form: a power of two of channels, R a multiple of 8, everything aligned for four channels.
// A thread owns two quads of a head: four pairs, or eight channels that are not turned.
template <class T, bool kInter, int kHeads, bool kPastCaches>
__device__ __forceinline__ void back_wide(const RotaryArgs<kMaxPairs>& rot, const BackArgs<T>& A,
                                          const BackCall& C, int block, float (*sums)[8]) {
  using Quad = typename T::Quad;
  const int per_head = C.dim / 8, per_row = A.head_slots * per_head;
  const int t = threadIdx.x;
  const int r = t / per_row, in_row = t - r * per_row;
  const int h0 = in_row / per_head, j = in_row - h0 * per_head;
  const int R8 = rot.rdim / 8;
  const bool turned = j < R8;
  const int2 qd = quads_of<T, kInter>(j, R8, per_head);
  float wa[4], wb[4], da[4] = {}, db[4] = {};
  norm_weights(A.norm, 4 * qd.x, wa);
  norm_weights(A.norm, 4 * qd.y, wb);
  if (r < A.block_rows) {
    for (int64_t row = int64_t(block) * A.block_rows + r; row < C.rows; row += int64_t(A.blocks) * A.block_rows) {
      float2 cs[4];
      if (turned) {
        const int32_t pos = C.positions[row];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          cs[i] = rotary_cos_sin(rot.turn[pair_of<kInter>(qd, j, i)], pos, rot.amplitude);
          cs[i].y = -cs[i].y;
        }
      }
      for (int hb = h0; hb < A.heads; hb += kHeads * A.head_slots) {
        Quad xa[kHeads], xb[kHeads], ya[kHeads], yb[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
          const int h = hb + i * A.head_slots;
          if (h >= A.heads) continue;
          const typename T::Elem* x = A.x + row * A.x_row + h * A.x_head;
          const typename T::Elem* dy = A.dy + row * A.dy_row + h * A.dy_head;
          xa[i] = load_quad<kPastCaches>(reinterpret_cast<const Quad*>(x + 4 * qd.x));
          xb[i] = load_quad<kPastCaches>(reinterpret_cast<const Quad*>(x + 4 * qd.y));
          ya[i] = load_quad<kPastCaches>(reinterpret_cast<const Quad*>(dy + 4 * qd.x));
          yb[i] = load_quad<kPastCaches>(reinterpret_cast<const Quad*>(dy + 4 * qd.y));
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
          const int h = hb + i * A.head_slots;
          if (h >= A.heads) continue;  // a head's threads all take part, or none
          float f[4], g[4], u[4], v[4];
          T::unpack(xa[i], f);
          T::unpack(xb[i], g);
          T::unpack(ya[i], u);
          T::unpack(yb[i], v);
          if (turned) {
            float y[4], z[4];
            turn_values<kInter>(u, v, cs, y, z);
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = y[e], v[e] = z[e];
          }
          float squares = 0.f, along = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(f[e], f[e], squares);
#pragma unroll
          for (int e = 0; e < 4; ++e) squares = __builtin_fmaf(g[e], g[e], squares);
#pragma unroll
          for (int e = 0; e < 4; ++e) along = __builtin_fmaf(u[e] * wa[e], f[e], along);
#pragma unroll
          for (int e = 0; e < 4; ++e) along = __builtin_fmaf(v[e] * wb[e], g[e], along);
          const float s = norm_scale(group_sum(squares, per_head), C.dim, A.norm.eps);
          float m = group_sum(along, per_head) * s / float(C.dim);  // mean(w du n)
          if (!__builtin_isfinite(m)) {  // the same in a head's threads
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) t = __builtin_fmaf(u[e] * wa[e], f[e] * s, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) t = __builtin_fmaf(v[e] * wb[e], g[e] * s, t);
            m = group_sum(t, per_head) / float(C.dim);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float n = f[e] * s, o = g[e] * s;
            da[e] = __builtin_fmaf(u[e], n, da[e]);
            db[e] = __builtin_fmaf(v[e], o, db[e]);
            f[e] = s * __builtin_fmaf(-n, m, u[e] * wa[e]);
            g[e] = s * __builtin_fmaf(-o, m, v[e] * wb[e]);
          }
          typename T::Elem* dx = A.dx + row * A.dx_row + h * A.dx_head;
          store_quad<kPastCaches>(reinterpret_cast<Quad*>(dx + 4 * qd.x), T::pack(f));
          store_quad<kPastCaches>(reinterpret_cast<Quad*>(dx + 4 * qd.y), T::pack(g));
        }
      }
    }
  }
  if (!A.parts) return;  // uniform over the workgroup
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[t][e] = da[e], sums[t][4 + e] = db[e];
  __syncthreads();
  const int used = per_row * A.block_rows;
  for (int c = t; c < C.dim; c += kThreads) {  // value c % 8 of piece c / 8
    float sum = 0.f;
    for (int i = c / 8; i < used; i += per_head) sum += sums[i][c % 8];
    const int2 q = quads_of<T, kInter>(c / 8, R8, per_head);
    A.parts[size_t(block) * C.dim + 4 * (c % 8 < 4 ? q.x : q.y) + c % 4] = sum;
  }
}

template <class T, bool kInter, int kHeads, bool kPastCaches>
__global__ __launch_bounds__(kThreads) void norm_back_wide_kernel(RotaryArgs<kMaxPairs> rot, BackArgs<T> Q,
                                                                  BackArgs<T> K, BackCall C) {
  __shared__ float sums[kThreads][8];
  const int i = int(blockIdx.x);
  if (i < Q.blocks) back_wide<T, kInter, kHeads, kPastCaches>(rot, Q, C, i, sums);
  else back_wide<T, kInter, kHeads, kPastCaches>(rot, K, C, i - Q.blocks, sums);
}

// Any head size, R, alignment: a wave per head, whose values go through LDS, where a channel finds
// its partner.  A pass of 4,093 rows of 40 / 8 heads in bf16 (norms, gradients and their sum) takes
// 268-272 us at head sizes 80 and 96 and at R = 20, 67 in the wide form; 2,047 rows in float32 144-158
// and 57.  So a head takes the same time whatever its bytes: instructions and their latency bound it.
template <class T>
__device__ __forceinline__ void back_any(const RotaryArgs<kMaxPairs>& rot, const BackArgs<T>& A,
                                         const BackCall& C, int block, float (*shared)[kMaxRotaryHead]) {
  constexpr int kPer = kMaxRotaryHead / 64, kWaves = kThreads / 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* const u = shared[wave];
  float dw[kPer] = {};
  const int64_t vectors = C.rows * A.heads;
  for (int64_t at = int64_t(block) * kWaves + wave; at < vectors; at += int64_t(A.blocks) * kWaves) {
    const int64_t row = at / A.heads;
    const int h = int(at - row * A.heads);
    const typename T::Elem* x = A.x + row * A.x_row + h * A.x_head;
    const typename T::Elem* dy = A.dy + row * A.dy_row + h * A.dy_head;
    typename T::Elem* dx = A.dx + row * A.dx_row + h * A.dx_head;
    float f[kPer], du[kPer], squares = 0.f, along = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = lane + 64 * i;
      f[i] = 0.f;
      if (d < C.dim) f[i] = T::get(x[d]), u[d] = T::get(dy[d]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int32_t pos = C.positions[row];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = lane + 64 * i;
      du[i] = 0.f;
      if (d >= C.dim) continue;
      du[i] = u[d];
      if (d < rot.rdim) {
        const bool first = rot.interleaved ? !(d & 1) : d < rot.rdim / 2;
        const int o = rot.interleaved ? d ^ 1 : first ? d + rot.rdim / 2 : d - rot.rdim / 2;
        float2 cs = rotary_cos_sin(rot.turn[rot.interleaved ? d / 2 : first ? d : o], pos, rot.amplitude);
        cs.y = -cs.y;
        du[i] = first ? turn_first(du[i], u[o], cs) : turn_second(u[o], du[i], cs);
      }
      squares = __builtin_fmaf(f[i], f[i], squares);
      along = __builtin_fmaf(du[i] * norm_weight(A.norm, d), f[i], along);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const float s = norm_scale(group_sum(squares, 64), C.dim, A.norm.eps);
    float m = group_sum(along, 64) * s / float(C.dim);
    if (!__builtin_isfinite(m)) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (lane + 64 * i < C.dim) t = __builtin_fmaf(du[i] * norm_weight(A.norm, lane + 64 * i), f[i] * s, t);
      m = group_sum(t, 64) / float(C.dim);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = lane + 64 * i;
      if (d >= C.dim) continue;
      const float n = f[i] * s;
      dw[i] = __builtin_fmaf(du[i], n, dw[i]);
      dx[d] = T::put(s * __builtin_fmaf(-n, m, du[i] * norm_weight(A.norm, d)));
    }
  }
  if (!A.parts) return;  // uniform over the workgroup
#pragma unroll
  for (int i = 0; i < kPer; ++i) u[lane + 64 * i] = dw[i];
  __syncthreads();
  for (int d = threadIdx.x; d < C.dim; d += kThreads) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += shared[w][d];
    A.parts[size_t(block) * C.dim + d] = sum;
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void norm_back_any_kernel(RotaryArgs<kMaxPairs> rot, BackArgs<T> Q,
                                                                 BackArgs<T> K, BackCall C) {
  __shared__ float shared[kThreads / 64][kMaxRotaryHead];
  const int i = int(blockIdx.x);
  if (i < Q.blocks) back_any<T>(rot, Q, C, i, shared);
  else back_any<T>(rot, K, C, i - Q.blocks, shared);
}

// Adds the workgroups' parts of 16 channels of a weight's gradient: 64 threads to a channel, in
// float64, which costs nothing here and leaves float32's last rounding alone.
struct SumArgs {
  const float* parts[2];
  float* out[2];
  int blocks[2];
  int dim;
};
constexpr int kSumThreads = 1024, kSumRows = kSumThreads / 16;
__global__ __launch_bounds__(kSumThreads) void norm_weight_sum_kernel(SumArgs A) {
  __shared__ double sums[kSumRows][17];
  const int which = blockIdx.y, c = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int d = blockIdx.x * 16 + c, n = A.blocks[which];
  if (!A.out[which]) return;
  double sum = 0;
  if (d < A.dim) {
#pragma unroll
    for (int i = 0; i < kMaxParts / kSumRows; ++i)
      if (k + i * kSumRows < n) sum += double(A.parts[which][size_t(k + i * kSumRows) * A.dim + d]);
  }
  sums[k][c] = sum;
  __syncthreads();
  if (k < 8)
    for (int i = k + 8; i < kSumRows; i += 8) sum += sums[i][c];
  __syncthreads();
  if (k < 8) sums[k][c] = sum;
  __syncthreads();
  if (k > 0 || d >= A.dim) return;
  for (int i = 1; i < 8; ++i) sum += sums[i][c];
  A.out[which][d] = float(sum);
}

bool aligned_quads(const void* p, int64_t row, int64_t head, size_t quad) {
  return reinterpret_cast<uintptr_t>(p) % quad == 0 && ((row | head) & 3) == 0;
}

template <class T>
bool wide_rows(const NormBackRows& a) {
  const size_t quad = sizeof(typename T::Quad);
  return !a.heads || (aligned_quads(a.x, a.x_row, a.x_head, quad) && aligned_quads(a.dy, a.dy_row, a.dy_head, quad) &&
                      aligned_quads(a.dx, a.dx_row, a.dx_head, quad));
}

template <class T>
hipError_t back(const Rotary& r, const NormBackRows& q, const NormBackRows& k, const RowNorms& norms,
                const int32_t* positions, int64_t rows, void* ws, hipStream_t s) {
  const int dim = r.head_dim;
  const bool wide = r.rotary_dim % 8 == 0 && dim % 8 == 0 && (dim & (dim - 1)) == 0 && wide_rows<T>(q) && wide_rows<T>(k);
  float* const parts = static_cast<float*>(ws);
  auto args = [&](const NormBackRows& a, const HeadNorm& n, int which) {
    BackArgs<T> A{};
    A.x = static_cast<const typename T::Elem*>(a.x);
    A.dy = static_cast<const typename T::Elem*>(a.dy);
    A.dx = static_cast<typename T::Elem*>(a.dx);
    A.x_row = a.x_row, A.x_head = a.x_head, A.dy_row = a.dy_row, A.dy_head = a.dy_head;
    A.dx_row = a.dx_row, A.dx_head = a.dx_head;
    A.norm = n;
    A.heads = a.heads;
    A.parts = a.dweight ? parts + size_t(which) * kMaxParts * dim : nullptr;
    if (!a.heads) return A;
    int64_t blocks;
    if (wide) {
      A.head_slots = std::min(a.heads, kThreads / (dim / 8));
      A.block_rows = kThreads / (A.head_slots * (dim / 8));
      blocks = (rows + A.block_rows - 1) / A.block_rows;
    } else {
      blocks = (rows * a.heads + kThreads / 64 - 1) / (kThreads / 64);
    }
    A.blocks = int(std::min<int64_t>(blocks, kMaxParts));
    return A;
  };
  const BackArgs<T> Q = args(q, norms.q, 0), K = args(k, norms.k, 1);
  const BackCall C{positions, rows, dim};
  const int64_t bytes = rows * (q.heads + k.heads) * dim * int64_t(sizeof(typename T::Elem));
  const bool past = bytes >= kPastBytes;
  auto wide_form = [&](auto pairing) {
    constexpr bool kInter = decltype(pairing)::value;
    return past ? norm_back_wide_kernel<T, kInter, 4, true> : norm_back_wide_kernel<T, kInter, 4, false>;
  };
  auto form = !wide ? norm_back_any_kernel<T>
              : r.pairing == LIBRA_ROTARY_INTERLEAVED ? wide_form(std::true_type{}) : wide_form(std::false_type{});
  if (Q.blocks + K.blocks > 0) {  // none without rows, whose weight gradients are 0
    hipLaunchKernelGGL(form, dim3(unsigned(Q.blocks + K.blocks)), dim3(kThreads), 0, s, rotary_args<kMaxPairs>(r), Q, K, C);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!q.dweight && !k.dweight) return hipSuccess;
  const SumArgs S{{Q.parts, K.parts}, {q.dweight, k.dweight}, {Q.blocks, K.blocks}, dim};
  hipLaunchKernelGGL(norm_weight_sum_kernel, dim3(unsigned((dim + 15) / 16), 2), dim3(kSumThreads), 0, s, S);
  return hipGetLastError();
}

}  // namespace

size_t norm_back_workspace(int32_t head_dim) { return size_t(2) * kMaxParts * head_dim * sizeof(float); }

hipError_t launch_norm_back(const Rotary& r, int32_t dtype, const NormBackRows& q, const NormBackRows& k,
                            const RowNorms& norms, const int32_t* positions, int64_t rows, void* ws,
                            hipStream_t s) {
  switch (dtype) {
    case LIBRA_DTYPE_BF16: return back<Bf16>(r, q, k, norms, positions, rows, ws, s);
    case LIBRA_DTYPE_FP16: return back<Fp16>(r, q, k, norms, positions, rows, ws, s);
    default: return back<Fp32>(r, q, k, norms, positions, rows, ws, s);
  }
}

}  // namespace libra
