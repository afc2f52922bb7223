// Entry points of the rotary operators (declared and documented in include/libra.h).
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "rotary_calls.h"
#include "row_checks.h"
#include "turns.h"

using namespace libra;

namespace {

constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;

bool positive(double x) { return std::isfinite(x) && x > 0; }

libra_status fill(const libra_rotary_desc& d, Rotary* r) {
  if (d.head_dim < 2 || d.head_dim > kMaxRotaryHead)
    return set_error(LIBRA_E_UNSUPPORTED, "head_dim must lie in [2, 512]");
  const int R = d.rotary_dim == 0 ? d.head_dim : d.rotary_dim;
  if (R < 2 || R % 2 || R > d.head_dim)
    return set_error(LIBRA_E_INVAL, "rotary_dim must be even and lie in [2, head_dim]");
  if (R > kMaxRotaryDim) return set_error(LIBRA_E_UNSUPPORTED, "rotary_dim must be <= 256");
  if (d.pairing != LIBRA_ROTARY_HALF && d.pairing != LIBRA_ROTARY_INTERLEAVED)
    return set_error(LIBRA_E_INVAL, "unknown pairing");
  if (!d.frequencies && !positive(d.base))
    return set_error(LIBRA_E_INVAL, "base must be positive and finite");
  if (d.amplitude != 0 && (!positive(d.amplitude) || !positive(float(d.amplitude))))
    return set_error(LIBRA_E_INVAL, "amplitude must be positive and finite in float32, or 0 for 1");
  long double base = d.base;
  switch (d.scaling) {
    case LIBRA_ROTARY_PLAIN:
      break;
    case LIBRA_ROTARY_BASE:
      if (d.frequencies)
        return set_error(LIBRA_E_INVAL, "base scaling and explicit frequencies exclude each other");
      if (R == 2) return set_error(LIBRA_E_INVAL, "base scaling needs rotary_dim > 2");
      if (!positive(d.factor)) return set_error(LIBRA_E_INVAL, "factor must be positive and finite");
      base *= std::pow((long double)d.factor, (long double)R / (R - 2));
      break;
    case LIBRA_ROTARY_BANDS:
      if (d.original_length <= 0)
        return set_error(LIBRA_E_INVAL, "original_length must be > 0");
      if (!std::isfinite(d.fast) || !(d.slow >= 0) || !(d.fast > d.slow))
        return set_error(LIBRA_E_INVAL, "bands need fast > slow >= 0, finite");
      [[fallthrough]];
    case LIBRA_ROTARY_LINEAR:
      if (!positive(d.factor)) return set_error(LIBRA_E_INVAL, "factor must be positive and finite");
      break;
    default:
      return set_error(LIBRA_E_INVAL, "unknown scaling");
  }
  r->head_dim = d.head_dim;
  r->rotary_dim = R;
  r->pairing = d.pairing;
  r->amplitude = d.amplitude == 0 ? 1.f : float(d.amplitude);
  for (int j = 0; j < R / 2; ++j) {
    long double th = d.frequencies ? (long double)d.frequencies[j]
                                   : std::pow(base, -2.0L * j / R);
    if (d.scaling == LIBRA_ROTARY_LINEAR) {
      th /= d.factor;
    } else if (d.scaling == LIBRA_ROTARY_BANDS) {
      const long double n = std::fabs(d.original_length * th / kTwoPi);
      long double w = (n - d.slow) / ((long double)d.fast - d.slow);
      w = w < 0 ? 0 : w > 1 ? 1 : w;
      th *= w + (1 - w) / d.factor;
    }
    if (!(std::fabs(th) <= 1e6L))
      return set_error(LIBRA_E_INVAL, "a frequency is not finite or beyond 1e6 radians");
    r->theta[j] = double(th);
    r->turn[j] = rotary_turns(th);
  }
  return LIBRA_OK;
}

}  // namespace

extern "C" {

libra_status libra_rotary_create(const libra_rotary_desc* desc, libra_rotary* out) {
  if (!out) return set_error(LIBRA_E_INVAL, "out is NULL");
  *out = nullptr;
  if (!desc) return set_error(LIBRA_E_INVAL, "rotary descriptor is NULL");
  auto* r = new (std::nothrow) libra_rotary_s();
  if (!r) return set_error(LIBRA_E_NOMEM, "rotary allocation failed");
  const libra_status st = fill(*desc, r);
  if (st != LIBRA_OK) {
    delete r;
    return st;
  }
  *out = r;
  return LIBRA_OK;
}

void libra_rotary_destroy(libra_rotary rotary) { delete rotary; }

libra_status libra_rotary_get(libra_rotary rotary, int32_t* head_dim, int32_t* rotary_dim,
                              double* frequencies, double* amplitude) {
  if (!rotary) return set_error(LIBRA_E_INVAL, "rotary is NULL");
  if (head_dim) *head_dim = rotary->head_dim;
  if (rotary_dim) *rotary_dim = rotary->rotary_dim;
  if (frequencies)
    for (int j = 0; j < rotary->rotary_dim / 2; ++j) frequencies[j] = rotary->theta[j];
  if (amplitude) *amplitude = rotary->amplitude;
  return LIBRA_OK;
}

libra_status libra_rotary_apply(libra_rotary rotary, int32_t dtype, const void* x,
                                int64_t x_row_stride, int64_t x_head_stride,
                                const int32_t* positions, int64_t rows, int32_t num_heads,
                                int32_t head_dim, int32_t backward, void* out,
                                int64_t out_row_stride, int64_t out_head_stride, void* stream) {
  if (!rotary) return set_error(LIBRA_E_INVAL, "rotary is NULL");
  if (head_dim != rotary->head_dim)
    return set_error(LIBRA_E_INVAL, "head_dim differs from the rotary's");
  if (dtype != LIBRA_DTYPE_BF16 && dtype != LIBRA_DTYPE_FP16 && dtype != LIBRA_DTYPE_FP32)
    return set_error(LIBRA_E_UNSUPPORTED, "dtype must be bf16, fp16 or fp32");
  if (rows < 0 || num_heads < 0) return set_error(LIBRA_E_INVAL, "rows / num_heads < 0");
  if (rows == 0 || num_heads == 0) return LIBRA_OK;
  if (rows > INT32_MAX || num_heads > 65535)
    return set_error(LIBRA_E_UNSUPPORTED, "rows must be < 2^31 and num_heads <= 65535");
  if (!x || !out || !positions) return set_error(LIBRA_E_INVAL, "x, out or positions is NULL");
  const size_t size = dtype == LIBRA_DTYPE_FP32 ? 4 : 2;
  if (!aligned_to(x, size) || !aligned_to(out, size))
    return set_error(LIBRA_E_INVAL, "x / out must be aligned to their type");
  if (x_row_stride < 0 || x_head_stride < 0 || out_row_stride < 0 || out_head_stride < 0 ||
      !addressable(rows, num_heads, x_row_stride, x_head_stride) ||
      !addressable(rows, num_heads, out_row_stride, out_head_stride))
    return set_error(LIBRA_E_INVAL, "strides must be >= 0, and offsets below 2^56 elements");
  if (!disjoint(rows, num_heads, rotary->head_dim, out_row_stride, out_head_stride))
    return set_error(LIBRA_E_INVAL, "out's heads overlap each other");
  if (x == out && ((rows > 1 && x_row_stride != out_row_stride) ||
                   (num_heads > 1 && x_head_stride != out_head_stride)))
    return set_error(LIBRA_E_INVAL, "in place, x and out need the same strides");
  const RotaryRows a{x, out, x_row_stride, x_head_stride, out_row_stride, out_head_stride,
                     positions, rows, num_heads, dtype, backward != 0};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_ROTARY, static_cast<hipStream_t>(stream), true);
    e = launch_rotary(*rotary, a, static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "rotary launch");
}

libra_status libra_kv_append(libra_kv_layout layout, libra_rotary rotary,
                             const int32_t* positions, const int64_t* slots, int64_t rows,
                             const void* q, int64_t q_row_stride, int32_t num_q_heads,
                             const void* k_new, int64_t k_row_stride, const void* v_new,
                             int64_t v_row_stride, int32_t num_kv_heads, void* q_out,
                             void* stream) {
  if (!layout) return set_error(LIBRA_E_INVAL, "layout is NULL");
  if (rows < 0) return set_error(LIBRA_E_INVAL, "rows < 0");
  if (rows > INT32_MAX) return set_error(LIBRA_E_UNSUPPORTED, "rows must be < 2^31");
  if (!q != !q_out) return set_error(LIBRA_E_INVAL, "q and q_out come together");
  if (q && !rotary) return set_error(LIBRA_E_INVAL, "q needs a rotary");
  libra_status st = check_cached(*layout, rotary, num_kv_heads);
  if (st != LIBRA_OK) return st;
  if (rows == 0) return LIBRA_OK;
  if (!slots || (rotary && !positions))
    return set_error(LIBRA_E_INVAL, "slots or positions is NULL");
  st = check_rows(k_new, rows, k_row_stride, num_kv_heads, "k_new");
  if (st == LIBRA_OK) st = check_rows(v_new, rows, v_row_stride, num_kv_heads, "v_new");
  if (st != LIBRA_OK) return st;
  if (q) {
    if (num_q_heads <= 0 || num_q_heads > 65535)
      return set_error(LIBRA_E_INVAL, "num_q_heads must lie in [1, 65535] with q");
    st = check_rows(q, rows, q_row_stride, num_q_heads, "q");
    if (st != LIBRA_OK) return st;
    if (!aligned16(q_out)) return set_error(LIBRA_E_INVAL, "q_out must be 16-byte aligned");
    if (q == q_out && q_row_stride != int64_t(num_q_heads) * kDim)
      return set_error(LIBRA_E_INVAL, "in place, q's rows must be dense");
  }
  const NewRows n{rotary, positions, q, k_new, v_new, q_row_stride, k_row_stride, v_row_stride};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_CACHE_WRITE, static_cast<hipStream_t>(stream), true);
    e = launch_kv_append(*layout, n, slots, rows, q ? num_q_heads : 0, q_out,
                         static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "cache append launch");
}

libra_status libra_append_attn_rotary(libra_kv_layout layout, libra_plan plan,
                                      libra_rotary rotary, const int32_t* positions, int64_t rows,
                                      const void* q, int64_t q_row_stride, const void* k_new,
                                      int64_t k_row_stride, const void* v_new,
                                      int64_t v_row_stride, int32_t num_kv_heads,
                                      const int32_t* block_table, int32_t bt_stride,
                                      int32_t batch, int32_t num_q_heads, float scale,
                                      int32_t round_queries, void* workspace, size_t ws_bytes,
                                      void* out, float* lse, void* stream) {
  libra_status st = check_call(layout, plan, LIBRA_MODE_APPEND, q, block_table, bt_stride, batch,
                               num_q_heads, scale, out);
  if (st != LIBRA_OK) return st;
  if (!rotary) return set_error(LIBRA_E_INVAL, "rotary is NULL");
  st = check_cached(*layout, rotary, num_kv_heads);
  if (st != LIBRA_OK) return st;
  if (rows != plan->info.n_rows)
    return set_error(LIBRA_E_INVAL, "rows differ from the plan's new tokens");
  if (rows > 0) {
    st = check_rows(q, rows, q_row_stride, num_q_heads, "q");
    if (st == LIBRA_OK) st = check_rows(k_new, rows, k_row_stride, num_kv_heads, "k_new");
    if (st == LIBRA_OK) st = check_rows(v_new, rows, v_row_stride, num_kv_heads, "v_new");
    if (st != LIBRA_OK) return st;
  }
  if (ws_bytes < plan->ws_bytes)
    return set_error(LIBRA_E_WORKSPACE, "workspace smaller than libra_plan_workspace_bytes");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Plan* form = nullptr;
  st = upload(*plan, workspace, ws_bytes, s, false, &form);
  if (st != LIBRA_OK) return st;
  const Plan& P = *form;
  const KvLayout& L = *layout;
  const NewRows n{rotary, positions, q, k_new, v_new, q_row_stride, k_row_stride, v_row_stride,
                  round_queries != 0};
  // Decode units of up to 8 heads write their rows' tokens themselves, and without chunk rows
  // there are no others.
  const bool fused = P.info.n_chunk == 0 && P.group <= 8;
  if (!fused) {
    hipError_t e;
    {
      ProfScope ps(LIBRA_KERNEL_CACHE_WRITE, s, P.info.n_write_tiles > 0);
      e = launch_cache_write_rotary(L, P, workspace, n, block_table, bt_stride, s);
    }
    if (e != hipSuccess) return hip_error(e, "cache-write launch");
  }
  return run_attention(
      P, workspace, out, lse, s, /*timed=*/true,
      [&](hipStream_t at) {
        return launch_chunk_rotary(L, P, workspace, n, block_table, bt_stride, scale, out, lse, at);
      },
      [&](hipStream_t at) {
        return launch_decode_rotary(L, P, workspace, n, block_table, bt_stride, scale, out, lse, fused,
                                    at);
      });
}

}  // extern "C"
