// Entry points of the drafted step's operators (declared and documented in include/libra.h).
#include <cfloat>
#include <climits>
#include <cmath>
#include <initializer_list>
#include <string>

#include "drafts.h"
#include "row_checks.h"

using namespace libra;

namespace {

constexpr libra_norm_heads kNoHeads{};
constexpr int32_t kMaxBatch = 1 << 30;  // indices behind the last one, in turns, fit 32 bits

bool known_dtype(int32_t d) {
  return d == LIBRA_DTYPE_BF16 || d == LIBRA_DTYPE_FP16 || d == LIBRA_DTYPE_FP32;
}
size_t dtype_size(int32_t d) { return d == LIBRA_DTYPE_FP32 ? 4 : 2; }

// Whether the arrays (of 32-bit values; some may be NULL) are aligned, with the error set if not.
bool int32_arrays(std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (!aligned_to(p, 4)) return set_error(LIBRA_E_INVAL, "32-bit arrays must be 4-byte aligned"), false;
  return true;
}

libra_status check_eps(float eps) {
  // Below the normal numbers v_rsq_f32 takes 0 for it, and a head of zeros would give NaN.
  if (!(eps >= FLT_MIN) || !std::isfinite(eps))
    return set_error(LIBRA_E_INVAL, "eps must be positive, finite and no subnormal number");
  return LIBRA_OK;
}

libra_status check_weight(const void* w, int32_t dtype, const char* what) {
  if (!w) return set_error(LIBRA_E_INVAL, std::string(what) + " is NULL");
  if (!aligned_to(w, dtype_size(dtype)))
    return set_error(LIBRA_E_INVAL, std::string(what) + " must be aligned to its type");
  return LIBRA_OK;
}

// One of a call's tensors, rows x num_heads vectors; written: whether its vectors must be apart.
libra_status check_heads(const void* p, int64_t rows, int32_t heads, int32_t dim, int64_t row, int64_t head,
                         size_t size, bool written, const char* tensor, const char* part) {
  const char* wrong = nullptr;
  if (!p) wrong = " is NULL";
  else if (!aligned_to(p, size)) wrong = " must be aligned to its type";
  else if (row < 0 || head < 0 || !addressable(rows, heads, row, head))
    wrong = ": strides must be >= 0, and offsets below 2^56 elements";
  else if (written && !disjoint(rows, heads, dim, row, head)) wrong = "'s heads overlap each other";
  return wrong ? set_error(LIBRA_E_INVAL, std::string(tensor) + part + wrong) : LIBRA_OK;
}

// Whether the written tensor, where it is an input, has its strides.
bool in_place(const void* a, int64_t a_row, int64_t a_head, const libra_norm_heads& t, int64_t rows) {
  return a != t.out || ((rows <= 1 || a_row == t.out_row_stride) &&
                        (t.num_heads <= 1 || a_head == t.out_head_stride));
}

libra_status check_norm(libra_rotary rotary, int32_t dtype, int32_t weight_dtype, float eps,
                        const int32_t* positions, int64_t rows, int32_t head_dim,
                        const libra_norm_heads& q, const libra_norm_heads& k, bool backward) {
  if (!rotary) return set_error(LIBRA_E_INVAL, "rotary is NULL");
  if (head_dim != rotary->head_dim)
    return set_error(LIBRA_E_INVAL, "head_dim differs from the rotary's");
  if (!known_dtype(dtype) || !known_dtype(weight_dtype))
    return set_error(LIBRA_E_UNSUPPORTED, "dtype and weight_dtype must be bf16, fp16 or fp32");
  libra_status st = check_eps(eps);
  if (st != LIBRA_OK) return st;
  if (rows < 0 || q.num_heads < 0 || k.num_heads < 0)
    return set_error(LIBRA_E_INVAL, "rows / num_heads < 0");
  if (rows > INT32_MAX || q.num_heads > 65535 || k.num_heads > 65535)
    return set_error(LIBRA_E_UNSUPPORTED, "rows must be < 2^31 and num_heads <= 65535");
  const size_t size = dtype_size(dtype);
  for (const libra_norm_heads* t : {&q, &k}) {
    if (!t->num_heads) continue;
    const char* const name = t == &q ? "q" : "k";
    st = check_weight(t->weight, weight_dtype, t == &q ? "q's weight" : "k's weight");
    if (st != LIBRA_OK) return st;
    if (backward && t->weight_grad && !aligned_to(t->weight_grad, 4))
      return set_error(LIBRA_E_INVAL, std::string(name) + "'s weight_grad must be aligned to float32");
    if (rows == 0) continue;
    st = check_heads(t->x, rows, t->num_heads, head_dim, t->x_row_stride, t->x_head_stride, size, false, name, "'s x");
    if (st == LIBRA_OK)
      st = check_heads(t->out, rows, t->num_heads, head_dim, t->out_row_stride, t->out_head_stride, size, true, name, "'s out");
    if (st == LIBRA_OK && backward)
      st = check_heads(t->grad, rows, t->num_heads, head_dim, t->grad_row_stride, t->grad_head_stride, size, false, name, "'s grad");
    if (st != LIBRA_OK) return st;
    if (!in_place(t->x, t->x_row_stride, t->x_head_stride, *t, rows) ||
        (backward && !in_place(t->grad, t->grad_row_stride, t->grad_head_stride, *t, rows)))
      return set_error(LIBRA_E_INVAL, std::string("in place, ") + name + "'s tensors need the same strides");
  }
  if (rows > 0 && q.num_heads + k.num_heads > 0 && !positions)
    return set_error(LIBRA_E_INVAL, "positions is NULL");
  return LIBRA_OK;
}

}  // namespace

extern "C" {

libra_status libra_kv_map(int32_t batch, const int32_t* prior_lens, const int32_t* new_lens,
                          const int32_t* held_pages, int32_t* block_table, int32_t bt_stride,
                          int32_t* free_pages, int64_t free_capacity, const int32_t* num_free,
                          const int32_t* depths, int64_t rows, int64_t* slots, int32_t* positions,
                          int32_t* row_starts, int32_t* held_out, int32_t* num_free_out,
                          int32_t* refused, void* stream) {
  if (batch < 0 || bt_stride < 0 || free_capacity < 0 || rows < 0)
    return set_error(LIBRA_E_INVAL, "batch / bt_stride / free_capacity / rows < 0");
  if (rows > INT32_MAX || free_capacity > INT32_MAX)
    return set_error(LIBRA_E_UNSUPPORTED, "rows and free_capacity must be < 2^31");
  if (batch > kMaxBatch) return set_error(LIBRA_E_UNSUPPORTED, "batch must be <= 2^30");
  if (!num_free || !num_free_out || !row_starts)
    return set_error(LIBRA_E_INVAL, "num_free, num_free_out or row_starts is NULL");
  if (batch > 0 && (!prior_lens || !new_lens || !held_pages || !held_out || !refused ||
                    (bt_stride > 0 && !block_table)))
    return set_error(LIBRA_E_INVAL, "a per-request array is NULL");
  if (free_capacity > 0 && !free_pages) return set_error(LIBRA_E_INVAL, "free_pages is NULL");
  if (rows > 0 && (!slots || !positions)) return set_error(LIBRA_E_INVAL, "slots or positions is NULL");
  if (!int32_arrays({prior_lens, new_lens, held_pages, block_table, free_pages, num_free, depths, positions,
                     row_starts, held_out, num_free_out, refused}))
    return LIBRA_E_INVAL;
  if (!aligned_to(slots, 8)) return set_error(LIBRA_E_INVAL, "slots must be 8-byte aligned");
  const MapArgs a{prior_lens, new_lens, held_pages, block_table, bt_stride, free_pages, free_capacity,
                  num_free, depths, slots, positions, row_starts, held_out, num_free_out, refused,
                  batch, rows};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_TABLES, static_cast<hipStream_t>(stream), true);
    e = launch_kv_map(a, static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "table launch");
}

libra_status libra_kv_accept(libra_kv_layout layout, int32_t batch, const int32_t* prior_lens,
                             const int32_t* accepted, int32_t max_accepted, const int32_t* counts,
                             const int32_t* block_table, int32_t bt_stride, void* stream) {
  if (!layout) return set_error(LIBRA_E_INVAL, "layout is NULL");
  if (batch < 0 || max_accepted < 0 || bt_stride < 0)
    return set_error(LIBRA_E_INVAL, "batch / max_accepted / bt_stride < 0");
  if (batch == 0 || max_accepted == 0 || bt_stride == 0) return LIBRA_OK;
  if (!int32_arrays({prior_lens, accepted, counts, block_table})) return LIBRA_E_INVAL;
  const int32_t hkv = layout->desc.num_kv_heads;
  if (int64_t(batch) * hkv > INT32_MAX)
    return set_error(LIBRA_E_UNSUPPORTED, "batch * num_kv_heads must be < 2^31");
  if (max_accepted > kMaxBatch) return set_error(LIBRA_E_UNSUPPORTED, "max_accepted must be <= 2^30");
  if (!prior_lens || !accepted || !counts || !block_table)
    return set_error(LIBRA_E_INVAL, "prior_lens, accepted, counts or block_table is NULL");
  const AcceptArgs a{static_cast<uint16_t*>(layout->desc.k_cache), static_cast<uint16_t*>(layout->desc.v_cache),
                     layout->desc.num_pages, hkv, prior_lens, accepted, counts, batch, max_accepted,
                     block_table, bt_stride};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_ACCEPT, static_cast<hipStream_t>(stream), true);
    e = launch_kv_accept(a, static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "accept launch");
}

libra_status libra_qk_norm_rotary(libra_rotary rotary, int32_t dtype, int32_t weight_dtype, float eps,
                                  const int32_t* positions, int64_t rows, int32_t head_dim,
                                  const libra_norm_heads* q, const libra_norm_heads* k, void* stream) {
  const libra_norm_heads &tq = q ? *q : kNoHeads, &tk = k ? *k : kNoHeads;
  const libra_status st = check_norm(rotary, dtype, weight_dtype, eps, positions, rows, head_dim, tq, tk, false);
  if (st != LIBRA_OK) return st;
  if (rows == 0 || tq.num_heads + tk.num_heads == 0) return LIBRA_OK;
  auto as_rows = [&](const libra_norm_heads& t) {
    return RotaryRows{t.x, t.out, t.x_row_stride, t.x_head_stride, t.out_row_stride, t.out_head_stride,
                      positions, rows, t.num_heads, dtype, false};
  };
  const RowNorms norms{head_norm(tq.weight, weight_dtype, eps), head_norm(tk.weight, weight_dtype, eps)};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_ROTARY, static_cast<hipStream_t>(stream), true);
    e = launch_norm_rotary(*rotary, as_rows(tq), as_rows(tk), norms, static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "norm launch");
}

size_t libra_qk_norm_rotary_workspace_bytes(int64_t rows, int32_t num_q_heads, int32_t num_k_heads,
                                            int32_t head_dim) {
  if (rows < 0 || num_q_heads < 0 || num_k_heads < 0 || head_dim < 0) return 0;
  return norm_back_workspace(head_dim);
}

libra_status libra_qk_norm_rotary_backward(libra_rotary rotary, int32_t dtype, int32_t weight_dtype,
                                           float eps, const int32_t* positions, int64_t rows,
                                           int32_t head_dim, const libra_norm_heads* q,
                                           const libra_norm_heads* k, void* workspace, size_t ws_bytes,
                                           void* stream) {
  const libra_norm_heads &tq = q ? *q : kNoHeads, &tk = k ? *k : kNoHeads;
  const libra_status st = check_norm(rotary, dtype, weight_dtype, eps, positions, rows, head_dim, tq, tk, true);
  if (st != LIBRA_OK) return st;
  if (tq.num_heads + tk.num_heads == 0) return LIBRA_OK;
  float* const dq = tq.num_heads ? tq.weight_grad : nullptr;
  float* const dk = tk.num_heads ? tk.weight_grad : nullptr;
  if (rows == 0 && !dq && !dk) return LIBRA_OK;
  if (dq || dk) {
    if (!workspace || !aligned16(workspace))
      return set_error(LIBRA_E_INVAL, "workspace is NULL or not 16-byte aligned");
    if (ws_bytes < norm_back_workspace(head_dim))
      return set_error(LIBRA_E_WORKSPACE, "workspace smaller than libra_qk_norm_rotary_workspace_bytes");
    if (dq && dq == dk) return set_error(LIBRA_E_INVAL, "q's and k's weight_grad are the same");
  }
  auto as_rows = [&](const libra_norm_heads& t, float* dw) {
    return NormBackRows{t.x, t.grad, t.out, t.x_row_stride, t.x_head_stride, t.grad_row_stride,
                        t.grad_head_stride, t.out_row_stride, t.out_head_stride, t.num_heads, dw};
  };
  const RowNorms norms{head_norm(tq.weight, weight_dtype, eps), head_norm(tk.weight, weight_dtype, eps)};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_ROTARY, static_cast<hipStream_t>(stream), true);
    e = launch_norm_back(*rotary, dtype, as_rows(tq, dq), as_rows(tk, dk), norms, positions, rows, workspace,
                         static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "norm gradient launch");
}

libra_status libra_kv_append_norm(libra_kv_layout layout, libra_rotary rotary, int32_t weight_dtype,
                                  float eps, const int32_t* positions, const int64_t* slots, int64_t rows,
                                  const void* q, int64_t q_row_stride, int32_t num_q_heads,
                                  const void* q_weight, const void* k_new, int64_t k_row_stride,
                                  const void* k_weight, const void* v_new, int64_t v_row_stride,
                                  int32_t num_kv_heads, void* q_out, void* stream) {
  if (!layout) return set_error(LIBRA_E_INVAL, "layout is NULL");
  if (!rotary) return set_error(LIBRA_E_INVAL, "rotary is NULL");
  if (rows < 0) return set_error(LIBRA_E_INVAL, "rows < 0");
  if (rows > INT32_MAX) return set_error(LIBRA_E_UNSUPPORTED, "rows must be < 2^31");
  if (!known_dtype(weight_dtype))
    return set_error(LIBRA_E_UNSUPPORTED, "weight_dtype must be bf16, fp16 or fp32");
  libra_status st = check_eps(eps);
  if (st != LIBRA_OK) return st;
  if (!q != !q_out) return set_error(LIBRA_E_INVAL, "q and q_out come together");
  st = check_cached(*layout, rotary, num_kv_heads);
  if (st == LIBRA_OK) st = check_weight(k_weight, weight_dtype, "k_weight");
  if (st == LIBRA_OK && q) st = check_weight(q_weight, weight_dtype, "q_weight");
  if (st != LIBRA_OK) return st;
  if (rows == 0) return LIBRA_OK;
  if (!slots || !positions) return set_error(LIBRA_E_INVAL, "slots or positions is NULL");
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
  const RowNorms norms{head_norm(q_weight, weight_dtype, eps), head_norm(k_weight, weight_dtype, eps)};
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_CACHE_WRITE, static_cast<hipStream_t>(stream), true);
    e = launch_kv_append_norm(*layout, n, norms, slots, rows, q ? num_q_heads : 0, q_out,
                              static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "cache append launch");
}

size_t libra_tree_attn_workspace_bytes(int64_t rows, int32_t batch, int32_t num_q_heads,
                                       int32_t num_kv_heads) {
  if (rows < 0 || batch < 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads) return 0;
  return tree_workspace();
}

libra_status libra_tree_attn(libra_kv_layout layout, const void* q, int64_t rows,
                             const int32_t* prior_lens, const int32_t* row_starts, const uint32_t* mask,
                             int32_t mask_words, const int32_t* block_table, int32_t bt_stride,
                             int32_t batch, int32_t num_q_heads, float scale, void* workspace,
                             size_t ws_bytes, void* out, float* lse, void* stream) {
  if (!layout) return set_error(LIBRA_E_INVAL, "layout is NULL");
  if (rows < 0 || batch < 0) return set_error(LIBRA_E_INVAL, "rows / batch < 0");
  const int32_t hkv = layout->desc.num_kv_heads;
  if (num_q_heads <= 0 || num_q_heads % hkv)
    return set_error(LIBRA_E_INVAL, "num_q_heads must be a positive multiple of the layout's num_kv_heads");
  if (num_q_heads / hkv > LIBRA_MAX_GROUP)
    return set_error(LIBRA_E_UNSUPPORTED, "num_q_heads / num_kv_heads > 16");
  if (rows > INT32_MAX / num_q_heads)
    return set_error(LIBRA_E_UNSUPPORTED, "rows * num_q_heads must be < 2^31");
  if (batch > kMaxBatch) return set_error(LIBRA_E_UNSUPPORTED, "batch must be <= 2^30");
  if (!(scale > 0.f) || !std::isfinite(scale))
    return set_error(LIBRA_E_INVAL, "scale must be positive and finite");
  if (mask ? mask_words < 1 : mask_words != 0)
    return set_error(LIBRA_E_INVAL, "mask_words must be positive with a mask, 0 without");
  if (mask_words > LIBRA_MAX_MASK_WORDS)
    return set_error(LIBRA_E_UNSUPPORTED, "mask_words must be <= LIBRA_MAX_MASK_WORDS");
  if (rows == 0 || batch == 0) return LIBRA_OK;
  if (!q || !out) return set_error(LIBRA_E_INVAL, "q / out is NULL");
  if (!aligned16(q) || !aligned16(out)) return set_error(LIBRA_E_INVAL, "q / out must be 16-byte aligned");
  if (q == out) return set_error(LIBRA_E_INVAL, "q and out must be apart");
  if (!prior_lens || !row_starts || !block_table)
    return set_error(LIBRA_E_INVAL, "prior_lens, row_starts or block_table is NULL");
  if (!int32_arrays({prior_lens, row_starts, mask, block_table, lse})) return LIBRA_E_INVAL;
  if (bt_stride < 1) return set_error(LIBRA_E_INVAL, "bt_stride must be positive");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)
    return set_error(LIBRA_E_INVAL, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < tree_workspace())
    return set_error(LIBRA_E_WORKSPACE, "workspace smaller than libra_tree_attn_workspace_bytes");
  const TreeCall c{q, rows, prior_lens, row_starts, mask, mask_words, block_table, bt_stride, batch,
                   num_q_heads, scale, workspace, out, lse};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  {
    ProfScope ps(LIBRA_KERNEL_TREE, s, true);
    e = launch_tree(*layout, c, s);
  }
  if (e != hipSuccess) return hip_error(e, "tree attention launch");
  {
    ProfScope ps(LIBRA_KERNEL_MERGE, s, true);
    e = launch_tree_merge(*layout, c, s);
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "tree merge launch");
}

}  // extern "C"
