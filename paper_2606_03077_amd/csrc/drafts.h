// Launchers of the drafted step's operators: norms with rotary positions (rotary.hip, norm.hip),
// block tables and accepted tokens (kv_map.hip), tree attention (tree.hip).
#pragma once

#include "rotary_calls.h"

namespace libra {

// n = x / sqrt(mean(x^2) + eps) over a head's channels, u = w n.
struct HeadNorm {
  const void* weight;  // [head size], of weight_dtype
  int32_t weight_dtype;
  float eps;
  int32_t quads;  // whether the weight is aligned to four of its elements
};
inline HeadNorm head_norm(const void* weight, int32_t dtype, float eps) {
  const size_t quad = dtype == LIBRA_DTYPE_FP32 ? 16 : 8;
  return {weight, dtype, eps, reinterpret_cast<uintptr_t>(weight) % quad == 0};
}
// The norms of a call's queries and keys.
struct RowNorms {
  HeadNorm q, k;
};

// Heads normalised, then turned: queries and keys (either may have no heads).
hipError_t launch_norm_rotary(const Rotary& r, const RotaryRows& q, const RotaryRows& k, const RowNorms& norms,
                              hipStream_t s);
// launch_kv_append with keys and queries normalised before they are turned.
hipError_t launch_kv_append_norm(const KvLayout& L, const NewRows& n, const RowNorms& norms, const int64_t* slots,
                                 int64_t rows, int32_t hq, void* q_out, hipStream_t s);

// The gradient's pass of launch_norm_rotary: x and dy to dx, and the weights' gradients.
struct NormBackRows {
  const void* x;
  const void* dy;
  void* dx;
  int64_t x_row, x_head, dy_row, dy_head, dx_row, dx_head;
  int32_t heads;
  float* dweight;  // [head size], or null
};
size_t norm_back_workspace(int32_t head_dim);
hipError_t launch_norm_back(const Rotary& r, int32_t dtype, const NormBackRows& q, const NormBackRows& k,
                            const RowNorms& norms, const int32_t* positions, int64_t rows, void* ws,
                            hipStream_t s);

// Block tables, slots and positions from lengths.
struct MapArgs {
  const int32_t* prior;
  const int32_t* added;
  const int32_t* held;
  int32_t* table;
  int64_t stride;
  int32_t* free_pages;
  int64_t capacity;
  const int32_t* num_free;
  const int32_t* depths;
  int64_t* slots;
  int32_t* positions;
  int32_t* starts;
  int32_t* held_out;
  int32_t* num_free_out;
  int32_t* refused;
  int32_t batch;
  int64_t rows;
};
hipError_t launch_kv_map(const MapArgs& a, hipStream_t s);

// Accepted nodes' rows to the end of their sequences.
struct AcceptArgs {
  uint16_t* k_cache;
  uint16_t* v_cache;
  int64_t num_pages;
  int32_t hkv;
  const int32_t* prior;
  const int32_t* accepted;
  const int32_t* counts;
  int32_t batch, most;
  const int32_t* table;
  int64_t stride;
};
hipError_t launch_kv_accept(const AcceptArgs& a, hipStream_t s);

// Attention of drafted nodes.
struct TreeCall {
  const void* q;
  int64_t rows;
  const int32_t* prior;
  const int32_t* starts;
  const uint32_t* mask;
  int32_t mask_words;
  const int32_t* table;
  int64_t stride;
  int32_t batch, hq;
  float scale;
  void* ws;
  void* out;
  float* lse;
};
size_t tree_workspace();
// The attention, and the merge of the parts of items that workgroups share.
hipError_t launch_tree(const KvLayout& L, const TreeCall& c, hipStream_t s);
hipError_t launch_tree_merge(const KvLayout& L, const TreeCall& c, hipStream_t s);

}  // namespace libra
