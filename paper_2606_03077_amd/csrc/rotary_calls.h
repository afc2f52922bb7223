// Launchers of the rotary operators (rotary.hip, decode.hip, chunk.hip).
#pragma once

#include "internal.h"
#include "rotary.h"

namespace libra {

// What libra_rotary_apply turns: rows x heads, element strides.
struct RotaryRows {
  const void* x;
  void* out;
  int64_t x_row, x_head, out_row, out_head;
  const int32_t* positions;
  int64_t rows;
  int32_t heads;
  int32_t dtype;
  bool backward;
};
hipError_t launch_rotary(const Rotary& r, const RotaryRows& a, hipStream_t s);

// New rows for the cache, and the rotation on the way (none if rotary is null).
struct NewRows {
  const Rotary* rotary;
  const int32_t* positions;  // null: the index in the cache (append plans)
  const void* q;
  const void* k;
  const void* v;
  int64_t q_row, k_row, v_row;  // row strides in elements; heads are 128 apart
  bool round_queries = false;   // attention: to bf16, instead of two bf16 parts
};
// Rows to slots[row]; q (if given) turned to q_out.
hipError_t launch_kv_append(const KvLayout& L, const NewRows& n, const int64_t* slots,
                            int64_t rows, int32_t hq, void* q_out, hipStream_t s);
// Rows to the (sequence, page) tiles of an append plan.
hipError_t launch_cache_write_rotary(const KvLayout& L, const Plan& P, const void* ws,
                                     const NewRows& n, const int32_t* bt, int32_t stride,
                                     hipStream_t s);
// Attention whose queries are turned as they are loaded.  write: the decode units also write
// the new tokens to the cache (plans of single rows only: chunk tiles read what others write).
hipError_t launch_decode_rotary(const KvLayout& L, const Plan& P, void* ws, const NewRows& n,
                                const int32_t* bt, int32_t stride, float scale, void* out,
                                float* lse, bool write, hipStream_t s);
hipError_t launch_chunk_rotary(const KvLayout& L, const Plan& P, void* ws, const NewRows& n,
                               const int32_t* bt, int32_t stride, float scale, void* out,
                               float* lse, hipStream_t s);

}  // namespace libra
