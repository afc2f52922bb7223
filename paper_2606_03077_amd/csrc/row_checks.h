// The rotary handle, and the argument checks of calls that take rows of heads.
#pragma once

#include <cstdint>
#include <string>

#include "calls.h"
#include "rotary.h"

struct libra_rotary_s : libra::Rotary {};

namespace libra {

constexpr int64_t kMaxOffset = int64_t(1) << 56;  // elements

inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Whether rows x heads vectors of n elements at these strides never overlap.
inline bool disjoint(int64_t rows, int64_t heads, int64_t n, int64_t row, int64_t head) {
  if (rows > 1 && row < n) return false;
  if (heads > 1 && head < n) return false;
  if (rows == 1 || heads == 1) return true;
  if (row >= (heads - 1) * head + n || head >= (rows - 1) * row + n) return true;
  // Vectors (r, h + j) and (r + i, h) lie j head - i row apart; the nearest to j head are two.
  for (int64_t j = 1; j < heads; ++j) {
    const int64_t i = j * head / row;
    if (i >= 1 && i < rows && j * head - i * row < n) return false;
    if (i + 1 < rows && (i + 1) * row - j * head < n) return false;
  }
  return true;
}

// Whether an element's offset stays well inside 64 bits of bytes.
inline bool addressable(int64_t rows, int64_t heads, int64_t row, int64_t head) {
  return __int128(rows) * row + __int128(heads) * head <= kMaxOffset;
}

// A projection's rows: 16-byte aligned, heads 128 elements apart, rows row elements apart.
inline libra_status check_rows(const void* p, int64_t rows, int64_t row, int64_t heads, const char* what) {
  if (!p) return set_error(LIBRA_E_INVAL, std::string(what) + " is NULL");
  if (!aligned16(p) || row % 8)
    return set_error(LIBRA_E_INVAL, std::string(what) + " must be 16-byte aligned, its row stride a multiple of 8");
  if (row < heads * kDim || !addressable(rows, heads, row, kDim))
    return set_error(LIBRA_E_INVAL, std::string(what) + "'s row stride is smaller than its heads, or far too large");
  return LIBRA_OK;
}

inline libra_status check_cached(const KvLayout& L, const Rotary* r, int32_t num_kv_heads) {
  if (r && r->head_dim != L.desc.head_dim)
    return set_error(LIBRA_E_INVAL, "rotary and layout disagree on head_dim");
  if (num_kv_heads != L.desc.num_kv_heads)
    return set_error(LIBRA_E_INVAL, "num_kv_heads differs from the layout's");
  return LIBRA_OK;
}

}  // namespace libra
