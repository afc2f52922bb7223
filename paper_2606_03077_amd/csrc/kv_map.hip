// Block tables, slots and positions from request lengths that live on the GPU, and the move of
// accepted tokens.  Both are integer or copy work of microseconds, bound by launches and by chains
// of dependent loads.
//
// The table's kernel is one workgroup: requests 1,024 at a time, one to a thread, whose page counts
// are added up by scans, and then the pages that move, each found by a search in the scans' sums, so
// that an ended request of thousands of pages is everybody's work.  Pages given back are pushed
// before any is taken.
#include <algorithm>

#include "drafts.h"
#include "row_types.h"

namespace libra {
namespace {

constexpr int kMapThreads = 1024;
constexpr int kMapWaves = kMapThreads / 64;

// Inclusive sums over the workgroup's threads, and their total.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* wave_sums, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int n = 1; n < 64; n <<= 1) {
    const int64_t y = __shfl_up(x, n);
    if (lane >= n) x += y;
  }
  __syncthreads();  // the sums of an earlier scan have been read
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  int64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kMapWaves; ++w) {
    if (w < wave) before += wave_sums[w];
    total += wave_sums[w];
  }
  return x + before;
}

// The first index with sums[i] > x among n ascending sums, the last of which is.
template <class Int>
__device__ __forceinline__ int find(const Int* sums, int n, Int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

struct Request {
  int64_t prior, added, held, want;
  bool valid;
};
__device__ __forceinline__ Request load_request(const MapArgs& A, int b) {
  Request r{};
  if (b >= A.batch) return r;
  r.prior = A.prior[b], r.added = A.added[b], r.held = A.held[b];
  r.want = (r.prior + r.added + kPage - 1) / kPage;
  r.valid = r.prior >= 0 && r.added >= 0 && r.held >= 0 && r.held <= A.stride && r.want <= A.stride;
  return r;
}

// Slot and position of row r, request b's.
__device__ __forceinline__ void map_row(const MapArgs& A, int64_t r, int b, int64_t total) {
  int64_t slot = -1;
  int32_t position = 0;
  if (r < total) {
    const int64_t prior = A.prior[b], at = prior + r - A.starts[b];
    if (!A.refused[b]) slot = int64_t(A.table[b * A.stride + at / kPage]) * kPage + at % kPage;
    position = int32_t(A.depths ? prior + A.depths[r] : at);
  }
  A.slots[r] = slot;
  A.positions[r] = position;
}

// rows: how many of the rows this launch maps too (all or none).
__global__ __launch_bounds__(kMapThreads) void kv_map_kernel(MapArgs A, int64_t rows) {
  __shared__ int64_t wave_sums[kMapWaves];
  __shared__ int64_t sums[kMapThreads];
  const int t = threadIdx.x;
  const int64_t have = min(max(int64_t(*A.num_free), int64_t(0)), A.capacity);
  int64_t top = have, total;
  // Pages given back.
  for (int b0 = 0; b0 < A.batch; b0 += kMapThreads) {
    const Request q = load_request(A, b0 + t);
    const int64_t upto = block_scan(q.valid ? max(q.held - q.want, int64_t(0)) : 0, wave_sums, total);
    if (total == 0) continue;  // uniform
    sums[t] = upto;
    __syncthreads();
    for (int64_t i = t; i < total; i += kMapThreads) {
      const int n = find(sums, kMapThreads, i);
      // The request's last surplus page is its last held one.
      const int64_t column = A.held[b0 + n] - (sums[n] - i);
      if (top + i < A.capacity) A.free_pages[top + i] = A.table[(b0 + n) * A.stride + column];
    }
    top = min(top + total, A.capacity);
  }
  __syncthreads();  // the pages given back can be read
  int64_t asked = 0, given = 0, row0 = 0;
  for (int b0 = 0; b0 < A.batch; b0 += kMapThreads) {
    const int b = b0 + t;
    const Request q = load_request(A, b);
    const int64_t need = q.valid ? max(q.want - q.held, int64_t(0)) : 0;
    const int64_t upto = asked + block_scan(need, wave_sums, total);
    const int64_t wanted = total;
    int64_t n_rows;
    const int64_t row1 = row0 + block_scan(max(q.added, int64_t(0)), wave_sums, n_rows);
    // Once a request is refused for want of pages, so is every later one that needs any: those that
    // get theirs take the first of the pages asked for.
    const bool refused = !q.valid || (need > 0 && upto > top);
    sums[t] = upto;
    int64_t granted;
    block_scan(refused ? 0 : need, wave_sums, granted);
    if (b < A.batch) {
      A.starts[b + 1] = int32_t(min(row1, A.rows));
      A.held_out[b] = int32_t(refused ? q.held : q.want);
      A.refused[b] = refused;
    }
    __syncthreads();  // sums, refused and starts of this turn
    for (int64_t i = t; i < wanted; i += kMapThreads) {
      const int n = find(sums, kMapThreads, asked + i);
      if (A.refused[b0 + n]) continue;
      const int64_t want = (int64_t(A.prior[b0 + n]) + A.added[b0 + n] + kPage - 1) / kPage;
      A.table[(b0 + n) * A.stride + want - (sums[n] - asked - i)] = A.free_pages[top - 1 - asked - i];
    }
    asked += wanted, given += granted, row0 += n_rows;
    __syncthreads();
  }
  if (t == 0) *A.num_free_out = int32_t(top - given);
  if (t == 0) A.starts[0] = 0;
  __syncthreads();
  row0 = min(row0, A.rows);
  for (int64_t r = t; r < rows; r += kMapThreads)
    map_row(A, r, r < row0 ? find(A.starts + 1, A.batch, int32_t(r)) : 0, row0);
}

constexpr int kRowThreads = 256;
__global__ __launch_bounds__(kRowThreads) void kv_map_rows_kernel(MapArgs A) {
  const int64_t r = int64_t(blockIdx.x) * kRowThreads + threadIdx.x;
  if (r >= A.rows) return;
  const int64_t total = A.starts[A.batch];
  map_row(A, r, r < total ? find(A.starts + 1, A.batch, int32_t(r)) : 0, total);
}

// One workgroup per (sequence, KV head): accepted tokens 16 at a time, 16 threads to a token.  Nodes
// come in ascending order, so a token's new place is behind none that is still to be read; within
// the 16 all are read before one is written.
__global__ __launch_bounds__(256) void kv_accept_kernel(AcceptArgs A) {
  const int b = int(blockIdx.x) / A.hkv, g = int(blockIdx.x) - b * A.hkv;
  const int s = threadIdx.x >> 4, j = threadIdx.x & 15;
  const int64_t prior = A.prior[b];
  const int count = min(A.counts[b], A.most);
  // The tile of a token, or -1 where the table or the cache ends before it.
  auto tile_of = [&](int64_t token) -> int64_t {
    if (token < 0 || token >= A.stride * kPage) return -1;
    const int64_t page = A.table[b * A.stride + token / kPage];
    return uint64_t(page) < uint64_t(A.num_pages) ? (page * A.hkv + g) * kTileElems : -1;
  };
  for (int i0 = 0; i0 < count; i0 += 16) {
    const int i = i0 + s;
    int64_t from = -1, to = -1;
    int node = 0;
    if (i < count) {
      node = A.accepted[int64_t(b) * A.most + i];
      if (node > i && prior >= 0) from = tile_of(prior + node), to = tile_of(prior + i);
    }
    const bool moves = from >= 0 && to >= 0;
    uint4 k;
    uint16_t v[8];
    if (moves) {
      const int sl = int((prior + node) % kPage);
      k = *reinterpret_cast<const uint4*>(A.k_cache + from + k_off(sl, 8 * j));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = A.v_cache[from + v_off(sl, 8 * j + e)];
    }
    __syncthreads();
    if (moves) {
      const int sl = int((prior + i) % kPage);
      *reinterpret_cast<uint4*>(A.k_cache + to + k_off(sl, 8 * j)) = k;
#pragma unroll
      for (int e = 0; e < 8; ++e) A.v_cache[to + v_off(sl, 8 * j + e)] = v[e];
    }
    __syncthreads();
  }
}

// Rows that the one workgroup maps itself, instead of a second launch.
constexpr int64_t kOneLaunchRows = 4096;

}  // namespace

hipError_t launch_kv_map(const MapArgs& a, hipStream_t s) {
  const bool one = a.rows <= kOneLaunchRows;
  hipLaunchKernelGGL(kv_map_kernel, dim3(1), dim3(kMapThreads), 0, s, a, one ? a.rows : 0);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  hipLaunchKernelGGL(kv_map_rows_kernel, dim3(unsigned((a.rows + kRowThreads - 1) / kRowThreads)), dim3(kRowThreads),
                     0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_accept(const AcceptArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(kv_accept_kernel, dim3(unsigned(a.batch) * unsigned(a.hkv)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace libra
