// Block tables, slots and positions from request lengths that live on the GPU, and the move of
// accepted tokens.  Both are integer or copy work of microseconds, bound by launches and by chains
// of dependent loads.
//
// The table's kernel is one workgroup: requests 1,024 at a time, one to a thread, whose page counts
// are added up by scans, and then the pages that move, each found by a search in the scans' sums, so
// that an ended request of thousands of pages is everybody's work.  Pages given back are pushed
// before any is taken.  64 requests of a token each: 7 us of kernel with cold caches; 256 trees of
// which 9 ended: 14 us, and 5 for their 8,025 rows, which a launch of their own maps.  2,500 requests,
// taken in turns of 1,024: 30 us a pass of a token each, 80 of trees (45,617 pages move, 77,922 rows).
// Accepted tokens: 2,157 of 8 heads, of which 2,029 move (16.6 MB), 12 us, 22 with cold caches, bound
// by the V tiles' lines, as a value of a token is two bytes of every 16.
#include <algorithm>
#include <climits>

#include "drafts.h"
#include "row_types.h"

namespace libra {
namespace {

constexpr int kMapThreads = 1024;  // of the form that takes requests in turns

// Int: 32 bits where the call's sizes cannot exceed them, which takes half the scans' time.
template <class Int>
struct Sums {
  Int back, need, rows;
};
template <class Int>
__device__ __forceinline__ Sums<Int> operator+(const Sums<Int>& a, const Sums<Int>& b) {
  return {a.back + b.back, a.need + b.need, a.rows + b.rows};
}

// Inclusive sums over the workgroup's threads, and their total.
template <int kThreads, class Int>
__device__ __forceinline__ Sums<Int> block_scan(Sums<Int> x, Sums<Int>* wave_sums, Sums<Int>& total) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int n = 1; n < 64; n <<= 1) {
    const Sums<Int> y{__shfl_up(x.back, n), __shfl_up(x.need, n), __shfl_up(x.rows, n)};
    if (lane >= n) x = x + y;
  }
  __syncthreads();  // the sums of an earlier scan have been read
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  Sums<Int> before{};
  total = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before = before + wave_sums[w];
    total = total + wave_sums[w];
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
  // Rows past the call's do not count, so that their sum stays in bounds.
  template <class Int>
  __device__ __forceinline__ Sums<Int> sums(int64_t rows) const {
    return {valid ? Int(max(held - want, int64_t(0))) : 0, valid ? Int(max(want - held, int64_t(0))) : 0,
            Int(min(max(added, int64_t(0)), rows + 1))};
  }
};
__device__ __forceinline__ Request load_request(const MapArgs& A, int b) {
  Request r{};
  if (b >= A.batch) return r;
  r.prior = A.prior[b], r.added = A.added[b], r.held = A.held[b];
  r.want = (r.prior + r.added + kPage - 1) / kPage;
  r.valid = r.prior >= 0 && r.added >= 0 && r.held >= 0 && r.held <= A.stride && r.want <= A.stride;
  return r;
}

// Row r of request b, whose first row is `start`.
__device__ __forceinline__ void map_row(const MapArgs& A, int64_t r, int b, int64_t start, int64_t prior,
                                        bool refused) {
  const int64_t at = prior + r - start;
  A.slots[r] = refused ? -1 : int64_t(A.table[b * A.stride + at / kPage]) * kPage + at % kPage;
  A.positions[r] = int32_t(A.depths ? prior + A.depths[r] : at);
}
__device__ __forceinline__ void pad_row(const MapArgs& A, int64_t r) { A.slots[r] = -1, A.positions[r] = 0; }

// kTurns: more requests than threads, which are taken in turns and read again in the second pass.
// Otherwise a request stays in its thread's registers, and what the rows need of it in LDS.
// rows: how many of the rows this launch maps too (all or none).
template <int kThreads, bool kTurns, class Int>
__global__ __launch_bounds__(kThreads) void kv_map_kernel(MapArgs A, int64_t rows) {
  __shared__ Sums<Int> wave_sums[kThreads / 64];
  __shared__ Int upto[kThreads];  // of pages
  __shared__ int32_t start[kThreads], prior[kThreads], held[kThreads], want[kThreads];
  __shared__ uint8_t refusal[kThreads];
  __shared__ unsigned long long given_upto;
  const int t = threadIdx.x;
  const int64_t have = min(max(int64_t(*A.num_free), int64_t(0)), A.capacity);
  int64_t top = have;
  Request q;
  Sums<Int> sums, total;
  if (t == 0) given_upto = 0;
  // Pages given back.
  for (int b0 = 0; b0 < A.batch; b0 += kThreads) {
    q = load_request(A, b0 + t);
    sums = block_scan<kThreads>(q.sums<Int>(A.rows), wave_sums, total);
    if (total.back > 0) {  // uniform
      upto[t] = sums.back, held[t] = int32_t(q.held);
      __syncthreads();
#pragma unroll 4
      for (Int i = t; i < total.back; i += kThreads) {
        const int n = find(upto, min(kThreads, A.batch - b0), i);
        // The request's last surplus page is its last held one.
        if (top + i < A.capacity)
          A.free_pages[top + i] = A.table[(b0 + n) * A.stride + held[n] - (upto[n] - i)];
      }
      top = min(top + total.back, A.capacity);
    }
  }
  __syncthreads();  // the pages given back can be read
  Int asked = 0;
  int64_t row0 = 0;
  for (int b0 = 0; b0 < A.batch; b0 += kThreads) {
    const int b = b0 + t;
    if (kTurns) {
      q = load_request(A, b);
      sums = block_scan<kThreads>(q.sums<Int>(A.rows), wave_sums, total);
    }
    const Sums<Int> own = q.sums<Int>(A.rows);
    const Int need = own.need, asked_upto = asked + sums.need;
    const int64_t row1 = row0 + sums.rows;
    // Once a request is refused for want of pages, so is every later one that needs any: those that
    // get theirs take the first of the pages asked for.
    const bool refused = !q.valid || (need > 0 && asked_upto > top);
    upto[t] = asked_upto, refusal[t] = refused, want[t] = int32_t(q.valid ? q.want : 0);
    start[t] = int32_t(min(row1 - own.rows, A.rows)), prior[t] = int32_t(q.prior);
    if (!refused && need > 0) atomicMax(&given_upto, (unsigned long long)asked_upto);
    if (b < A.batch) {
      A.starts[b + 1] = int32_t(min(row1, A.rows));
      A.held_out[b] = int32_t(refused ? q.held : q.want);
      A.refused[b] = refused;
    }
    __syncthreads();
#pragma unroll 4
    for (Int i = t; i < total.need; i += kThreads) {
      const int n = find(upto, min(kThreads, A.batch - b0), Int(asked + i));
      if (refusal[n]) continue;
      A.table[(b0 + n) * A.stride + want[n] - (upto[n] - asked - i)] = A.free_pages[top - 1 - asked - i];
    }
    asked += total.need, row0 += total.rows;
    __syncthreads();
  }
  if (t == 0) *A.num_free_out = int32_t(top - int64_t(given_upto));
  if (t == 0) A.starts[0] = 0;
  __syncthreads();
  row0 = min(row0, A.rows);
#pragma unroll 4
  for (int64_t r = t; r < rows; r += kThreads) {
    if (r >= row0) {
      pad_row(A, r);
    } else if (kTurns) {
      const int b = find(A.starts + 1, A.batch, int32_t(r));
      map_row(A, r, b, A.starts[b], A.prior[b], A.refused[b]);
    } else {
      // The last request that starts at or before the row (threads past the batch start after it).
      int lo = 0, hi = A.batch - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start[mid] <= r) lo = mid;
        else hi = mid - 1;
      }
      map_row(A, r, lo, start[lo], prior[lo], refusal[lo]);
    }
  }
}

constexpr int kRowThreads = 256;
constexpr int kRowStarts = 2048;  // requests whose starts a workgroup searches in LDS
__global__ __launch_bounds__(kRowThreads) void kv_map_rows_kernel(MapArgs A) {
  __shared__ int32_t ends[kRowStarts];
  const bool staged = A.batch <= kRowStarts;
  if (staged) {
    for (int b = threadIdx.x; b < A.batch; b += kRowThreads) ends[b] = A.starts[b + 1];
    __syncthreads();
  }
  const int64_t r = int64_t(blockIdx.x) * kRowThreads + threadIdx.x;
  if (r >= A.rows) return;
  if (A.batch == 0 || r >= (staged ? ends[A.batch - 1] : A.starts[A.batch])) return pad_row(A, r);
  const int b = staged ? find(ends, A.batch, int32_t(r)) : find(A.starts + 1, A.batch, int32_t(r));
  map_row(A, r, b, A.starts[b], A.prior[b], A.refused[b]);
}

// One workgroup per (sequence, KV head): accepted tokens 16 at a time, 16 threads to a token.  Nodes
// come in ascending order, so a token's new place is behind none that is still to be read; within
// the 16 all are read before one is written.  A thread moves a key's granule, and eight values 16
// channels apart, so that neighbouring threads touch neighbouring granules of the V tile.
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
      for (int e = 0; e < 8; ++e) v[e] = A.v_cache[from + v_off(sl, j + 16 * e)];
    }
    __syncthreads();
    if (moves) {
      const int sl = int((prior + i) % kPage);
      *reinterpret_cast<uint4*>(A.k_cache + to + k_off(sl, 8 * j)) = k;
#pragma unroll
      for (int e = 0; e < 8; ++e) A.v_cache[to + v_off(sl, j + 16 * e)] = v[e];
    }
    __syncthreads();
  }
}

// Rows that the one workgroup maps itself, instead of a second launch: 64 requests of a token 10.1
// against 12.1 us (with cold caches, and some 4 of two events), trees of 16 requests (620 rows) 10.8
// against 13.5, of 32 (900) 12.6 against 15.4, of 64 (2,494) 17.7 against 16.7, of 256 (8,025) 31.1
// against 21.3.
constexpr int64_t kOneLaunchRows = 1024;

}  // namespace

hipError_t launch_kv_map(const MapArgs& a, hipStream_t s) {
  const bool one = a.rows <= kOneLaunchRows;
  auto launch = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(1), dim3(unsigned(threads)), 0, s, a, one ? a.rows : 0);
    return hipGetLastError();
  };
  // Few rows a request, so that few pages move: 512 threads, whose scans are shorter.  With 512 and
  // 1,024 threads (cold caches, and some 4 us of two events): 64 requests of a token each 10.2 and 11.2
  // us, 512 12.2 and 12.7; trees of up to 64 nodes, 16 requests 11.1 and 10.6, 32 13.5 and 12.6, 64 16.5
  // and 17.1, 256 23.9 and 21.1.
  // Sums, and a thread's next index behind the last, fit 32 bits.
  const bool small = std::max(a.stride, a.rows + 1) * int64_t(std::max(a.batch, 1)) <= INT32_MAX - 4 * kMapThreads;
  const hipError_t e =
      a.batch > kMapThreads ? launch(kv_map_kernel<kMapThreads, true, int64_t>, kMapThreads)
      : !small              ? launch(kv_map_kernel<kMapThreads, false, int64_t>, kMapThreads)
      : a.batch <= 512 && a.rows <= 8 * int64_t(a.batch) ? launch(kv_map_kernel<512, false, int32_t>, 512)
                            : launch(kv_map_kernel<kMapThreads, false, int32_t>, kMapThreads);
  if (e != hipSuccess || one) return e;
  hipLaunchKernelGGL(kv_map_rows_kernel, dim3(unsigned((a.rows + kRowThreads - 1) / kRowThreads)), dim3(kRowThreads),
                     0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_accept(const AcceptArgs& a, hipStream_t s) {
  // A launch's threads are counted in 32 bits, and one of more runs a part of them without an error.
  constexpr int64_t kMaxBlocks = int64_t(1) << 22;
  const int64_t step = kMaxBlocks / a.hkv;
  for (int64_t b0 = 0; b0 < a.batch; b0 += step) {
    AcceptArgs part = a;
    part.batch = int32_t(std::min(step, a.batch - b0));
    part.prior += b0;
    part.accepted += b0 * a.most;
    part.counts += b0;
    part.table += b0 * a.stride;
    hipLaunchKernelGGL(kv_accept_kernel, dim3(unsigned(part.batch) * unsigned(a.hkv)), dim3(256), 0, s, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace libra
