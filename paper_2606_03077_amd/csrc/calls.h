// What the entry points share: handles, checks, per-kernel timing, the table upload and the
// order of an attention call's launches (defined in api.cpp unless inline here).
#pragma once

#include <cstdint>
#include <mutex>

#include "internal.h"

struct libra_kv_layout_s : libra::KvLayout {};
struct libra_plan_s : libra::Plan {};

namespace libra {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Brackets one kernel launch with events when profiling is on.
class ProfScope {
 public:
  ProfScope(int kind, hipStream_t s, bool active);
  ~ProfScope();

 private:
  void release();
  int kind_;
  hipStream_t s_;
  hipEvent_t a_ = nullptr, b_ = nullptr;
};

// Picks the form of plan P that runs in a workspace of ws_bytes bytes and copies its tables
// there unless they are there already (or always, if forced).  The faster form is taken if
// the workspace is large enough for it; a call whose workspace holds the plain tables runs
// the plain form, so that a call on uploaded tables enqueues kernels only, whatever size
// it states: the plain tables are there with the fine tiles' as well.
libra_status upload(Plan& P, void* ws, size_t ws_bytes, hipStream_t s, bool force,
                    const Plan** form);

// The argument checks that decode and append calls share.
libra_status check_call(const KvLayout* L, const Plan* P, int mode, const void* q,
                        const int32_t* bt, int32_t bt_stride, int32_t batch, int32_t hq,
                        float scale, const void* out);

// The current device's auxiliary stream, or null if it has none (then run sequentially).
hipStream_t aux_stream();
std::mutex& fork_mutex();  // record / wait pairs of concurrent callers must not interleave

// Decode units, chunk units, then the merge of split rows.  `chunk` and `decode` enqueue the
// two launches on the stream they are given.  `timed` allows per-kernel
// timing events (which may create events while timing is enabled).  When the plan has
// both decode rows and chunk tiles, the chunk launch goes first on `s` and the decode
// launch on the device's auxiliary stream, forked from `s` after everything enqueued
// before and joined back before the merge: the dispatcher then fills the CUs that the
// matrix-core bound chunk tiles free with the HBM-bound decode rows as they come.
template <class Chunk, class Decode>
libra_status run_attention(const Plan& P, void* ws, void* out, float* lse, hipStream_t s,
                           bool timed, Chunk chunk, Decode decode) {
  hipError_t e;
  hipStream_t s2 = nullptr;
  if (P.info.n_single > 0 && P.info.n_chunk > 0 && P.fork_ev && P.join_ev) s2 = aux_stream();
  if (s2) {
    {
      std::lock_guard<std::mutex> lk(fork_mutex());
      e = hipEventRecord(P.fork_ev, s);
      if (e == hipSuccess) e = hipStreamWaitEvent(s2, P.fork_ev, 0);
    }
    if (e != hipSuccess) return hip_error(e, "forking the decode rows");
    {
      ProfScope ps(LIBRA_KERNEL_CHUNK, s, timed);
      e = chunk(s);
    }
    if (e != hipSuccess) return hip_error(e, "chunk launch");
    {
      ProfScope ps(LIBRA_KERNEL_DECODE, s2, timed);
      e = decode(s2);
    }
    if (e != hipSuccess) return hip_error(e, "decode launch");
    {
      std::lock_guard<std::mutex> lk(fork_mutex());
      e = hipEventRecord(P.join_ev, s2);
      if (e == hipSuccess) e = hipStreamWaitEvent(s, P.join_ev, 0);
    }
    if (e != hipSuccess) return hip_error(e, "joining the decode rows");
  } else {
    {
      ProfScope ps(LIBRA_KERNEL_DECODE, s, timed && P.info.n_single > 0);
      e = decode(s);
    }
    if (e != hipSuccess) return hip_error(e, "decode launch");
    {
      ProfScope ps(LIBRA_KERNEL_CHUNK, s, timed && P.info.n_chunk > 0);
      e = chunk(s);
    }
    if (e != hipSuccess) return hip_error(e, "chunk launch");
  }
  {
    ProfScope ps(LIBRA_KERNEL_MERGE, s, timed && merge_launches(P));
    e = launch_merge(P, ws, out, lse, s);
  }
  return e == hipSuccess ? LIBRA_OK : hip_error(e, "merge launch");
}

}  // namespace libra
