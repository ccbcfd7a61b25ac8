// The context and small helpers of the host side, shared by the files that hold entry points.
#pragma once

#include <cstddef>
#include <cstdint>

#include "finch_internal.h"

struct finch_ctx {
  finch_config cfg;
  int device;
  size_t max_lds;   // largest dynamic LDS a workgroup may ask for
  int last_hip;     // hipError_t of the last failed HIP call
  int row_bytes;    // bytes of one K or V row
  // optional per-kernel timing (finch_profile): pairs of events around launches
  bool prof_on;
  int prof_used;
  hipEvent_t* prof_ev;   // 2 * kProfPairs events, or nullptr
  int* prof_kind;        // kernel class of each pair
  int n_cu;              // compute units of the device
  int step_path;         // FINCH_PATH_AUTO / _SEPARATE / _OWNER
  int slice_keys;        // target keys per workgroup slice of the bf16 scoring kernels
  finch_reposition repos;  // {OFF, ASCENDING}: plain copies
  int layer_group;         // > 1: runs of that many problems share one selection
  int64_t layer_wait_ticks;  // bound of a workgroup's wait for its layer, 100 MHz ticks
  int32_t* meet;             // meeting words of this context's launches with several workgroups per problem
  void* static_scratch;    // this device's copy of the file-scope scratch array (finch_step_static)
  int32_t* static_meet;    // and of the meeting words that go with it
  // finch_loop: fingerprint of the last descriptor set whose slots were found free of
  // overlaps (the check is repeated only when the descriptors change)
  uint64_t loop_checked_hash;
  bool loop_checked;
  bool loop_rows_may_stay;  // what check_slot_overlaps said of that set
  int32_t* loop_ways;       // LaunchParams::ways of its whole loops
  int32_t* attend_meet;     // counters of finch_attend's launches (attend_common.h)
  int scale_block;          // rows per power of two of an 8-bit cache
};

namespace finch {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + nb && b0 < a0 + na;
}

// Whether what is launched on `s` now is recorded into a graph (or cannot be told).
inline bool being_captured(hipStream_t s) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &status) != hipSuccess) {
    (void)hipGetLastError();
    return true;
  }
  return status != hipStreamCaptureStatusNone;
}

inline finch_status hip_fail(finch_ctx* ctx, hipError_t e) {
  ctx->last_hip = static_cast<int>(e);
  return FINCH_ERR_HIP;
}

}  // namespace finch
