// Internal interface between the host part of the paged cache (kv_host.hip)
// and its kernels.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "wf_kv.h"

namespace wfkv {

// Geometry as the kernels take it.
struct Geo {
  int hq, hk, d;        // heads, channels
  int group;            // query heads per kv head
  int b, b_log2;        // tokens per block
  int n_blocks, width;  // blocks of the cache, of a row
  int cell;             // bytes of a cell
};

struct StepArgs {
  const int32_t* fresh;
  int n_rows, n_tokens;
  const int32_t* len_in;
  int32_t* len_out;
  const int32_t* pool_in;
  int32_t* pool_out;
  int32_t* ring;
  int32_t* table;
  int32_t* q_off;
  int64_t* slot;
  int32_t* pos;
  uint8_t* granted;
};

struct StoreArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  int n_tokens;
  wf_kv_norm_rope how;
  const int32_t* pos;
  const int64_t* slot;
  void* q_out;
  uint8_t* cache;
};

struct LoadArgs {
  const uint8_t* cache;
  const int64_t* slot;
  int n_tokens;
  void *k, *v;
};

struct AttendArgs {
  const void* q;
  int64_t q_stride;
  int n_tokens;
  const uint8_t* cache;
  const int32_t *table, *kv_len, *q_off, *pos;
  int n_rows;
  float scale;
  int window, max_q, max_kv;
  void* out;
};

// The work area of launch_attend: partial sums, the number of shares that wrote
// those of each query's head, and counts of shares done, 0 between launches.  A context has one for each of
// the first kAreas streams that attend; without one (all sizes 0) no tokens are shared out.
constexpr size_t kPartBytes = size_t(32) << 20, kCountBytes = size_t(1) << 20;
constexpr size_t kAreaBytes = kPartBytes + 2 * kCountBytes;
constexpr int kAreas = WF_KV_ATTEND_STREAMS;
struct AttendWork {
  int n_cu;
  float* part;
  size_t part_bytes;
  int32_t *used, *arrived;
  size_t count_bytes;  // of each
};

hipError_t launch_step(const Geo& g, const StepArgs& a, hipStream_t s);
hipError_t launch_store(const Geo& g, int dtype, const StoreArgs& a, hipStream_t s);
hipError_t launch_load(const Geo& g, int dtype, const LoadArgs& a, hipStream_t s);
hipError_t launch_attend(const Geo& g, int dtype, const AttendArgs& a, const AttendWork& w, hipStream_t s);

// A 16-bit type of the queries and values: to and from fp32 (nearest even).
struct Bf16 {
  static constexpr float kMost = 3.38953138925e38f;
  static __device__ __forceinline__ float to(uint32_t u) { return __uint_as_float(u << 16); }
  static __device__ __forceinline__ uint32_t from(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
  }
};
struct F16 {
  static constexpr float kMost = 65504.0f;
  static __device__ __forceinline__ float to(uint32_t u) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)u);
  }
  static __device__ __forceinline__ uint32_t from(float x) {
    return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
};

}  // namespace wfkv
