// What the kernels of the attention over a paged cache share.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "kv_plan.cuh"

constexpr int KV_COUNTERS = 1024;  // at the start of a workspace: parts done of a unit, by the CTA it starts in

// One more part of a unit is in the workspace, of n; true for the last, whose caller joins them and finds the count back at
// zero.  By one thread, with a barrier between the stores of the part and this, and one between this and the loads.
FL_DEV bool kv_part_done(unsigned* counter, unsigned n) {
  unsigned before;
  asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(counter), "r"(n - 1) : "memory");
  return before == n - 1;
}
// All parts but the caller's are in the workspace.  Then nobody else touches the count any more: it goes back to zero.
FL_DEV bool kv_part_is_last(unsigned* counter, unsigned n) {
  unsigned before;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(before) : "l"(counter) : "memory");
  if (before != n - 1) return false;
  *counter = 0;
  return true;
}

struct KvAttnArgs {
  KvBatchDev b;
  const void *q, *k, *v;
  void* o;
  int64_t ldq, ldo, page_stride, head_stride, token_stride;
  int group, kvh;  // query heads per key / value head, key / value heads
  float* lse;
  float scale_log2;
  unsigned* counters;
  float* parts;
};

template <class T>
struct KvIo;
template <>
struct KvIo<__nv_bfloat16> {
  static constexpr bool is_half = false;
  // larger magnitudes of two pairs; NaN stays
  FL_DEV static uint32_t max_abs(uint32_t a, uint32_t x) {
    const __nv_bfloat162 y = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&x)));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  FL_DEV static float2 unpack(uint32_t x) { return unpack_bf16x2(x); }
  FL_DEV static uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
  FL_DEV static bool finite(uint32_t x) { return (x & 0x7f80u) != 0x7f80u && (x & 0x7f800000u) != 0x7f800000u; }  // both halves
};
template <>
struct KvIo<__half> {
  static constexpr bool is_half = true;
  FL_DEV static uint32_t max_abs(uint32_t a, uint32_t x) {
    const __half2 y = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&x)));
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  FL_DEV static float2 unpack(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
  FL_DEV static uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  FL_DEV static bool finite(uint32_t x) { return (x & 0x7c00u) != 0x7c00u && (x & 0x7c000000u) != 0x7c000000u; }
};

// Chunks of new tokens (kv_attention_tc.cu); _parts: bytes of a workspace's parts that it uses.
size_t fl_kv_attention_tc_parts(int head_dim);
int fl_launch_kv_attention_tc(const fl_kv_cache* c, const KvAttnArgs& a, int heads, cudaStream_t st);
