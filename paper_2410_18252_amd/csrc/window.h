// What the paged cache's plan, the per-head norm with rotation and the windowed attention share.  Internal to librlgen.so.
#pragma once
#include "common.h"

// ------------------------------------------------------------------ launchers
struct PlanArgs {
  const int *ctx_lens, *new_lens;
  int S, page_shift;
  const int* free_pages; int n_free;
  const int* free_head;                 // nullable: pages taken before this call
  int* page_table; int table_stride;
  int max_rows;
  int *total_lens, *row_starts, *slots, *positions, *counts;
  int group, chunks;                    // requests to a block, blocks to the rows of a group
};
hipError_t rl_plan_pages(PlanArgs a, hipStream_t s);

struct NormRopeArgs {
  const void* qkv; long long qkv_stride; int src_dtype, dtype;
  const float *q_gain, *k_gain; float eps;
  const float2* rope; int max_pos, r;   // [max_pos, r / 2] cos, sin
  const int* positions;
  int rows, Hq, Hkv, h;
  // forward: q [rows, Hq, h]; k and v either as rows or into the cache's pages
  void *q, *k, *v; long long q_stride, k_stride, v_stride;
  void* pages; int n_pages, page_shift; const int* slots;
  // backward
  const void *dq, *dk, *dv; long long dq_stride, dk_stride, dv_stride;
  void* dqkv; long long dqkv_stride;
  float *dq_gain, *dk_gain, *partial;
};
hipError_t rl_norm_rope(const NormRopeArgs& a, hipStream_t s);
size_t rl_norm_rope_backward_bytes(int rows, int h);
hipError_t rl_norm_rope_backward(const NormRopeArgs& a, hipStream_t s);

struct WindowArgs {
  int dtype, Hq, Hkv, h, S, rows;
  int window, sinks; float scale;       // window 0: every earlier key is visible
  const int* row_starts;
  int max_new;                          // most rows of a sequence
  const void *q, *k, *v; long long q_stride, k_stride, v_stride;
  void* out; long long out_stride; float* lse;
  // keys and values from the cache instead of k and v
  const void* pages; int n_pages, page_shift; const int* page_table; int table_stride; const int* total_lens; int max_total;
  // backward
  const void *o, *dout; long long o_stride, dout_stride;
  void *dq, *dk, *dv; long long dq_stride, dk_stride, dv_stride;
  void* ws; size_t ws_bytes;
};
// What a launch of each would have in blocks of 256 threads, which have to stay below MOST_BLOCKS (a launch has fewer than 2^32 threads)
constexpr long long MOST_BLOCKS = 1 << 24;
long long rl_window_rows_blocks(const WindowArgs& a);
long long rl_window_decode_blocks(const WindowArgs& a);
long long rl_window_backward_blocks(const WindowArgs& a);
hipError_t rl_window_rows(const WindowArgs& a, hipStream_t s);
size_t rl_window_rows_bytes(const WindowArgs& a);
size_t rl_window_decode_bytes(const WindowArgs& a);
hipError_t rl_window_decode(const WindowArgs& a, hipStream_t s);
size_t rl_window_backward_bytes(const WindowArgs& a);
hipError_t rl_window_backward(const WindowArgs& a, hipStream_t s);

// ------------------------------------------------------------------ element types
struct TypeBf16 {
  typedef bf16x8 vec8;
  static __device__ __forceinline__ f32x16 mfma32(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x4 mfma16(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
  static __device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
};
struct TypeF16 {
  typedef f16x8 vec8;
  static __device__ __forceinline__ f32x16 mfma32(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x4 mfma16(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  // nearest even; beyond the largest finite value infinity, as a cast gives it
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (f16_t)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (f16_t)hi) << 16);
  }
  static __device__ __forceinline__ float low(uint32_t w) { return f16_bits_to_f32((uint16_t)w); }
  static __device__ __forceinline__ float high(uint32_t w) { return f16_bits_to_f32((uint16_t)(w >> 16)); }
};
