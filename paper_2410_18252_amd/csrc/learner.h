// What the norm with residual and dropout, the token log-probs and the pairs' loss share.  Internal to librlgen.so.
#pragma once
#include "window.h"

// ------------------------------------------------------------------ launchers
struct AddNormArgs {
  int dtype, res_dtype, y_dtype;        // of x, dy and dx; of residual, h and their gradients; of y
  int rows, width;
  unsigned drop; float keep_scale;      // an element is dropped if its 16 random bits are below `drop`
  const unsigned long long* rng;        // seed, offset
  const float* gain; float eps;         // gain null: no norm
  const void *x, *residual; long long x_stride, residual_stride;
  void *h, *y; long long h_stride, y_stride;
  float* scales; int scale_group;       // columns to a scale, 0: the whole row
  // backward (h is an input there)
  const void *dy, *dh; long long dy_stride, dh_stride;
  void *dres, *dx; long long dres_stride, dx_stride;
  float *dgain, *partial;
};
hipError_t rl_add_norm(const AddNormArgs& a, hipStream_t s);
size_t rl_add_norm_backward_bytes(int rows, int width);
hipError_t rl_add_norm_backward(const AddNormArgs& a, hipStream_t s);
constexpr int MOST_WIDTH = 16384;

struct LogprobArgs {
  int dtype, rows, vocab;
  const void* logits; long long stride;
  const int* tokens; float temperature;
  float *logprobs, *stats, *entropy;
  int n_top; int* top_tokens; float* top_logprobs;
  float4* partial; uint64_t* part_keys; // of rows that are parted: two of numbers, and n_top keys, of each part
  // backward
  const float *g, *g_entropy;
  void* dlogits; long long d_stride;
};
size_t rl_token_logprobs_bytes(const LogprobArgs& a);
hipError_t rl_token_logprobs(LogprobArgs a, void* workspace, hipStream_t s);
long long rl_token_logprobs_backward_blocks(const LogprobArgs& a);
hipError_t rl_token_logprobs_backward(const LogprobArgs& a, hipStream_t s);
constexpr int MOST_TOP = 64;

struct PairArgs {
  const float *pol, *ref; int rows;
  const int* row_starts; int B, k;
  const int *pos, *neg;
  float beta, weight;
  float *loss, *grad;
};
hipError_t rl_dpo_pairs(const PairArgs& a, hipStream_t s);

// ------------------------------------------------------------------ over a wave
// Sum and largest value of a wave's lanes, in every lane: shifts within rows of 16 lanes, then from row to row, as operands of the additions
// themselves (six shuffles through LDS take about ten times as long).  The order is fixed.  NaN passes through sums, not through maxima.
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float v, float other) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63)); }
__device__ __forceinline__ float lanes_sum(float v) {
  v += moved<0x111, 0xf>(v, 0.f);       // from the lanes 1, 2, 4 and 8 before in a row
  v += moved<0x112, 0xf>(v, 0.f);
  v += moved<0x114, 0xf>(v, 0.f);
  v += moved<0x118, 0xf>(v, 0.f);
  v += moved<0x142, 0xa>(v, 0.f);       // a row's last lane to the next row, then the second row's to the last two
  v += moved<0x143, 0xc>(v, 0.f);
  return last_lane(v);
}
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, moved<0x111, 0xf>(v, -INFINITY));
  v = fmaxf(v, moved<0x112, 0xf>(v, -INFINITY));
  v = fmaxf(v, moved<0x114, 0xf>(v, -INFINITY));
  v = fmaxf(v, moved<0x118, 0xf>(v, -INFINITY));
  v = fmaxf(v, moved<0x142, 0xa>(v, -INFINITY));
  v = fmaxf(v, moved<0x143, 0xc>(v, -INFINITY));
  return last_lane(v);
}

// ------------------------------------------------------------------ past the caches
// Data that the last-level cache (256 MB) does not hold between one call and the next is better passed by it: the hint keeps lines that come once from
// driving each other out.  Below that it costs what the cache would have given (rows of 16 MB in all: 9.4 us without, 11.4 with it).
constexpr double CACHE_BYTES = 256e6;
template <bool ONCE, class V> __device__ __forceinline__ V take(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, class V, class P> __device__ __forceinline__ void leave(P* p, V v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// ------------------------------------------------------------------ element types
struct TypeF32 {};
// Eight elements of a row in registers, 16-byte accesses
template <class T> struct Vec8 {
  u32x4 w;
  template <bool ONCE = false> static __device__ __forceinline__ Vec8 load(const void* p, long long at) {
    return {take<ONCE>((const u32x4*)((const uint16_t*)p + at))};
  }
  static __device__ __forceinline__ Vec8 zero() { return {u32x4{0, 0, 0, 0}}; }
  // what is known of the values ends here
  __device__ __forceinline__ void opaque() { asm volatile("" : "+v"(w)); }
  __device__ __forceinline__ void to(float* y) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { y[2 * e] = T::low(w[e]); y[2 * e + 1] = T::high(w[e]); }
  }
  template <bool ONCE = false> static __device__ __forceinline__ void store(void* p, long long at, const float* y) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = T::pack(y[2 * e], y[2 * e + 1]);
    leave<ONCE>((u32x4*)((uint16_t*)p + at), w);
  }
};
template <> struct Vec8<TypeF32> {
  f32x4 a, b;
  template <bool ONCE = false> static __device__ __forceinline__ Vec8 load(const void* p, long long at) {
    const float* x = (const float*)p + at;
    return {take<ONCE>((const f32x4*)x), take<ONCE>((const f32x4*)(x + 4))};
  }
  static __device__ __forceinline__ Vec8 zero() { return {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}}; }
  __device__ __forceinline__ void opaque() {}
  __device__ __forceinline__ void to(float* y) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { y[e] = a[e]; y[4 + e] = b[e]; }
  }
  template <bool ONCE = false> static __device__ __forceinline__ void store(void* p, long long at, const float* y) {
    float* x = (float*)p + at;
    leave<ONCE>((f32x4*)x, f32x4{y[0], y[1], y[2], y[3]});
    leave<ONCE>((f32x4*)(x + 4), f32x4{y[4], y[5], y[6], y[7]});
  }
};
