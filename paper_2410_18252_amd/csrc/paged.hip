// The paged cache's bookkeeping, and the per-head norms with rotation that write into it.
//
// A cache is pages [n_pages, 2, Hkv, page_size, h]: a page holds page_size keys of every kv head and then the values of the same
// tokens, a head's rows one behind the other, so that a token's key is one run of 2 h bytes wherever its page lies.
#include "../../include/rlgen.h"
#include "window.h"

namespace {

constexpr int TPB = 256;

// The plan's counts are of lengths that only the device knows: sums of numbers that are not negative, which stay at the largest int instead of
// passing it.
constexpr int MOST = 0x7fffffff;
__device__ __forceinline__ int add_counts(int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)MOST); }
__device__ __forceinline__ int block_sum(int v, int* red) {          // of a block of 256 threads; red: 4 ints
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = add_counts(v, __shfl_xor(v, o, WAVE));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return add_counts(add_counts(red[0], red[1]), add_counts(red[2], red[3]));
}
__device__ __forceinline__ int block_max(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, WAVE));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}
__device__ __forceinline__ int block_exclusive(int v, int* red) {    // exclusive prefix sum over the block's threads
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, WAVE);
    if ((threadIdx.x & 63) >= (unsigned)o) x = add_counts(x, y);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = x;
  __syncthreads();
  const int up = __shfl_up(x, 1, WAVE);
  int before = (threadIdx.x & 63) ? up : 0;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before = add_counts(before, red[w]);
  return before;
}

constexpr int PLAN_GROUP = 4 * TPB;          // most requests to a block

// How far a request's lengths go.  A negative length counts as zero, a length after the pass that an int does not hold is cut.
struct Lens { int ctx, add, had, need; bool odd; };
__device__ __forceinline__ Lens plan_lens(const PlanArgs& a, int s) {
  Lens l;
  const int ctx = a.ctx_lens[s], add = a.new_lens[s];
  l.ctx = max(ctx, 0);
  l.add = min(max(add, 0), MOST - l.ctx);
  l.odd = (ctx < 0) | (add < 0) | (add > l.add);
  const int round = (1 << a.page_shift) - 1;
  l.had = (int)(((unsigned)l.ctx + round) >> a.page_shift);
  l.need = (int)(((unsigned)l.ctx + (unsigned)l.add + round) >> a.page_shift);
  return l;
}

// A pass's plan in one launch without scratch memory: a block owns the `group` requests from blockIdx.x * group on and adds up the
// lengths of all requests before them itself (8 bytes a request out of L2: 1000 requests are four loads a thread), then scans its own in
// LDS and writes their rows and pages.  Where a group has many rows, blockIdx.y parts them.  Bound by a launch and three or four
// dependent memory latencies, not by its bytes (1000 requests of a token each: 5.6 us).
__global__ __launch_bounds__(TPB) void plan_pages_kernel(PlanArgs a) {
  __shared__ int red[4];
  __shared__ int row_end[PLAN_GROUP], page_end[PLAN_GROUP], lens_ctx[PLAN_GROUP], lens_had[PLAN_GROUP];
  const int s0 = blockIdx.x * a.group, n = min(a.group, a.S - s0);
  const bool last = s0 + n == a.S, writer = blockIdx.y == 0;
  const int asked = a.free_head ? max(*a.free_head, 0) : 0, head = min(asked, a.n_free);      // (beyond the list there is no page)
  int rows = 0, pages = 0, longest = 0, faults = 0;
  for (int s = threadIdx.x; s < s0; s += TPB) {
    const Lens l = plan_lens(a, s);
    rows = add_counts(rows, l.add);
    pages = add_counts(pages, l.need - l.had);
    if (last) {
      longest = max(longest, l.ctx + l.add);
      if (l.need > a.table_stride) faults |= RLGEN_PLAN_TABLE;
      if (l.odd) faults |= RLGEN_PLAN_LENGTH;
    }
  }
  const int rows0 = block_sum(rows, red), pages0 = add_counts(head, block_sum(pages, red));
  // this block's own requests: consecutive ones to a thread, so that the scan is one over threads
  const int per = (n + TPB - 1) / TPB, own0 = threadIdx.x * per, own1 = min(own0 + per, n);
  rows = pages = 0;
  for (int i = own0; i < own1; ++i) {
    const Lens l = plan_lens(a, s0 + i);
    rows = add_counts(rows, l.add);
    pages = add_counts(pages, l.need - l.had);
    row_end[i] = rows;
    page_end[i] = pages;
    lens_ctx[i] = l.ctx;
    lens_had[i] = l.had;
    longest = max(longest, l.ctx + l.add);
    if (l.need > a.table_stride) faults |= RLGEN_PLAN_TABLE;
    if (l.odd) faults |= RLGEN_PLAN_LENGTH;
    if (writer) a.total_lens[s0 + i] = l.ctx + l.add;
  }
  const int rows_before = add_counts(rows0, block_exclusive(rows, red)), pages_before = add_counts(pages0, block_exclusive(pages, red));
  for (int i = own0; i < own1; ++i) {
    if (writer) a.row_starts[s0 + i] = i > own0 ? row_end[i - 1] : rows_before;
    row_end[i] = add_counts(row_end[i], rows_before);
    page_end[i] = add_counts(page_end[i], pages_before);
  }
  __syncthreads();
  const int rows1 = row_end[n - 1], pages1 = page_end[n - 1];
  if (last && writer) {
    longest = block_max(longest, red);
    if (block_sum(faults & RLGEN_PLAN_TABLE, red)) faults |= RLGEN_PLAN_TABLE;
    if (block_sum((faults & RLGEN_PLAN_LENGTH) ? 1 : 0, red)) faults |= RLGEN_PLAN_LENGTH;
    if (threadIdx.x == 0) {
      if (pages1 > a.n_free || asked > a.n_free) faults |= RLGEN_PLAN_PAGES;
      if (rows1 > a.max_rows || rows1 == MOST) faults |= RLGEN_PLAN_ROWS;
      a.row_starts[a.S] = rows1;
      a.counts[0] = rows1;
      a.counts[1] = min(pages1, a.n_free);
      a.counts[2] = longest;
      a.counts[3] = faults;
    }
  }
  // (a page that the free list no longer has is -1, and so are the slots in it)
  auto fresh = [&](unsigned at) { return at < (unsigned)a.n_free ? a.free_pages[at] : -1; };
  if (writer && pages1 < MOST) {
    for (unsigned at = pages0 + threadIdx.x; at < (unsigned)pages1; at += TPB) {
      int lo = 0, hi = n - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((unsigned)page_end[mid] > at) hi = mid; else lo = mid + 1;
      }
      const int entry = lens_had[lo] + (int)(at - (lo ? page_end[lo - 1] : pages0));
      if (entry < a.table_stride) a.page_table[(size_t)(s0 + lo) * a.table_stride + entry] = fresh(at);
      else at += (page_end[lo] - 1 - at) / TPB * TPB;      // (to the last of this request that would be this thread's: none has a place)
    }
  } else if (writer) {
    // more pages than can be counted: the places in the table are, and those past the free list get none
    for (int i = 0; i < n; ++i) {
      const Lens l = plan_lens(a, s0 + i);
      const unsigned first = i ? page_end[i - 1] : pages0;
      for (int entry = l.had + threadIdx.x; entry < min(l.need, a.table_stride); entry += TPB)
        a.page_table[(size_t)(s0 + i) * a.table_stride + entry] = fresh(first + (entry - l.had));
    }
  }
  const int round = (1 << a.page_shift) - 1;
  const int row_stop = last ? a.max_rows : min(rows1, a.max_rows);
  for (unsigned r = rows0 + blockIdx.y * TPB + threadIdx.x; r < (unsigned)row_stop; r += gridDim.y * TPB) {
    if (r >= (unsigned)rows1) {
      a.slots[r] = -1;
      a.positions[r] = 0;
      continue;
    }
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((unsigned)row_end[mid] > r) hi = mid; else lo = mid + 1;
    }
    const int pos = lens_ctx[lo] + (int)(r - (lo ? row_end[lo - 1] : rows0));
    const int entry = pos >> a.page_shift;
    int page = -1;
    if (entry < a.table_stride)
      page = entry < lens_had[lo] ? a.page_table[(size_t)(s0 + lo) * a.table_stride + entry]
                                  : fresh((unsigned)(lo ? page_end[lo - 1] : pages0) + (entry - lens_had[lo]));
    // (of a page whose slots an int does not hold, one outside any cache, there is none)
    a.slots[r] = page < 0 || page > (MOST >> a.page_shift) ? -1 : (page << a.page_shift) + (pos & round);
    a.positions[r] = pos;
  }
}

// ------------------------------------------------------------------ per-head norm and rotation
// A head's vector sits in LPH lanes of a wave, eight dims to a lane.  One or four waves take a row; their lane groups go through the
// heads of it, first the queries', then the keys', then the values', AHEAD heads of a kind to a step, and the next step is requested before
// the present one is used.  A lane keeps the same dims throughout, so a row's angles are loaded once and met with the gains (which wait in
// LDS, each with its rotary partner's) once for each kind.
template <class T> struct Eight;
template <> struct Eight<float> {
  typedef float word;
  f32x4 a, b;
  static __device__ __forceinline__ Eight load(const void* p, long long at) {
    const float* x = (const float*)p + at;
    return {*(const f32x4*)x, *(const f32x4*)(x + 4)};
  }
  static __device__ __forceinline__ Eight zero() { return {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}}; }
  __device__ __forceinline__ void to(float* y) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { y[e] = a[e]; y[4 + e] = b[e]; }
  }
  __device__ __forceinline__ Eight from_lane(int lane) const {
    Eight r;
#pragma unroll
    for (int e = 0; e < 4; ++e) { r.a[e] = __shfl(a[e], lane, WAVE); r.b[e] = __shfl(b[e], lane, WAVE); }
    return r;
  }
  __device__ __forceinline__ void leave(float* lds) const { *(f32x4*)lds = a; *(f32x4*)(lds + 4) = b; }
  static __device__ __forceinline__ float2 pair(const float* lds, int at) { return *(const float2*)(lds + at); }
  static __device__ __forceinline__ float one(const float* lds, int at) { return lds[at]; }
  static __device__ __forceinline__ void store(void* p, long long at, const float* y) {
    float* x = (float*)p + at;
    *(f32x4*)x = f32x4{y[0], y[1], y[2], y[3]};
    *(f32x4*)(x + 4) = f32x4{y[4], y[5], y[6], y[7]};
  }
};
template <class T> struct Eight {
  typedef uint16_t word;
  u32x4 w;
  static __device__ __forceinline__ Eight load(const void* p, long long at) { return {*(const u32x4*)((const uint16_t*)p + at)}; }
  static __device__ __forceinline__ Eight zero() { return {u32x4{0, 0, 0, 0}}; }
  __device__ __forceinline__ void to(float* y) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) { y[2 * e] = T::low(w[e]); y[2 * e + 1] = T::high(w[e]); }
  }
  __device__ __forceinline__ Eight from_lane(int lane) const {
    Eight r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.w[e] = __shfl(w[e], lane, WAVE);
    return r;
  }
  __device__ __forceinline__ void leave(uint16_t* lds) const { *(u32x4*)lds = w; }
  static __device__ __forceinline__ float2 pair(const uint16_t* lds, int at) {
    const uint32_t v = *(const uint32_t*)(lds + at);
    return make_float2(T::low(v), T::high(v));
  }
  static __device__ __forceinline__ float one(const uint16_t* lds, int at) { return T::low(lds[at]); }
  static __device__ __forceinline__ void store(void* p, long long at, const float* y) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = T::pack(y[2 * e], y[2 * e + 1]);
    *(u32x4*)((uint16_t*)p + at) = w;
  }
};

__device__ __forceinline__ int rotary_partner(int d, int r) { return d < (r >> 1) ? d + (r >> 1) : d < r ? d - (r >> 1) : d; }
// A lane's angles at one position: out = y c + (the partner's y) t, t with the partner's sign; c = 1, t = 0 for dims past r
struct Angles { float c[8], t[8]; };
__device__ __forceinline__ void load_angles(Angles& w, const float2* rope, int r, int pos, int d0, float sign) {
  const int half = r >> 1;
  const float2* row = rope + (size_t)pos * half;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = d0 + e;
    const float2 v = d < r ? row[d < half ? d : d - half] : make_float2(1.f, 0.f);
    w.c[e] = v.x;
    w.t[e] = d < half ? -sign * v.y : sign * v.y;
  }
}
// The rotary partners of AHEAD heads' values.  ALIGNED: half a rotation is whole lanes, which exchange their registers; else the rotated
// lanes leave them in LDS and read them shifted, in pairs where half a rotation is even.
template <class T, bool ALIGNED, int AHEAD, int LPH>
__device__ __forceinline__ void partners(const Eight<T> (&x)[AHEAD], float (&y)[AHEAD][8], typename Eight<T>::word* lds, int d0, int r, int lane0) {
  const int half = r >> 1;
  if constexpr (ALIGNED) {
    const int from = lane0 + (rotary_partner(d0, r) >> 3);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u].from_lane(from).to(y[u]);
  } else {
    const bool turned = d0 < r;
    __builtin_amdgcn_wave_barrier();          // (the readers of what this overwrites are lanes of this wave)
    if (turned) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) x[u].leave(lds + u * LPH * 8 + d0);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) y[u][e] = 0.f;
    if (turned) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (half & 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[u][e] = d0 + e < r ? Eight<T>::one(lds + u * LPH * 8, rotary_partner(d0 + e, r)) : 0.f;
        } else {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float2 v = d0 + e < r ? Eight<T>::pair(lds + u * LPH * 8, rotary_partner(d0 + e, r)) : make_float2(0.f, 0.f);
            y[u][e] = v.x;
            y[u][e + 1] = v.y;
          }
        }
    }
  }
}
template <int LPH> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}
// One step of a row: AHEAD heads of one kind to a lane group
enum { QUERIES, KEYS, VALUES };
struct Step { int kind, first; };
template <int AHEAD> __device__ __forceinline__ Step step_of(int j, int groups, int Hq, int Hkv) {
  const int per = groups * AHEAD, nq = (Hq + per - 1) / per, nk = (Hkv + per - 1) / per;
  return j < nq ? Step{QUERIES, j * per} : j < nq + nk ? Step{KEYS, (j - nq) * per} : Step{VALUES, (j - nq - nk) * per};
}
template <int AHEAD> __device__ __forceinline__ int steps_of(int groups, int Hq, int Hkv) {
  const int per = groups * AHEAD;
  return (Hq + per - 1) / per + 2 * ((Hkv + per - 1) / per);
}

// Bound by HBM: every head is read and written once.  Measured: 8056 rows of 96 heads of 80 in fp16 67 us, 3.7 TB/s; 128 rows of 48 heads of
// 128: 7 us, a launch and three dependent loads (the position, its angles, the heads).  Registers for four waves to a SIMD and two heads of a
// lane group at once (three waves where sources are 32 bits wide).
template <class TI, class TO, int LPH, bool ALIGNED>
__global__ __launch_bounds__(TPB, sizeof(typename Eight<TI>::word) == 2 ? 4 : 3) void norm_rope_kernel(NormRopeArgs a, int row_waves) {
  constexpr int AHEAD = 2;
  typedef typename Eight<TI>::word word;
  __shared__ __attribute__((aligned(16))) float gains[2][2][LPH * 8];            // of queries, keys: a dim's own, its partner's
  __shared__ __attribute__((aligned(16))) word shift[ALIGNED ? 1 : TPB / LPH][ALIGNED ? 1 : AHEAD * LPH * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane % LPH, d0 = li * 8, lane0 = lane - li;
  for (int d = threadIdx.x; d < LPH * 8; d += TPB) {
    const int p = rotary_partner(d, a.r);
    gains[0][0][d] = d < a.h ? a.q_gain[d] : 0.f;
    gains[0][1][d] = d < a.h ? a.q_gain[p] : 0.f;
    gains[1][0][d] = d < a.h ? a.k_gain[d] : 0.f;
    gains[1][1][d] = d < a.h ? a.k_gain[p] : 0.f;
  }
  __syncthreads();
  const bool on = d0 < a.h;
  const float inv_h = 1.0f / (float)a.h;
  const int groups = row_waves * (64 / LPH), group = (wave & (row_waves - 1)) * (64 / LPH) + lane / LPH;
  const int n_steps = steps_of<AHEAD>(groups, a.Hq, a.Hkv);
  const int per_block = 4 / row_waves, row_step = gridDim.x * per_block;
  auto load = [&](int row, int j, Eight<TI> (&x)[AHEAD]) {
    const Step s = step_of<AHEAD>(j, groups, a.Hq, a.Hkv);
    const int heads = s.kind == QUERIES ? a.Hq : a.Hkv, head0 = s.kind == QUERIES ? 0 : s.kind == KEYS ? a.Hq : a.Hq + a.Hkv;
    const long long src = (long long)row * a.qkv_stride + (long long)head0 * a.h + d0;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int hd = s.first + u * groups + group;
      x[u] = on && hd < heads ? Eight<TI>::load(a.qkv, src + (long long)hd * a.h) : Eight<TI>::zero();
    }
  };
  int row = blockIdx.x * per_block + wave / row_waves;
  if (row >= a.rows) return;
  Eight<TI> x[AHEAD], x_next[AHEAD];
  load(row, 0, x);
  int pos = a.positions[row], slot = a.pages ? a.slots[row] : -1;
  for (; row < a.rows; row += row_step) {
    Angles w;
    load_angles(w, a.rope, on ? a.r : 0, min(max(pos, 0), a.max_pos - 1), d0, 1.f);
    const int page = slot >> a.page_shift, to_slot = slot >= 0 && page < a.n_pages ? slot : -1;
    const int row_next = row + row_step;
    if (row_next < a.rows) {
      pos = a.positions[row_next];
      if (a.pages) slot = a.slots[row_next];
    }
    float own[8], other[8];
    int kind = -1;
    for (int j = 0; j < n_steps; ++j) {
      if (j + 1 < n_steps) load(row, j + 1, x_next);
      else if (row_next < a.rows) load(row_next, 0, x_next);
      const Step s = step_of<AHEAD>(j, groups, a.Hq, a.Hkv);
      const int heads = s.kind == QUERIES ? a.Hq : a.Hkv;
      if (s.kind != kind && s.kind != VALUES) {
        kind = s.kind;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          own[e] = gains[kind][0][d0 + e] * w.c[e];
          other[e] = gains[kind][1][d0 + e] * w.t[e];
        }
      }
      float p[AHEAD][8];
      if (s.kind != VALUES) partners<TI, ALIGNED, AHEAD, LPH>(x, p, shift[ALIGNED ? 0 : threadIdx.x / LPH], d0, a.r, lane0);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int hd = s.first + u * groups + group;
        float y[8];
        x[u].to(y);
        if (s.kind != VALUES) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
          const float inv = rsqrtf(fmaf(group_sum<LPH>(ss), inv_h, a.eps));
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = inv * fmaf(y[e], own[e], p[u][e] * other[e]);
        }
        if (!on || hd >= heads) continue;
        if (s.kind == QUERIES) {
          Eight<TO>::store(a.q, (long long)row * a.q_stride + (long long)hd * a.h + d0, y);
          continue;
        }
        const int which = s.kind == VALUES;
        if (to_slot >= 0) {
          const long long at = ((((long long)page * 2 + which) * a.Hkv + hd) << a.page_shift) + (to_slot & ((1 << a.page_shift) - 1));
          Eight<TO>::store(a.pages, at * a.h + d0, y);
        }
        void* dst = which ? a.v : a.k;
        if (dst) Eight<TO>::store(dst, (long long)row * (which ? a.v_stride : a.k_stride) + (long long)hd * a.h + d0, y);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) x[u] = x_next[u];
    }
  }
}

// Gradients: the same walk over x and the incoming gradients.  The gains' gradients are sums over all rows and heads: every lane keeps
// those of its dims in registers over all its rows, the lane groups of the block meet in LDS in their order, and a second launch adds up
// the blocks, so that a result does not depend on which block came first.  Bound by HBM: 8193 rows of 48 heads of 128 in 61 us, 4.7 TB/s, and 5
// us for the second launch.
template <class TI, class TO, int LPH, bool ALIGNED>
__global__ __launch_bounds__(TPB) void norm_rope_backward_kernel(NormRopeArgs a, int row_waves) {
  constexpr int AHEAD = 1;
  typedef typename Eight<TO>::word word;
  __shared__ __attribute__((aligned(16))) float gains[2][LPH * 8];
  __shared__ __attribute__((aligned(16))) float sums[TPB / LPH][LPH * 8];
  __shared__ __attribute__((aligned(16))) word shift[ALIGNED ? 1 : TPB / LPH][ALIGNED ? 1 : AHEAD * LPH * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane % LPH, d0 = li * 8, lane0 = lane - li;
  for (int d = threadIdx.x; d < LPH * 8; d += TPB) {
    gains[0][d] = d < a.h ? a.q_gain[d] : 0.f;
    gains[1][d] = d < a.h ? a.k_gain[d] : 0.f;
  }
  __syncthreads();
  const bool on = d0 < a.h;
  const float inv_h = 1.0f / (float)a.h;
  const int groups = row_waves * (64 / LPH), group = (wave & (row_waves - 1)) * (64 / LPH) + lane / LPH;
  const int n_steps = steps_of<AHEAD>(groups, a.Hq, a.Hkv);
  const int per_block = 4 / row_waves, row_step = gridDim.x * per_block;
  auto load = [&](int row, int j, Eight<TI> (&x)[AHEAD], Eight<TO> (&g)[AHEAD]) {
    const Step s = step_of<AHEAD>(j, groups, a.Hq, a.Hkv);
    const int heads = s.kind == QUERIES ? a.Hq : a.Hkv;
    const void* from = s.kind == QUERIES ? a.dq : s.kind == KEYS ? a.dk : a.dv;
    const long long at = (long long)row * (s.kind == QUERIES ? a.dq_stride : s.kind == KEYS ? a.dk_stride : a.dv_stride) + d0;
    const long long src = (long long)row * a.qkv_stride + (s.kind == QUERIES ? 0ll : (long long)a.Hq * a.h) + d0;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int hd = s.first + u * groups + group;
      const bool live = on && hd < heads;
      x[u] = live && s.kind != VALUES ? Eight<TI>::load(a.qkv, src + (long long)hd * a.h) : Eight<TI>::zero();
      g[u] = live ? Eight<TO>::load(from, at + (long long)hd * a.h) : Eight<TO>::zero();
    }
  };
  float sum_q[8], sum_k[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum_q[e] = sum_k[e] = 0.f;
  int row = blockIdx.x * per_block + wave / row_waves;
  Eight<TI> x[AHEAD], x_next[AHEAD];
  Eight<TO> g[AHEAD], g_next[AHEAD];
  int pos = 0;
  if (row < a.rows) {
    load(row, 0, x, g);
    pos = a.positions[row];
  }
  for (; row < a.rows; row += row_step) {
    Angles w;
    load_angles(w, a.rope, on ? a.r : 0, min(max(pos, 0), a.max_pos - 1), d0, -1.f);
    const int row_next = row + row_step;
    if (row_next < a.rows) pos = a.positions[row_next];
    for (int j = 0; j < n_steps; ++j) {
      if (j + 1 < n_steps) load(row, j + 1, x_next, g_next);
      else if (row_next < a.rows) load(row_next, 0, x_next, g_next);
      const Step s = step_of<AHEAD>(j, groups, a.Hq, a.Hkv);
      const int heads = s.kind == QUERIES ? a.Hq : a.Hkv, head0 = s.kind == QUERIES ? 0 : s.kind == KEYS ? a.Hq : a.Hq + a.Hkv;
      float p[AHEAD][8];
      if (s.kind != VALUES) partners<TO, ALIGNED, AHEAD, LPH>(g, p, shift[ALIGNED ? 0 : threadIdx.x / LPH], d0, a.r, lane0);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int hd = s.first + u * groups + group;
        float d[8];
        g[u].to(d);
        if (s.kind != VALUES) {
          float y[8], t[8], ss = 0.f, tx = 0.f;
          x[u].to(y);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            d[e] = fmaf(d[e], w.c[e], p[u][e] * w.t[e]);
            t[e] = d[e] * gains[s.kind][d0 + e];
            ss = fmaf(y[e], y[e], ss);
            tx = fmaf(t[e], y[e], tx);
          }
          ss = group_sum<LPH>(ss);
          tx = group_sum<LPH>(tx);
          const float inv = rsqrtf(fmaf(ss, inv_h, a.eps)), back = inv * inv * tx * inv_h;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float dg = d[e] * (y[e] * inv);
            if (s.kind == QUERIES) sum_q[e] += dg; else sum_k[e] += dg;
            d[e] = inv * (t[e] - y[e] * back);
          }
        }
        if (on && hd < heads) Eight<TI>::store(a.dqkv, (long long)row * a.dqkv_stride + (long long)(head0 + hd) * a.h + d0, d);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        x[u] = x_next[u];
        g[u] = g_next[u];
      }
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x / LPH][d0 + e] = which ? sum_k[e] : sum_q[e];
    __syncthreads();
    for (int d = threadIdx.x; d < a.h; d += TPB) {
      float v = 0.f;
      for (int i = 0; i < TPB / LPH; ++i) v += sums[i][d];
      a.partial[((size_t)blockIdx.x * 2 + which) * a.h + d] = v;
    }
  }
}

// The gains' gradients over the blocks of norm_rope_backward_kernel: a block adds up eight dims, 128 runs of blocks at once and then the
// runs, always in the same order.
__global__ __launch_bounds__(1024) void gain_grad_kernel(const float* partial, int blocks, int h, float* dq_gain, float* dk_gain) {
  __shared__ float red[128][8];
  const int col = threadIdx.x & 7, part = threadIdx.x >> 3, d = blockIdx.x * 8 + col;       // 2 h is a multiple of 8
  float v = 0.f;
#pragma unroll 8
  for (int b = part; b < blocks; b += 128) v += partial[(size_t)b * 2 * h + d];
  red[part][col] = v;
  __syncthreads();
  if (part < 8) {
    for (int p = part + 8; p < 128; p += 8) v += red[p][col];
    // the eight runs left sit in lanes 8 apart
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) v += __shfl_xor(v, o, WAVE);
    if (part == 0) (d < h ? dq_gain : dk_gain - h)[d] = v;
  }
}

// Blocks, and waves to a row.  Four waves share a row while rows are fewer than waves that the CUs hold (128 rows of 48 heads of 128: 7.2
// us, 10.9 with a wave to a row); beyond that a row to a wave spares the others' copies of its angles (8056 rows of 96 heads of 80: 67 us,
// 85 with four waves to a row).
struct Launch { int blocks, row_waves; };
Launch norm_rope_launch(int rows) {
  const int row_waves = rows < 4096 ? 4 : 1;
  const long long blocks = ((long long)rows * row_waves + 3) / 4;
  return {(int)(blocks < 1024 ? blocks : 1024), row_waves};
}
template <class TI, class TO, int LPH>
hipError_t launch_norm_rope(const NormRopeArgs& a, bool backward, Launch l, hipStream_t s) {
  const bool aligned = (a.r >> 1) % 8 == 0;
  const dim3 grid(l.blocks), block(TPB);
  if (backward) {
    if (aligned) hipLaunchKernelGGL((norm_rope_backward_kernel<TI, TO, LPH, true>), grid, block, 0, s, a, l.row_waves);
    else hipLaunchKernelGGL((norm_rope_backward_kernel<TI, TO, LPH, false>), grid, block, 0, s, a, l.row_waves);
  } else {
    if (aligned) hipLaunchKernelGGL((norm_rope_kernel<TI, TO, LPH, true>), grid, block, 0, s, a, l.row_waves);
    else hipLaunchKernelGGL((norm_rope_kernel<TI, TO, LPH, false>), grid, block, 0, s, a, l.row_waves);
  }
  return hipGetLastError();
}
template <class TI, class TO>
hipError_t by_head(const NormRopeArgs& a, bool backward, Launch l, hipStream_t s) {
  if (a.h <= 64) return launch_norm_rope<TI, TO, 8>(a, backward, l, s);
  if (a.h <= 128) return launch_norm_rope<TI, TO, 16>(a, backward, l, s);
  return launch_norm_rope<TI, TO, 32>(a, backward, l, s);
}
hipError_t by_type(const NormRopeArgs& a, bool backward, Launch l, hipStream_t s) {
  const bool f16 = a.dtype == RLGEN_DTYPE_F16;
  switch (a.src_dtype) {
    case RLGEN_DTYPE_F32: return f16 ? by_head<float, TypeF16>(a, backward, l, s) : by_head<float, TypeBf16>(a, backward, l, s);
    case RLGEN_DTYPE_BF16: return f16 ? by_head<TypeBf16, TypeF16>(a, backward, l, s) : by_head<TypeBf16, TypeBf16>(a, backward, l, s);
    case RLGEN_DTYPE_F16: return f16 ? by_head<TypeF16, TypeF16>(a, backward, l, s) : by_head<TypeF16, TypeBf16>(a, backward, l, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t rl_plan_pages(PlanArgs a, hipStream_t s) {
  // 256 blocks of requests at most while a block's requests fit its LDS (1000 requests of one token: 5.6 us, 6.6 in 16 blocks; 512 prompts of
  // 256 to 512 tokens: 6.5 us, 9.0); rows of a group are parted until a part has 1024 of them or the launch 1024 blocks (4
  // requests of 50000 tokens: 8.5 us, 22 with parts of 16384)
  a.group = (a.S + 255) / 256;
  if (a.group > PLAN_GROUP) a.group = PLAN_GROUP;
  const int groups = (a.S + a.group - 1) / a.group;
  const long long per = ((long long)a.max_rows + groups - 1) / groups;
  long long chunks = (per + 1023) / 1024, most = 1024 / groups > 1 ? 1024 / groups : 1;
  a.chunks = (int)(chunks < 1 ? 1 : chunks < most ? chunks : most);
  hipLaunchKernelGGL(plan_pages_kernel, dim3(groups, a.chunks), dim3(TPB), 0, s, a);
  return hipGetLastError();
}
hipError_t rl_norm_rope(const NormRopeArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return by_type(a, false, norm_rope_launch(a.rows), s);
}
size_t rl_norm_rope_backward_bytes(int rows, int h) { return (size_t)norm_rope_launch(rows < 1 ? 1 : rows).blocks * 2 * h * sizeof(float); }
hipError_t rl_norm_rope_backward(const NormRopeArgs& a, hipStream_t s) {
  const Launch l = norm_rope_launch(a.rows);
  if (l.blocks > 0) {
    const hipError_t e = by_type(a, true, l, s);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(gain_grad_kernel, dim3(a.h / 4), dim3(1024), 0, s, a.partial, l.blocks, a.h, a.dq_gain, a.dk_gain);
  return hipGetLastError();
}
