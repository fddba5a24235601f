// Log-probs of given tokens, entropy and the n likeliest tokens of rows of logits, in one pass over them, and the gradient of the first two.
//   m = max z, S = sum exp((z - m) / T), log p_j = (z_j - m) / T - log S, H = log S - sum p_j (z_j - m) / T
//   dz_j = (g (1[j = t] - p_j) - h p_j (log p_j + H)) / T
#include "learner.h"
#include "../../include/rlgen.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.4028234663852886e38f;

// 16 bytes of a row's logits: read at multiples of 16, written anywhere (the gradient's row may start elsewhere within 16 bytes than the logits'; global
// memory takes such stores at no loss: 2461 rows of 50304 bf16 values 100 us either way, 149 element by element)
typedef u32x4 any4 __attribute__((aligned(2)));
typedef f32x4 any4f __attribute__((aligned(4)));
template <class E> struct Some {
  static constexpr int N = 8;
  u32x4 w;
  template <bool ONCE = false> static __device__ __forceinline__ Some load(const void* row, long long at) {
    return {take<ONCE>((const u32x4*)((const uint16_t*)row + at))};
  }
  static __device__ __forceinline__ Some of(u32x4 w) { return {w}; }
  __device__ __forceinline__ void opaque() { asm volatile("" : "+v"(w)); }     // what is known of the values ends here
  static __device__ __forceinline__ Some masked() {
    const uint32_t w = E::pack(-INFINITY, -INFINITY);
    return {u32x4{w, w, w, w}};
  }
  __device__ __forceinline__ float operator[](int e) const { return e & 1 ? E::high(w[e >> 1]) : E::low(w[e >> 1]); }
  static __device__ __forceinline__ float one(const void* row, long long at) { return E::low(((const uint16_t*)row)[at]); }
  template <bool ONCE> static __device__ __forceinline__ void store(void* row, long long at, const float* y) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = E::pack(y[2 * e], y[2 * e + 1]);
    if constexpr (ONCE) __builtin_nontemporal_store(w, (any4*)((uint16_t*)row + at));
    else *(any4*)((uint16_t*)row + at) = w;
  }
  static __device__ __forceinline__ void store_one(void* row, long long at, float y) { ((uint16_t*)row)[at] = (uint16_t)E::pack(y, 0.f); }
};
template <> struct Some<TypeF32> {
  static constexpr int N = 4;
  f32x4 w;
  template <bool ONCE = false> static __device__ __forceinline__ Some load(const void* row, long long at) {
    return {take<ONCE>((const f32x4*)((const float*)row + at))};
  }
  static __device__ __forceinline__ Some of(u32x4 w) { return {__builtin_bit_cast(f32x4, w)}; }
  __device__ __forceinline__ void opaque() {}
  static __device__ __forceinline__ Some masked() { return {f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY}}; }
  __device__ __forceinline__ float operator[](int e) const { return w[e]; }
  static __device__ __forceinline__ float one(const void* row, long long at) { return ((const float*)row)[at]; }
  template <bool ONCE> static __device__ __forceinline__ void store(void* row, long long at, const float* y) {
    const f32x4 v = {y[0], y[1], y[2], y[3]};
    if constexpr (ONCE) __builtin_nontemporal_store(v, (any4f*)((float*)row + at));
    else *(any4f*)((float*)row + at) = v;
  }
  static __device__ __forceinline__ void store_one(void* row, long long at, float y) { ((float*)row)[at] = y; }
};
template <class E> constexpr int SIZE = 16 / Some<E>::N;

// A row may start anywhere: `head` elements up to the first 16-byte border, then `full` pieces of 16 bytes (the first one at element `first`),
// then `tail` elements.  Of a row that is parted the first part has the head and the tail beside its pieces.
struct Cut { int head, first, full, tail; };
template <class E> __device__ __forceinline__ Cut cut_row(const void* row, int vocab) {
  constexpr int N = Some<E>::N;
  const int lead = (int)((uintptr_t)row & 15) / SIZE<E>;
  Cut c;
  c.head = c.first = lead ? min(N - lead, vocab) : 0;
  c.full = (vocab - c.head) / N;
  c.tail = vocab - c.head - c.full * N;
  return c;
}
template <class E> __device__ __forceinline__ Cut cut_part(Cut c, int part, int parts) {
  const int per = (c.full + parts - 1) / parts, from = min(part * per, c.full);
  c.full = min(per, c.full - from);
  c.first += from * Some<E>::N;
  if (part > 0) c.head = c.tail = 0;
  return c;
}
// The pieces of a row through a bounded buffer: past the last one a load brings zeros and no traffic
template <class E> __device__ __forceinline__ auto pieces_of(const void* row, const Cut& c) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)row + (long long)c.first * SIZE<E>), 0, c.full * 16, 0x00027000);
}
template <class E> __device__ __forceinline__ const void* row_at(const void* p, long long row, long long stride) {
  return (const char*)p + row * stride * SIZE<E>;
}
// the element of the head or the tail that this thread has, -1: none
__device__ __forceinline__ int edge_of(const Cut& c, int vocab) {
  const int t = threadIdx.x;
  return t < c.head ? t : t >= 8 && t - 8 < c.tail ? vocab - c.tail + t - 8 : -1;
}

// An order of values as whole numbers: NaN above infinity, both zeros the same
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// larger values first, of equal ones the lower index
__device__ __forceinline__ uint64_t key_of(uint32_t order, int index) { return ((uint64_t)order << 32) | (0xffffffffu - (uint32_t)index); }

template <int T> __device__ __forceinline__ int count_block(int v, int* slots) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) t += slots[w];
  return t;
}
// The n-th largest of the lanes' values, n from 1 to 64
__device__ __forceinline__ float nth_of_lanes(float v, int n) {
  float most = lanes_max(v);
  for (int i = 1; i < n; ++i) {
    const unsigned long long at = __ballot(v == most);
    if (__ffsll((long long)at) - 1 == (int)(threadIdx.x & 63)) v = -INFINITY;
    most = lanes_max(v);
  }
  return most;
}

constexpr int CANDIDATES = 512, EQUALS = 256, HITS = 512;

// What the likeliest tokens' search holds in LDS
struct Found {
  uint64_t key[CANDIDATES], same[EQUALS];        // of values above the bound, and equal to it
  uint32_t hit[HITS];                            // steps of threads that hold such values: step * T + thread
  int counts[16];
  int hits, above, equal;
};

template <class F> __device__ __forceinline__ void note_hits(const float* kept, int steps, int threads, F&& wanted, Found& f) {
#pragma unroll 4
  for (int step = 0; step < steps; ++step)
    if (wanted(kept[step * threads + threadIdx.x])) {
      const int i = atomicAdd(&f.hits, 1);
      if (i < HITS) f.hit[i] = step * threads + threadIdx.x;
    }
}

// Of the values equal to `least` (as orders) the first ones, in the order of their indices (the head, the pieces, the tail), behind the
// `have` keys that there are, until there are n.
template <class E, int T> __device__ void fill_equal(const void* row, const Cut& c, int vocab, int n, uint32_t least, int have, Found& f) {
  constexpr int N = Some<E>::N;
  const int turns = 2 + (c.full + T - 1) / T;
  for (int turn = 0; turn < turns && have < n; ++turn) {
    uint32_t same = 0;
    int first = 0;
    if (turn == 0 || turn == turns - 1) {
      const int at = turn == 0 ? ((int)threadIdx.x < c.head ? (int)threadIdx.x : -1)
                               : ((int)threadIdx.x < c.tail ? vocab - c.tail + (int)threadIdx.x : -1);
      if (at >= 0 && order_of(Some<E>::one(row, at)) == least) { same = 1; first = at; }
    } else {
      const int k = (turn - 1) * T + threadIdx.x;
      if (k < c.full) {
        const Some<E> s = Some<E>::load(row, c.first + (long long)k * N);
        first = c.first + k * N;
#pragma unroll
        for (int e = 0; e < N; ++e) same |= (order_of(s[e]) == least ? 1u : 0u) << e;
      }
    }
    // places before this thread's: lanes before it, waves before its own
    const int mine = __popc(same), lane = threadIdx.x & 63;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int t = __shfl_up(upto, o, WAVE);
      if (lane >= o) upto += t;
    }
    __syncthreads();
    if (lane == 63) f.counts[threadIdx.x >> 6] = upto;
    __syncthreads();
    int at = have + upto - mine, all = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
      if (w < (int)(threadIdx.x >> 6)) at += f.counts[w];
      all += f.counts[w];
    }
    for (; same && at < n; same &= same - 1, ++at) f.key[at] = key_of(least, first + __ffs((int)same) - 1);
    have += all;
  }
  __syncthreads();
}

// The n largest of a row where no simple bound leaves few values (crowded ones, NaN): the n-th largest order by halving, every step counting
// over the row, then the values above it, and of those equal to it the first ones.  33 passes over the row, which is what it costs: with a NaN in every row 64
// rows of 128256 bf16 values 202 us (16 without), 300 of 100003 881 (22), 256 of 50304 338 (13), one of 50304 279 (12); 70 rows of 400003, more than maxima
// are kept of, 3290 (40 for 390003).
template <class E, int T> __device__ void select_top(const void* row, const Cut& c, int vocab, int n, Found& f) {
  constexpr int N = Some<E>::N;
  const int edge = edge_of(c, vocab);
  auto each = [&](auto&& use) {
    for (int k = threadIdx.x; k < c.full; k += T) {
      const Some<E> s = Some<E>::load(row, c.first + (long long)k * N);
#pragma unroll
      for (int e = 0; e < N; ++e) use(order_of(s[e]), c.first + k * N + e);
    }
    if (edge >= 0) use(order_of(Some<E>::one(row, edge)), edge);
  };
  uint32_t least = 0;                              // the n-th largest order, as far as its bits have been found
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t trial = least | (1u << bit);
    int mine = 0;
    each([&](uint32_t o, int) { mine += o >= trial; });
    if (count_block<T>(mine, f.counts) >= n) least = trial;
  }
  __syncthreads();
  if (threadIdx.x == 0) f.above = 0;
  __syncthreads();
  each([&](uint32_t o, int at) {
    if (o > least) f.key[atomicAdd(&f.above, 1)] = key_of(o, at);     // (fewer than n of them)
  });
  __syncthreads();
  fill_equal<E, T>(row, c, vocab, n, least, f.above, f);
}

// What a row adds up to: its largest value, the sum of the terms 2^y, and that of y 2^y.  Where one value has more than half of the probability its own
// term, 1, is counted (once) and not among the sums: beside it the others would keep few of their bits.
struct Sums { float M, count, sum, along; };
__device__ __forceinline__ bool all_masked(const Sums& s) { return s.M == -INFINITY && s.sum == 0.f; }
__device__ __forceinline__ float log_sum_of(const Sums& s) {
  // (log(1 + x) as log(u) x / (u - 1) with u = 1 + x rounded, which makes up for the rounding: Goldberg, "What every computer scientist should know about
  // floating-point arithmetic", 1991, theorem 4; -infinity for a row that is masked as a whole)
  const float u = s.count + s.sum, l = logf(u);
  return s.count == 1.f && u < 2.f ? (u == 1.f ? s.sum : l * (s.sum / (u - 1.f))) : l;
}
__device__ __forceinline__ void finish(const LogprobArgs& a, long long row, const Sums& s, float z_token) {
  const bool empty = all_masked(s);
  const float log_sum = log_sum_of(s);
  if (a.logprobs) a.logprobs[row] = empty ? -INFINITY : (z_token - s.M) / a.temperature - log_sum;
  a.stats[2 * row] = s.M;
  a.stats[2 * row + 1] = log_sum;
  if (a.entropy) a.entropy[row] = empty ? 0.f : log_sum - s.along / (s.count + s.sum) * LN2;
}
// An alternative's place in the result
struct Likely {
  float M, log_sum, temperature;
  bool empty;
  __device__ __forceinline__ void put(const LogprobArgs& a, long long row, int rank, uint64_t key) const {
    const long long at = row * a.n_top + rank;
    a.top_tokens[at] = (int)(0xffffffffu - (uint32_t)key);
    a.top_logprobs[at] = empty ? -INFINITY : (value_of((uint32_t)(key >> 32)) - M) / temperature - log_sum;
  }
};
__device__ __forceinline__ Likely likely_of(const Sums& s, float temperature) { return {s.M, log_sum_of(s), temperature, all_masked(s)}; }
// Each key's place among them all, for those among the first n
template <class F> __device__ __forceinline__ void rank_keys(const uint64_t* keys, int have, int n, int threads, F&& put) {
  for (int i = threadIdx.x; i < have; i += threads) {
    const uint64_t key = keys[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < have; ++j) rank += keys[j] > key;
    if (rank < n) put(key, rank);
  }
}
// A row that was not asked for
template <bool TOP> __device__ __forceinline__ void leave_out(const LogprobArgs& a, long long row) {
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[row] = 0.f;
    a.stats[2 * row] = a.stats[2 * row + 1] = 0.f;
    if (a.entropy) a.entropy[row] = 0.f;
  }
  if (TOP && (int)threadIdx.x < a.n_top) {
    a.top_tokens[row * a.n_top + threadIdx.x] = -1;
    a.top_logprobs[row * a.n_top + threadIdx.x] = -INFINITY;
  }
}

// One block to a row or to a part of one, one pass.  Every lane sums exp((z - m) / T) relative to the largest value m that its wave has met, which rises
// a few times a row; the entropy's sum goes along.  The likeliest tokens cost the pass a maximum per thread and step, kept in LDS: a wave's share of
// n among its lanes' maxima bounds the n-th largest from below so closely that little more than n values lie above, and only the steps
// that hold one are read again, a value to a thread.  ONE: a row of a single step, whose values are still in registers then.
// Bound by HBM where rows are many.
template <class E, int T, bool TOP, bool ONE, bool ONCE>
__global__ __launch_bounds__(T) void token_logprobs_kernel(LogprobArgs a, int steps_kept, int parts) {
  constexpr int N = Some<E>::N, U = 32 / N, WAVES = T / 64;
  extern __shared__ float kept[];                // [steps][T]: the largest value of a thread's step
  __shared__ float red[4][WAVES];
  __shared__ Found found;
  const int row = parts > 1 ? blockIdx.x / parts : blockIdx.x, part = parts > 1 ? blockIdx.x % parts : 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int token = a.tokens ? a.tokens[row] : 0;
  if (a.tokens && (token < 0 || token >= a.vocab)) {          // not asked for
    if (parts == 1) leave_out<TOP>(a, row);
    return;
  }
  const void* z = row_at<E>(a.logits, row, a.stride);
  Cut c = cut_row<E>(z, a.vocab);
  if (parts > 1) c = cut_part<E>(c, part, parts);
  const float scale = LOG2E / a.temperature;
  const int steps = ONE ? 1 : (c.full + T * U - 1) / (T * U);
  const auto pieces = pieces_of<E>(z, c);
  auto load = [&](int step, Some<E> (&s)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] = Some<E>::of(__builtin_amdgcn_raw_buffer_load_b128(pieces, ((step * U + u) * T + threadIdx.x) * 16, 0, ONCE ? 2 : 0));
  };
  // (requested first, so that waiting for these leaves the pieces on their way)
  const int edge = edge_of(c, a.vocab);
  const float some_edge = Some<E>::one(z, max(edge, 0)), z_token = Some<E>::one(z, token);
  Some<E> s0[U], s1[U];
  load(0, s0);
  if (!ONE) load(1, s1);
  const float at_edge = edge >= 0 ? some_edge : -INFINITY;
  // In powers of two, relative to m: a term is 2^y with y = v scale - shift, one fma, where shift is base scale rounded to a float; the largest value's own
  // y is then `off`, known exactly and taken out at the end.  (Where base scale is so large that off would be: y = (v - base) scale.)
  float m = -INFINITY, own = at_edge, sum = 0.f, along = 0.f;     // m: of the wave, own: of this lane
  float base = 0.f, shift = 0.f, off = 0.f;                       // base: m, or 0 before there is one
  bool near = true, masks = false;                                // masks: this wave has met masked values
  auto rise = [&](float most) {                                   // m to the largest of the lanes'
    if (!__any(most > m)) return;
    const float up = lanes_max(fmaxf(most, m)), before = off;
    shift = up * scale;
    near = fabsf(shift) < 65536.f;
    off = near ? fmaf(up, scale, -shift) : 0.f;
    if (m == -INFINITY) {
      along = 0.f;                               // (nothing but NaN so far)
    } else {
      const float by = (m - up) * scale - before + off, f = __builtin_amdgcn_exp2f(by);
      along = f > 0.f ? fmaf(sum, by, along) * f : 0.f;         // (by may be infinite)
      sum *= f;
    }
    m = base = up;
  };
  auto add = [&](float v) {
    const float y = fmaf(v - base, scale, off), e = __builtin_amdgcn_exp2f(y);
    sum += e;
    along = fmaf(e, fmaxf(y, LOWEST), along);    // (a masked value counts 0, not 0 times infinity)
  };
  auto use = [&](int step, Some<E> (&s)[U]) {
    const bool whole = (step + 1) * (T * U) <= c.full;
    if (!whole) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((step * U + u) * T + (int)threadIdx.x >= c.full) s[u] = Some<E>::masked();
    }
    float most = s[0][0];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) most = fmaxf(most, s[u][e]);
    rise(most);
    own = fmaxf(own, most);
    if (TOP && !ONE && step < steps_kept) kept[step * T + threadIdx.x] = most;
    // a step's own sums, so that a masked value (0 times minus infinity in the second) shows there, and is left out in a second go
    float step_sum = 0.f, step_along = 0.f;
    if (near && whole && !masks) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float y = fmaf(s[u][e], scale, -shift), f = __builtin_amdgcn_exp2f(y);
          step_sum += f;
          step_along = fmaf(f, y, step_along);
        }
    }
    if (!near || !whole || masks || __any(step_along != step_along)) {
      masks |= near && whole;                    // (where some are, there are more as a rule: the next steps take this way at once)
#pragma unroll
      for (int u = 0; u < U; ++u) s[u].opaque();           // (widened again: kept, they would cost every step 30 registers)
      const float sum_before = sum, along_before = along;
      sum = along = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < N; ++e) add(s[u][e]);
      step_sum = sum;
      step_along = along;
      sum = sum_before;
      along = along_before;
    }
    sum += step_sum;
    along += step_along;
  };
  if (TOP && threadIdx.x == 0) found.hits = found.above = found.equal = 0;
  if constexpr (ONE) {
    use(0, s0);
  } else {
    for (int step = 0; step < steps; step += 2) {
      use(step, s0);
      load(step + 2, s0);
      if (step + 1 >= steps) break;
      use(step + 1, s1);
      load(step + 3, s1);
    }
  }
  if (c.head + c.tail > 0) {
    rise(at_edge);
    add(at_edge);
  }
  // over the block
  if (lane == 0) red[0][wave] = m;
  const int n = TOP ? min(a.n_top, c.head + c.tail + c.full * N) : 0;
  if constexpr (TOP) {
    // the waves that have values: a short row fills the first ones
    const int busy = max(1, min(WAVES, (c.full + 63) / 64));
    const float bound = wave < busy ? nth_of_lanes(own, (n + busy - 1) / busy) : INFINITY;
    if (lane == 0) red[3][wave] = bound;
  }
  __syncthreads();
  float M = red[0][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) M = fmaxf(M, red[0][w]);
  {
    // `off` out of both sums (by division, so that a term of 1 is exactly that)
    const float one = __builtin_amdgcn_exp2f(off);
    along = fmaf(-off, sum, along) / one;
    sum /= one;
    const float by = m == M ? 0.f : (m - M) * scale;      // (both -infinity: nothing to shift)
    const float f = __builtin_amdgcn_exp2f(by);
    along = f > 0.f ? fmaf(sum, by, along) * f : 0.f;
    sum *= f;
  }
  {
    const float wave_sum = lanes_sum(sum), wave_along = lanes_sum(along);
    if (lane == 0) { red[1][wave] = wave_sum; red[2][wave] = wave_along; }
  }
  float least = -INFINITY;
  if constexpr (TOP) {
    // every busy wave has its share of n values that are not below the smallest of their bounds
    least = red[3][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) least = fminf(least, red[3][w]);
    if (!ONE && steps <= steps_kept && own >= least) note_hits(kept, steps, T, [&](float v) { return v >= least; }, found);
  }
  __syncthreads();
  Sums all = {M, 0.f, 0.f, 0.f};
  auto add_waves = [&]() {
    all.sum = all.along = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { all.sum += red[1][w]; all.along += red[2][w]; }
  };
  add_waves();
  if (all.sum < 2.f && all.sum >= 1.f) {
    // One value has more than half of the probability: the lane that has it added up small terms beside 1, in a step 32 and then the steps, each off by 2^-24
    // at most.  Some 40 of them are 2e-7 as a rule and 2.4e-6 at worst, of a log S that may be as small; from S = 2 on, log S is 0.69 and there may be two such
    // values.  The wave goes over that lane's values again, a piece to a lane, without the largest (the block comes here as one, and so does the wave).
    __syncthreads();
    const unsigned long long which = __ballot(own == M);
    if (which) {
      const int from = __ffsll((long long)which) - 1, thread = wave * 64 + from;
      if (lane == from) sum = along = 0.f;
      auto again = [&](float v) {
        const float y = (v - M) * scale, e = v == M ? 0.f : __builtin_amdgcn_exp2f(y);
        sum += e;
        along = fmaf(e, fmaxf(y, LOWEST), along);
      };
      for (int k = lane * T + thread; k < c.full; k += 64 * T) {
        const Some<E> s = Some<E>::load(z, c.first + (long long)k * N);
#pragma unroll
        for (int e = 0; e < N; ++e) again(s[e]);
      }
      if (lane == from) again(at_edge);
      const float wave_sum = lanes_sum(sum), wave_along = lanes_sum(along);
      if (lane == 0) { red[1][wave] = wave_sum; red[2][wave] = wave_along; }
    }
    __syncthreads();
    add_waves();
    all.count = 1.f;
  }
  if (parts > 1) {
    if (threadIdx.x == 0) {
      float4* to = a.partial + 2 * ((long long)row * parts + part);
      to[0] = make_float4(M, all.count, all.sum, all.along);
      to[1] = make_float4(z_token, 0.f, 0.f, 0.f);
    }
  } else if (threadIdx.x == 0) {
    finish(a, row, all, z_token);
  }
  if constexpr (TOP) {
    const bool known = all.sum == all.sum && steps <= steps_kept;          // (NaN, or an infinity, which makes one: the maxima passed over it)
    int hits = found.hits;
    const bool crowded = hits > HITS;
    if (crowded && known) {
      // many values equal to the bound, masked ones as a rule: the values above it alone
      __syncthreads();
      if (threadIdx.x == 0) found.hits = 0;
      __syncthreads();
      note_hits(kept, steps, T, [&](float v) { return v > least; }, found);
      __syncthreads();
      hits = found.hits;
    }
    const bool simple = known && hits <= HITS;
    if (simple) {
      auto take = [&](float v, int at) {
        if (v > least) {
          const int i = atomicAdd(&found.above, 1);
          if (i < CANDIDATES) found.key[i] = key_of(order_of(v), at);
        } else if (v == least && !crowded && found.equal <= EQUALS) {
          const int i = atomicAdd(&found.equal, 1);
          if (i < EQUALS) found.same[i] = key_of(order_of(v), at);
        }
      };
      if (edge >= 0) take(at_edge, edge);
      if constexpr (ONE) {
        if (own >= least)
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e)
              if (s0[u][e] >= least && u * T + (int)threadIdx.x < c.full) take(s0[u][e], c.first + (u * T + (int)threadIdx.x) * N + e);
      } else {
        // a thread to every value of the steps noted, eight of them requested at once
        constexpr int B = 8;
        const int values = hits * U * N;
        for (int i0 = threadIdx.x; i0 < values; i0 += T * B) {
          float v[B];
          int at[B];
#pragma unroll
          for (int b = 0; b < B; ++b) {
            const int i = min(i0 + b * T, values - 1);
            const uint32_t hit = found.hit[i / (U * N)];
            const int k = ((int)(hit / T) * U + i % (U * N) / N) * T + (int)(hit % T);
            at[b] = i == i0 + b * T && k < c.full ? c.first + k * N + i % N : -1;
            v[b] = Some<E>::one(z, at[b] >= 0 ? at[b] : 0);
          }
#pragma unroll
          for (int b = 0; b < B; ++b)
            if (at[b] >= 0) take(v[b], at[b]);
        }
      }
      __syncthreads();
    }
    const int above = found.above, equal = found.equal;
    int have = n;
    if (!simple || above > CANDIDATES) {
      select_top<E, T>(z, c, a.vocab, n, found);
    } else if (above >= n) {
      have = above;
    } else if (!crowded && equal <= EQUALS && above + equal <= CANDIDATES) {
      have = above + equal;
      for (int i = threadIdx.x; i < equal; i += T) found.key[above + i] = found.same[i];
      __syncthreads();
    } else {
      fill_equal<E, T>(z, c, a.vocab, n, order_of(least), above, found);
    }
    if (parts > 1) {
      uint64_t* keys = a.part_keys + ((long long)row * parts + part) * a.n_top;
      rank_keys(found.key, have, n, T, [&](uint64_t key, int rank) { keys[rank] = key; });
      for (int i = n + threadIdx.x; i < a.n_top; i += T) keys[i] = 0;        // (below every value's)
    } else {
      const Likely l = likely_of(all, a.temperature);
      rank_keys(found.key, have, n, T, [&](uint64_t key, int rank) { l.put(a, row, rank, key); });
    }
  }
}

// A parted row's numbers and likeliest tokens from those of its parts, in their order.  One block to a row.
constexpr int MOST_PARTS = 8;
__global__ __launch_bounds__(256) void token_logprobs_join_kernel(LogprobArgs a, int parts) {
  __shared__ uint64_t keys[MOST_PARTS * MOST_TOP];
  __shared__ int found;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int token = a.tokens ? a.tokens[row] : 0;
  if (a.tokens && (token < 0 || token >= a.vocab)) {
    leave_out<true>(a, row);
    return;
  }
  if (threadIdx.x == 0) found = 0;
  const bool on = lane < parts;
  const float4* of = a.partial + 2 * ((long long)row * parts + lane);
  const float4 p = on ? of[0] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const float z_token = on ? of[1].x : 0.f;
  const int share = (a.n_top + parts - 1) / parts;
  const uint64_t* from = a.part_keys + (long long)row * parts * a.n_top;
  // every part has `share` values that are not below the smallest of the parts' bounds
  uint64_t bound = a.n_top > 0 && on ? from[lane * a.n_top + share - 1] : ~0ull;
#pragma unroll
  for (int o = 1; o < MOST_PARTS; o <<= 1) {
    const uint64_t other = ((uint64_t)(uint32_t)__shfl_xor((int)(bound >> 32), o, WAVE) << 32) | (uint32_t)__shfl_xor((int)bound, o, WAVE);
    bound = other < bound ? other : bound;
  }
  bound = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(bound >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)bound);
  const float M = lanes_max(p.x), scale = LOG2E / a.temperature;
  float count = p.y, sum = p.z, along = p.w;
  if (p.x != M) {
    const float by = (p.x - M) * scale, f = __builtin_amdgcn_exp2f(by);
    sum += count;
    count = 0.f;
    along = f > 0.f ? fmaf(sum, by, along) * f : 0.f;
    sum *= f;
  }
  const Sums all = {M, lanes_sum(count), lanes_sum(sum), lanes_sum(along)};
  if (threadIdx.x == 0) finish(a, row, all, z_token);
  if (a.n_top == 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < parts * a.n_top; i += 256) {
    const uint64_t key = from[i];
    if (key >= bound && key != 0) keys[atomicAdd(&found, 1)] = key;
  }
  __syncthreads();
  const Likely l = likely_of(all, a.temperature);
  rank_keys(keys, found, a.n_top, 256, [&](uint64_t key, int rank) { l.put(a, row, rank, key); });
}

// Gradient: every value read once and written once, by the same thread, so that the gradient may take the logits' place.  Bound by HBM.
constexpr int GU = 4;
template <class E, int GT, bool ONCE>
__global__ __launch_bounds__(GT) void token_logprobs_backward_kernel(LogprobArgs a, int parts) {
  constexpr int N = Some<E>::N;
  const int row = blockIdx.x / parts, part = blockIdx.x % parts;
  const void* z = row_at<E>(a.logits, row, a.stride);
  void* dz = const_cast<void*>(row_at<E>(a.dlogits, row, a.d_stride));
  const int token = a.tokens ? a.tokens[row] : -1;
  const float m = a.stats[2ll * row], log_sum = a.stats[2ll * row + 1];
  const bool none = (a.tokens && (token < 0 || token >= a.vocab)) || (m == -INFINITY && log_sum == -INFINITY);
  const float g = a.g ? a.g[row] : 0.f, h = a.g_entropy ? a.g_entropy[row] : 0.f, H = h != 0.f ? a.entropy[row] : 0.f;
  const float inv_t = 1.0f / a.temperature;
  auto grad = [&](float v) {
    const float lp = (v - m) * inv_t - log_sum, p = __builtin_amdgcn_exp2f(lp * LOG2E);
    // (masked: p is 0 and its logarithm infinite)
    return -p * fmaf(h, fmaxf(lp, -1000.f) + H, g) * inv_t;
  };
  // the token's own: g (1 - p) from the logarithm, as the difference would keep few bits where p is near 1
  auto grad_token = [&](float v) {
    const float lp = (v - m) * inv_t - log_sum, p = __builtin_amdgcn_exp2f(lp * LOG2E);
    return fmaf(g, -expm1f(lp), -p * h * (fmaxf(lp, -1000.f) + H)) * inv_t;
  };
  const Cut c = cut_row<E>(z, a.vocab);
  if (part == 0) {
    const int edge = edge_of(c, a.vocab);
    if (edge >= 0) {
      const float v = Some<E>::one(z, edge);
      Some<E>::store_one(dz, edge, none ? 0.f : edge == token ? grad_token(v) : grad(v));
    }
  }
  // the thread that has the token's piece reads its logit ahead and writes its gradient over the piece's
  const int k_token = token >= c.first && token < c.first + c.full * N ? (token - c.first) / N : -1;
  const bool own = !none && k_token >= 0 && k_token / (GT * GU) % parts == part && k_token % GT == (int)threadIdx.x;
  const float at_token = own ? Some<E>::one(z, token) : 0.f;
  for (int k0 = part * GT * GU; k0 < c.full; k0 += parts * GT * GU) {
    Some<E> s[GU];
#pragma unroll
    for (int u = 0; u < GU; ++u) {
      const int k = k0 + u * GT + threadIdx.x;
      if (k < c.full && !none) s[u] = Some<E>::template load<ONCE>(z, c.first + (long long)k * N);
    }
#pragma unroll
    for (int u = 0; u < GU; ++u) {
      const int k = k0 + u * GT + threadIdx.x;
      if (k >= c.full) continue;
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = none ? 0.f : grad(s[u][e]);
      Some<E>::template store<ONCE>(dz, c.first + (long long)k * N, y);
    }
  }
  if (own) Some<E>::store_one(dz, token, grad_token(at_token));
}

// Threads to a block and blocks to a row.  Four waves to a row; one where that holds the whole row in a step and rows are many (8192 rows of 1000 bf16 values,
// us: 8.6 and 25 without alternatives, 17 and 35 with five, 33 and 48 with 32, but 145 and 69 with 64).  Few long rows are parted (100000 fp16
// values without and with 20 alternatives, us: 16 rows 6.7 and 12.9 in eight parts, 7.8 and 14.7 in four, 10.3 and 16.2 whole; 64 rows 8.2 and 15.2,
// 8.2 and 14.4, 10.4 and 16.5; 200 rows 15.3 and 23.9, 16.0 and 22.3, 12.2 and 18.4; of 66000 values 16 rows with 20 alternatives 12.0 in eight,
// 12.9 whole; one row of 50304 with five 9.0 in eight, 9.4 whole and without a workspace).  More waves to a row gain nothing (256 rows of
// 100000: 12.8 with four, 13.2 with eight, 15.2 with sixteen).
struct Shape { int threads, parts; };
Shape shape_of(const LogprobArgs& a) {
  if (a.vocab <= 64 * 32 && a.rows > 256 && a.n_top <= 32) return {64, 1};
  return {256, a.vocab < 65536 || a.rows > 64 ? 1 : a.rows > 16 ? 4 : 8};
}
// Of rows past the caches (8192 of 128256 bf16 values, a quarter left out: 243 us, 279 without; backward 644 and 667)
bool past_caches(const LogprobArgs& a, int times) { return (double)times * a.rows * a.vocab * (a.dtype == RLGEN_DTYPE_F32 ? 4 : 2) > CACHE_BYTES; }
template <class E, int T, bool ONE, bool ONCE> hipError_t launch_forward(const LogprobArgs& a, int parts, hipStream_t s) {
  constexpr int N = Some<E>::N, U = 32 / N;
  const dim3 grid((unsigned)(a.rows * parts)), block(T);
  if (a.n_top == 0) {
    hipLaunchKernelGGL((token_logprobs_kernel<E, T, false, ONE, ONCE>), grid, block, 0, s, a, 0, parts);
  } else {
    // 48 KB of maxima at most: rows or parts up to 393216 values, beyond them the likeliest tokens are searched by counting
    const int steps = ((a.vocab / N + parts - 1) / parts + T * U - 1) / (T * U), kept = ONE ? 1 : steps <= 12288 / T ? steps : 0;
    hipLaunchKernelGGL((token_logprobs_kernel<E, T, true, ONE, ONCE>), grid, block, ONE ? 0 : kept * T * sizeof(float), s, a, kept, parts);
  }
  if (parts > 1) hipLaunchKernelGGL(token_logprobs_join_kernel, dim3(a.rows), dim3(256), 0, s, a, parts);
  return hipGetLastError();
}
template <class E> hipError_t by_rows(const LogprobArgs& a, hipStream_t s) {
  const Shape f = shape_of(a);
  if (f.threads == 64) return launch_forward<E, 64, true, false>(a, f.parts, s);
  if (a.vocab <= 256 * 32) return launch_forward<E, 256, true, false>(a, f.parts, s);
  return past_caches(a, 1) ? launch_forward<E, 256, false, true>(a, f.parts, s) : launch_forward<E, 256, false, false>(a, f.parts, s);
}
// Backward: one wave to a row that it holds in a step (8192 rows of 1000 bf16 values: 9.5 us, 12.9 with four), else four to 1024 pieces
bool short_row(const LogprobArgs& a) { return a.vocab <= 64 * GU * (a.dtype == RLGEN_DTYPE_F32 ? 4 : 8); }
int parts_of(const LogprobArgs& a) {
  const int step = 256 * GU * (a.dtype == RLGEN_DTYPE_F32 ? 4 : 8);
  return (a.vocab + step - 1) / step;
}
template <class E> hipError_t launch_backward(const LogprobArgs& a, hipStream_t s) {
  const int parts = parts_of(a);
  if (short_row(a)) hipLaunchKernelGGL((token_logprobs_backward_kernel<E, 64, false>), dim3((unsigned)a.rows), dim3(64), 0, s, a, 1);
  else if (past_caches(a, 2)) hipLaunchKernelGGL((token_logprobs_backward_kernel<E, 256, true>), dim3((unsigned)(a.rows * parts)), dim3(256), 0, s, a, parts);
  else hipLaunchKernelGGL((token_logprobs_backward_kernel<E, 256, false>), dim3((unsigned)(a.rows * parts)), dim3(256), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace

size_t rl_token_logprobs_bytes(const LogprobArgs& a) {
  const Shape f = shape_of(a);
  return f.parts == 1 ? 0 : (size_t)a.rows * f.parts * (2 * sizeof(float4) + a.n_top * sizeof(uint64_t));
}
hipError_t rl_token_logprobs(LogprobArgs a, void* workspace, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  a.partial = (float4*)workspace;
  a.part_keys = (uint64_t*)(a.partial + 2 * (size_t)a.rows * shape_of(a).parts);
  switch (a.dtype) {
    case RLGEN_DTYPE_F32: return by_rows<TypeF32>(a, s);
    case RLGEN_DTYPE_BF16: return by_rows<TypeBf16>(a, s);
    case RLGEN_DTYPE_F16: return by_rows<TypeF16>(a, s);
    default: return hipErrorInvalidValue;
  }
}
long long rl_token_logprobs_backward_blocks(const LogprobArgs& a) { return (long long)a.rows * parts_of(a); }
hipError_t rl_token_logprobs_backward(const LogprobArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  switch (a.dtype) {
    case RLGEN_DTYPE_F32: return launch_backward<TypeF32>(a, s);
    case RLGEN_DTYPE_BF16: return launch_backward<TypeBf16>(a, s);
    case RLGEN_DTYPE_F16: return launch_backward<TypeF16>(a, s);
    default: return hipErrorInvalidValue;
  }
}
