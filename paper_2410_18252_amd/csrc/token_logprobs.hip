// Log-probs of given tokens, entropy and the n likeliest tokens of rows of logits, in one pass over them, and the gradient of the first two.
//   m = max z, S = sum exp((z - m) / T), log p_j = (z_j - m) / T - log S, H = log S - sum p_j (z_j - m) / T
//   dz_j = (g (1[j = t] - p_j) - h p_j (log p_j + H)) / T
#include "learner.h"
#include "../../include/rlgen.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.4028234663852886e38f;

// 16 bytes of a row's logits
template <class E> struct Some {
  static constexpr int N = 8;
  u32x4 w;
  static __device__ __forceinline__ Some load(const void* row, long long at) { return {*(const u32x4*)((const uint16_t*)row + at)}; }
  __device__ __forceinline__ float operator[](int e) const { return e & 1 ? E::high(w[e >> 1]) : E::low(w[e >> 1]); }
  static __device__ __forceinline__ float one(const void* row, long long at) { return E::low(((const uint16_t*)row)[at]); }
  static __device__ __forceinline__ void store(void* row, long long at, const float* y) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = E::pack(y[2 * e], y[2 * e + 1]);
    *(u32x4*)((uint16_t*)row + at) = w;
  }
  static __device__ __forceinline__ void store_one(void* row, long long at, float y) { ((uint16_t*)row)[at] = (uint16_t)E::pack(y, 0.f); }
};
template <> struct Some<TypeF32> {
  static constexpr int N = 4;
  f32x4 w;
  static __device__ __forceinline__ Some load(const void* row, long long at) { return {*(const f32x4*)((const float*)row + at)}; }
  __device__ __forceinline__ float operator[](int e) const { return w[e]; }
  static __device__ __forceinline__ float one(const void* row, long long at) { return ((const float*)row)[at]; }
  static __device__ __forceinline__ void store(void* row, long long at, const float* y) { *(f32x4*)((float*)row + at) = f32x4{y[0], y[1], y[2], y[3]}; }
  static __device__ __forceinline__ void store_one(void* row, long long at, float y) { ((float*)row)[at] = y; }
};
template <class E> constexpr int SIZE = 16 / Some<E>::N;

// A row may start anywhere: `head` elements up to the first 16-byte border, then `full` pieces of 16 bytes, then `tail` elements
struct Cut { int head, full, tail; };
template <class E> __device__ __forceinline__ Cut cut_row(const void* row, int vocab) {
  constexpr int N = Some<E>::N;
  const int lead = (int)((uintptr_t)row & 15) / SIZE<E>;
  Cut c;
  c.head = lead ? min(N - lead, vocab) : 0;
  c.full = (vocab - c.head) / N;
  c.tail = vocab - c.head - c.full * N;
  return c;
}
template <class E> __device__ __forceinline__ const void* row_at(const void* p, long long row, long long stride) {
  return (const char*)p + row * stride * SIZE<E>;
}
// the element of the head or the tail that this thread has, -1: none
__device__ __forceinline__ int edge_of(const Cut& c, int n, int vocab) {
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

template <int T> __device__ __forceinline__ float over_block(float v, float* slots, bool max) {
  v = max ? wave_max(v) : wave_sum(v);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = slots[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) t = max ? fmaxf(t, slots[w]) : t + slots[w];
  return t;
}
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
// the wave's values in descending order over its lanes
__device__ __forceinline__ float sorted_wave(float v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const float o = __shfl_xor(v, j, WAVE);
      v = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(v, o) : fminf(v, o);
    }
  return v;
}

constexpr int CANDIDATES = 256;

// What the likeliest tokens' search holds in LDS
struct Found {
  uint64_t key[CANDIDATES];
  float slots[16];
  int counts[16];
  int n;
};

// The n largest of a row whose values do not thin out above any simple bound (many equal ones, NaN): the n-th largest order by
// halving, every step counting over the row, then the values above it, and of those equal to it the first ones.
template <class E, int T> __device__ void select_top(const void* row, const Cut& c, int vocab, int n, Found& f) {
  constexpr int N = Some<E>::N;
  const int edge = edge_of(c, N, vocab);
  auto each = [&](auto&& use) {
    for (int k = threadIdx.x; k < c.full; k += T) {
      const Some<E> s = Some<E>::load(row, c.head + (long long)k * N);
#pragma unroll
      for (int e = 0; e < N; ++e) use(order_of(s[e]), c.head + k * N + e);
    }
    if (edge >= 0) use(order_of(Some<E>::one(row, edge)), edge);
  };
  uint32_t least = 0;                              // the n-th largest order
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t trial = least | (1u << bit);
    int mine = 0;
    each([&](uint32_t o, int) { mine += o >= trial; });
    if (count_block<T>(mine, f.counts) >= n) least = trial;
  }
  __syncthreads();
  if (threadIdx.x == 0) f.n = 0;
  __syncthreads();
  each([&](uint32_t o, int at) {
    if (o > least) f.key[atomicAdd(&f.n, 1)] = key_of(o, at);     // (fewer than n of them)
  });
  __syncthreads();
  int have = f.n;
  // equal ones in the order of their indices: the head, the pieces, the tail
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
        const Some<E> s = Some<E>::load(row, c.head + (long long)k * N);
        first = c.head + k * N;
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
  if (threadIdx.x == 0) f.n = n;
  __syncthreads();
}

// One block to a row, one pass.  Every lane sums exp((z - m) / T) relative to the largest value m that its wave has met, which rises a few
// times a row; the entropy's sum goes along.  The likeliest tokens cost the pass a maximum per thread and step, kept in LDS: n of the
// lanes' maxima bound the n-th largest from below so closely that little more than n values lie above, and only the steps that hold one
// are read again.  Bound by HBM.
template <class E, int T, bool TOP>
__global__ __launch_bounds__(T) void token_logprobs_kernel(LogprobArgs a, int steps_kept) {
  constexpr int N = Some<E>::N, U = 32 / N, WAVES = T / 64;
  extern __shared__ float kept[];                // [steps][T]: the largest value of a thread's step
  __shared__ float red[4][WAVES];
  __shared__ Found found;
  const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int token = a.tokens ? a.tokens[row] : 0;
  if (a.tokens && (token < 0 || token >= a.vocab)) {          // not asked for
    if (threadIdx.x == 0) {
      if (a.logprobs) a.logprobs[row] = 0.f;
      a.stats[2ll * row] = a.stats[2ll * row + 1] = 0.f;
      if (a.entropy) a.entropy[row] = 0.f;
    }
    if (TOP && (int)threadIdx.x < a.n_top) {
      a.top_tokens[(long long)row * a.n_top + threadIdx.x] = -1;
      a.top_logprobs[(long long)row * a.n_top + threadIdx.x] = -INFINITY;
    }
    return;
  }
  const void* z = row_at<E>(a.logits, row, a.stride);
  const Cut c = cut_row<E>(z, a.vocab);
  const float scale = LOG2E / a.temperature;
  const int steps = (c.full + T * U - 1) / (T * U);
  float m = -INFINITY, own = -INFINITY, sum = 0.f, along = 0.f;   // m: of the wave, own: of this lane
  auto rise = [&](float most) {                                   // m to the largest of the lanes'
    if (!__any(most > m)) return;
    const float up = wave_max(fmaxf(most, m));
    if (m == -INFINITY) {
      // (nothing but NaN so far)
      along = 0.f;
    } else {
      const float by = m - up, f = __builtin_amdgcn_exp2f(by * scale);
      along = f > 0.f ? fmaf(sum, by, along) * f : 0.f;         // (by may be the lowest value, the sum of it infinite)
      sum *= f;
    }
    m = up;
  };
  auto add = [&](float v, float base) {
    const float x = v - base, e = __builtin_amdgcn_exp2f(x * scale);
    sum += e;
    along = fmaf(e, fmaxf(x, LOWEST), along);    // (a masked value counts 0, not 0 times infinity)
  };
  const int edge = edge_of(c, N, a.vocab);
  const float at_edge = edge >= 0 ? Some<E>::one(z, edge) : -INFINITY;
  own = at_edge;
  rise(at_edge);
  add(at_edge, m == -INFINITY ? 0.f : m);
  for (int step = 0; step < steps; ++step) {
    Some<E> s[U];
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (step * U + u) * T + threadIdx.x;
      if (k < c.full) s[u] = Some<E>::load(z, c.head + (long long)k * N);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((step * U + u) * T + (int)threadIdx.x < c.full)
#pragma unroll
        for (int e = 0; e < N; ++e) most = fmaxf(most, s[u][e]);
    rise(most);
    if (TOP) {
      own = fmaxf(own, most);
      if (step < steps_kept) kept[step * T + threadIdx.x] = most;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((step * U + u) * T + (int)threadIdx.x < c.full)
#pragma unroll
        for (int e = 0; e < N; ++e) add(s[u][e], base);
  }
  // over the block
  if (lane == 0) red[0][wave] = m;
  __syncthreads();
  float M = red[0][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) M = fmaxf(M, red[0][w]);
  {
    const float by = m == M ? 0.f : m - M;       // (both -infinity: nothing to shift)
    const float f = __builtin_amdgcn_exp2f(by * scale);
    along = f > 0.f ? fmaf(sum, by, along) * f : 0.f;
    sum *= f;
  }
  sum = wave_sum(sum);
  along = wave_sum(along);
  if (lane == 0) { red[1][wave] = sum; red[2][wave] = along; }
  __syncthreads();
  sum = along = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { sum += red[1][w]; along += red[2][w]; }
  const bool empty = M == -INFINITY && sum == 0.f;
  const float log_sum = logf(sum);               // (-infinity for a row that is masked as a whole)
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[row] = empty ? -INFINITY : (Some<E>::one(z, token) - M) / a.temperature - log_sum;
    a.stats[2ll * row] = M;
    a.stats[2ll * row + 1] = log_sum;
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_sum - along / sum / a.temperature;
  }
  if constexpr (TOP) {
    const int n = a.n_top, per = (n + WAVES - 1) / WAVES;
    const float bound = __shfl(sorted_wave(own), per - 1, WAVE);
    if (lane == 0) red[3][wave] = bound;
    if (threadIdx.x == 0) found.n = 0;
    __syncthreads();
    float least = red[3][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) least = fminf(least, red[3][w]);
    // NaN (or an infinity, which makes one) in the sum: the maxima passed over it
    bool plain = sum == sum && steps <= steps_kept;
    if (plain) {
      auto take = [&](float v, int at) {
        if (v >= least) {
          const int i = atomicAdd(&found.n, 1);
          if (i < CANDIDATES) found.key[i] = key_of(order_of(v), at);
        }
      };
      if (least == -INFINITY && a.vocab > CANDIDATES) {
        plain = false;
      } else if (own >= least) {
        if (edge >= 0) take(at_edge, edge);
        for (int step = 0; step < steps; ++step) {
          if (!(kept[step * T + threadIdx.x] >= least)) continue;
          for (int u = 0; u < U; ++u) {
            const int k = (step * U + u) * T + threadIdx.x;
            if (k >= c.full) break;
            const Some<E> s = Some<E>::load(z, c.head + (long long)k * N);
#pragma unroll
            for (int e = 0; e < N; ++e) take(s[e], c.head + k * N + e);
          }
        }
      }
      __syncthreads();
      plain = plain && found.n <= CANDIDATES;
    }
    if (!plain) select_top<E, T>(z, c, a.vocab, n, found);
    const int have = found.n;
    for (int i = threadIdx.x; i < have; i += T) {
      const uint64_t key = found.key[i];
      int rank = 0;
      for (int j = 0; j < have; ++j) rank += found.key[j] > key;
      if (rank >= n) continue;
      const long long at = (long long)row * n + rank;
      a.top_tokens[at] = (int)(0xffffffffu - (uint32_t)key);
      a.top_logprobs[at] = empty ? -INFINITY : (value_of((uint32_t)(key >> 32)) - M) / a.temperature - log_sum;
    }
  }
}

// Gradient: every value read once and written once, by the same thread, so that the gradient may take the logits' place.  Bound by HBM.
constexpr int GT = 256, GU = 4;
template <class E>
__global__ __launch_bounds__(GT) void token_logprobs_backward_kernel(LogprobArgs a, int parts) {
  constexpr int N = Some<E>::N;
  const int row = blockIdx.x / parts, part = blockIdx.x % parts;
  const void* z = row_at<E>(a.logits, row, a.stride);
  void* dz = const_cast<void*>(row_at<E>(a.dlogits, row, a.d_stride));
  const int token = a.tokens ? a.tokens[row] : -1;
  const float m = a.stats[2ll * row], log_sum = a.stats[2ll * row + 1];
  const bool none = (a.tokens && (token < 0 || token >= a.vocab)) || m == -INFINITY;
  const float g = a.g ? a.g[row] : 0.f, h = a.g_entropy ? a.g_entropy[row] : 0.f, H = h != 0.f ? a.entropy[row] : 0.f;
  const float inv_t = 1.0f / a.temperature;
  auto grad = [&](float v, int at) {
    const float lp = (v - m) * inv_t - log_sum, p = __builtin_amdgcn_exp2f(lp * LOG2E);
    // (masked: p is 0 and its logarithm infinite)
    float d = -p * fmaf(h, fmaxf(lp, -1000.f) + H, g);
    if (at == token) d += g;
    return none ? 0.f : d * inv_t;
  };
  const Cut c = cut_row<E>(z, a.vocab);
  if ((((uintptr_t)z ^ (uintptr_t)dz) & 15) != 0) {
    // the two rows start differently within 16 bytes
    for (int i = part * GT + threadIdx.x; i < a.vocab; i += parts * GT) Some<E>::store_one(dz, i, grad(Some<E>::one(z, i), i));
    return;
  }
  if (part == 0) {
    const int edge = edge_of(c, N, a.vocab);
    if (edge >= 0) Some<E>::store_one(dz, edge, grad(Some<E>::one(z, edge), edge));
  }
  for (int k0 = part * GT * GU; k0 < c.full; k0 += parts * GT * GU) {
    Some<E> s[GU];
#pragma unroll
    for (int u = 0; u < GU; ++u) {
      const int k = k0 + u * GT + threadIdx.x;
      if (k < c.full && !none) s[u] = Some<E>::load(z, c.head + (long long)k * N);
    }
#pragma unroll
    for (int u = 0; u < GU; ++u) {
      const int k = k0 + u * GT + threadIdx.x;
      if (k >= c.full) continue;
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = none ? 0.f : grad(s[u][e], c.head + k * N + e);
      Some<E>::store(dz, c.head + (long long)k * N, y);
    }
  }
}

template <class E, int T> hipError_t launch_forward(const LogprobArgs& a, hipStream_t s) {
  constexpr int U = 32 / Some<E>::N;
  const dim3 grid(a.rows), block(T);
  if (a.n_top == 0) {
    hipLaunchKernelGGL((token_logprobs_kernel<E, T, false>), grid, block, 0, s, a, 0);
  } else {
    // 48 KB of maxima at most: vocabularies up to 393216, beyond them the likeliest tokens are searched by counting
    const int steps = (a.vocab / Some<E>::N + T * U - 1) / (T * U), kept = steps <= 12288 / T ? steps : 0;
    hipLaunchKernelGGL((token_logprobs_kernel<E, T, true>), grid, block, kept * T * sizeof(float), s, a, kept);
  }
  return hipGetLastError();
}
template <class E> hipError_t by_rows(const LogprobArgs& a, hipStream_t s) {
  return a.rows <= 256 ? launch_forward<E, 1024>(a, s) : launch_forward<E, 256>(a, s);
}
int parts_of(const LogprobArgs& a) {
  const int n = a.dtype == RLGEN_DTYPE_F32 ? 4 : 8;
  return (int)(((long long)a.vocab + n * GT * GU - 1) / (n * GT * GU));
}
template <class E> hipError_t launch_backward(const LogprobArgs& a, hipStream_t s) {
  const int parts = parts_of(a);
  hipLaunchKernelGGL((token_logprobs_backward_kernel<E>), dim3((unsigned)(a.rows * parts)), dim3(GT), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace

hipError_t rl_token_logprobs(const LogprobArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
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
