// Gradients of the windowed attention over packed rows.
//
// With P = exp(scale q k - lse), dP = dout v, delta = sum over dims of dout out and dS = P (dP - delta):
//   dv = sum over queries of P dout,   dk = scale sum over queries of dS q,   dq = scale sum over keys of dS k
// P is computed again from the saved log-sum-exp, once in a kernel whose blocks own keys and once in one whose blocks own queries:
// seven matrix products instead of the five that one kernel with atomic sums would need, but every sum has one order, so that results do
// not change from run to run.  P and dS are rounded to the inputs' type for their second products, errors of the order of the
// gradients' own rounding; fp16, whose smallest normal number a dS easily falls below, multiplies dS by a power of two taken from the
// largest |dout| and |v| that enter the sum: of the row and of the keys in its sight for dq, of the queries walked and of the keys in theirs for dk.
//
// The queries' side goes first, since it corrects delta for the rows that see few keys; its walk is the forward pass's.  Both sides are bound
// by their chains of products, exponentials and barriers with two or three waves to a SIMD (matrix unit 43 and 31 % busy at 128 dims),
// not by memory.  Measured: 8250 rows, 32 heads over 8 of 128, window 1024: delta 22 us, queries' side 187, keys' side 311, sums of the
// sinks' parts 5 (0.30 TFLOP without the products that are computed twice; 182 to 209 and 302 to 368 us on other cards); 9985 rows, 32 heads of
// 80 in fp16: 32, 104 and 150 us.
#include "../../include/rlgen.h"
#include "window_tiles.h"
#include <type_traits>

namespace {

constexpr int TPB = 256, BM = 128;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int FEW_KEYS = 32, FEW_ROWS = 64;
// fp16 takes every P times 2^15 (P is at most 1 but for roundings, so that stays in its range): a P down to 2^-29 is then a normal number, where
// beside one dominant key or among tens of thousands of keys it would lose its bits below 2^-14.  The shift is part of the exponent.
template <class T> constexpr float P_SHIFT = __is_same(T, TypeF16) ? 15.f : 0.f;
template <class T> constexpr float P_SIZE = __is_same(T, TypeF16) ? 32768.f : 1.f;

// Whether all rows of a sequence of n see few keys: a rule on the sequence alone, so that its gradients' precision is its own in any call
__device__ __forceinline__ bool sees_few(const WindowArgs& a, int n) { return (a.window > 0 && a.window <= FEW_KEYS) || n <= FEW_ROWS; }

// What a pair loses when it is rounded to the word that it was packed into, as such a word
template <class T> __device__ __forceinline__ uint32_t rest_of(float lo, float hi, uint32_t word) { return T::pack(lo - T::low(word), hi - T::high(word)); }

// Everything below in the caller's workspace, and how the queries that see the sinks from beyond the window are parted.
struct Backward {
  WindowArgs a;
  float *lse2, *delta, *part;           // [rows, Hq]: lse log2 e less P's shift, delta; the sinks' parts
  float *dout_peak, *v_peak;            // [S, delta_chunks]: the largest finite |dout| and |v| of delta_tokens tokens (fp16)
  int sinks, chunk, chunks;             // sinks that are parted (0: none); tokens to a part; parts of the longest sequence
  float* run_part;                      // [runs, rows, Hkv, 2, h]
  int delta_tokens, delta_chunks;       // tokens to a block of delta_kernel, blocks to the longest sequence
  int run, runs;                        // tokens to a part of what a tile of keys is seen by, most parts (1: not parted)
};

// delta and lse log2 e (less P's shift) of a sequence's tokens, delta_tokens of them to a block, and in fp16 the largest finite |dout| and |v| among them.
// Bound by HBM: out and dout (and v) once.
template <class T, int CH>
__global__ __launch_bounds__(TPB) void delta_kernel(Backward b) {
  __shared__ float red[2][4];
  const WindowArgs& a = b.a;
  constexpr int AHEAD = 4 / CH;                // (token, head) pairs requested before the first is used
  const int s = blockIdx.x / b.delta_chunks, tok0 = (blockIdx.x - s * b.delta_chunks) * b.delta_tokens, li = threadIdx.x & 15;
  const Seq q = load_seq(a, s, false);
  const int tokens = min(b.delta_tokens, q.n - tok0);
  if (tokens <= 0) return;
  const int items = tokens * a.Hq;
  const long long row0 = q.row0 + tok0;
  float peak[2] = {0.f, 0.f};
  auto finite_peak = [&](float& p, uint32_t w) {
    const float lo = fabsf(T::low(w)), hi = fabsf(T::high(w));
    p = fmaxf(p, fmaxf(lo < INFINITY ? lo : 0.f, hi < INFINITY ? hi : 0.f));
  };
  for (int it0 = threadIdx.x >> 4; it0 < items; it0 += 16 * AHEAD) {
    u32x4 o[AHEAD][CH], g[AHEAD][CH];
    float lse[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int it = it0 + 16 * u < items ? it0 + 16 * u : it0, tok = it / a.Hq;
      const long long row = row0 + tok, head = (long long)(it - tok * a.Hq) * a.h;
      lse[u] = a.lse[row0 * a.Hq + it];
#pragma unroll
      for (int x = 0; x < CH; ++x) {
        const int d = 128 * x + 8 * li;
        o[u][x] = d < a.h ? *(const u32x4*)((const uint16_t*)a.o + row * a.o_stride + head + d) : u32x4{0, 0, 0, 0};
        g[u][x] = d < a.h ? *(const u32x4*)((const uint16_t*)a.dout + row * a.dout_stride + head + d) : u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      float v = 0.f;
#pragma unroll
      for (int x = 0; x < CH; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v = fmaf(T::low(o[u][x][e]), T::low(g[u][x][e]), v);
          v = fmaf(T::high(o[u][x][e]), T::high(g[u][x][e]), v);
          if constexpr (__is_same(T, TypeF16)) finite_peak(peak[0], g[u][x][e]);
        }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
      const int it = it0 + 16 * u;
      if (li == 0 && it < items) {
        b.delta[row0 * a.Hq + it] = v;
        b.lse2[row0 * a.Hq + it] = fmaf(lse[u], LOG2E, -P_SHIFT<T>);
      }
    }
  }
  if constexpr (__is_same(T, TypeF16)) {
    const int values = tokens * a.Hkv;
    for (int it0 = threadIdx.x >> 4; it0 < values; it0 += 16 * AHEAD) {
      u32x4 w[AHEAD][CH];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int it = it0 + 16 * u < values ? it0 + 16 * u : it0, tok = it / a.Hkv;
        const uint16_t* p = (const uint16_t*)a.v + (row0 + tok) * a.v_stride + (long long)(it - tok * a.Hkv) * a.h;
#pragma unroll
        for (int x = 0; x < CH; ++x) {
          const int d = 128 * x + 8 * li;
          w[u][x] = d < a.h ? *(const u32x4*)(p + d) : u32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int x = 0; x < CH; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) finite_peak(peak[1], w[u][x][e]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      peak[i] = wave_max(peak[i]);
      if ((threadIdx.x & 63) == 0) red[i][threadIdx.x >> 6] = peak[i];
    }
    __syncthreads();
    if (threadIdx.x < 2) {
      const float* r = red[threadIdx.x];
      (threadIdx.x ? b.v_peak : b.dout_peak)[blockIdx.x] = fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]));
    }
  }
}

// What fp16 multiplies dS by: a power of two with which none leaves the type's range.  |dP| is at most h max|dout| max|v| and so is
// |delta|, v of all keys that the query sees, and P is at most 1.  Only finite values count: what an infinity makes of a dS no factor changes.  Only values that the sum
// is of count, so no other sequence, row or key takes bits from it.
__device__ __forceinline__ float ds_factor(int h, float dout_peak, float v_peak) {
  const float most = 2.f * (float)h * dout_peak * v_peak;
  if (!(most > 1e-30f)) return 1.f;
  // 2^14 over the power of two at or below `most`: dS is below 2^15
  return __uint_as_float((uint32_t)(254 + 14 - (int)(__float_as_uint(most) >> 23)) << 23);
}
// A sequence's peaks over the blocks that hold its tokens tok0 .. tok1 - 1.  A lane's first is on its way from where this is made on, the largest is
// found once other loads are waited for too.
struct Peaks { const float* from; int n; float first; };
__device__ __forceinline__ Peaks peaks_of(const Backward& b, const float* peaks, int s, int tok0, int tok1) {
  const int lane = threadIdx.x & 63, i0 = tok0 / b.delta_tokens;
  Peaks p{peaks + (long long)s * b.delta_chunks + i0, tok1 > tok0 ? (tok1 - 1) / b.delta_tokens - i0 + 1 : 0, 0.f};
  if (lane < p.n) p.first = p.from[lane];
  return p;
}
__device__ __forceinline__ float largest(const Peaks& p) {
  float peak = p.first;
  for (int i = (threadIdx.x & 63) + 64; i < p.n; i += 64) peak = fmaxf(peak, p.from[i]);
  return wave_max(peak);
}

// ------------------------------------------------------------------ keys' side
// A block owns 128 keys of a kv head, a wave 32 of them with K and V in registers; the rows of the group's queries that see them pass
// through LDS (q and dout, each read by rows for S = q K^T and dP = dout V^T, and transposed for dv^T = dout^T P and dk^T = q^T dS).
// Sinks are seen by every query behind them: what lies beyond the window is parted over blocks of its own, whose sums meet in
// parts_sum_kernel; else the block of the first keys would run for as long as all others together.  The same where few kv heads with many
// query heads, or a long sequence, would leave a few blocks the longest walks.
// At 128 dims eight waves share a block's keys, the second four taking the second half of every tile of queries, and add up in LDS at the
// end, since a block's queries are a long serial walk (three sequences of
// 1500 to 4000, window 1024, 32 heads over 8: 357 us, 480 with four waves).
template <int HD> constexpr int KEYS_HALVES = HD >= 128 ? 2 : 1;
// At 256 dims both gradients of a wave's keys would need all 512 registers and more: the first four waves take dv, the second dk, and both
// take S: five products for four, but two waves to a SIMD (six sequences of 500 to 2000, eight heads: 547 us as one wave to a SIMD, 244).

// The token behind the last that a tile of keys is seen by, its parted sinks apart
__device__ __forceinline__ int last_seer(const Backward& b, int kt, int n) {
  const WindowArgs& a = b.a;
  return a.window && (b.sinks > 0 || kt * BM >= a.sinks) ? (int)min((long long)n, (long long)kt * BM + BM - 1 + a.window) : n;
}

template <class T, int HD>
__global__ __launch_bounds__(TPB * KEYS_HALVES<HD>, 2) void keys_backward_kernel(Backward b, int key_tiles, int jobs) {
  typedef typename T::vec8 vec8;
  const WindowArgs& a = b.a;
  // Two waves to a SIMD hide each other's latencies, so a wave has 256 registers: from 128 dims on V waits in LDS instead.
  constexpr bool V_IN_LDS = HD >= 128;
  constexpr bool BY_GRADIENT = HD > 128;
  constexpr int HALVES = KEYS_HALVES<HD>, WAVES = 4 * HALVES;
  constexpr int BQ = HD > 128 ? 32 : 64, SUB = BY_GRADIENT ? 1 : BQ / 32 / HALVES, KS = HD / 16, DT = (HD + 31) / 32, TILE = BQ * HD;
  typedef Pieces<HD, BQ, WAVES> P;
  __shared__ __attribute__((aligned(256))) uint16_t lds[2][2][TILE];
  __shared__ __attribute__((aligned(256))) uint16_t v_tile[V_IN_LDS ? BM * HD : 128];
  __shared__ __attribute__((aligned(16))) float stat[2][3][64];            // of a tile's rows: lse log2 e less P's shift, delta, position (bits)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key_wave = HALVES > 1 ? wave & 3 : wave, half = HALVES > 1 ? wave >> 2 : 0;
  const int c = lane & 31, g = lane >> 5;
  const int G = a.Hq / a.Hkv;
  int unit, job;
  if (!map_block(blockIdx.x, a.S * a.Hkv, jobs, unit, job)) return;
  const int s = unit / a.Hkv, kvh = unit - s * a.Hkv;
  const Seq q = load_seq(a, s, false);
  // which keys, and the tokens that the job adds up
  const int sink_jobs = jobs - key_tiles * b.runs;
  int kt, tok0, tok1, slot = -1, run = 0;
  if (job < sink_jobs) {
    kt = job / b.chunks;
    slot = 1 + job % b.chunks;
    tok0 = kt * BM + BM - 1 + a.window + (slot - 1) * b.chunk;
    tok1 = min(tok0 + b.chunk, q.n);
  } else {
    kt = (job - sink_jobs) / b.runs;
    run = job - sink_jobs - kt * b.runs;
    tok0 = kt * BM;
    tok1 = last_seer(b, kt, q.n);
    if (b.runs > 1) {
      tok0 += run * b.run;
      tok1 = min(tok0 + b.run, tok1);
    } else if (kt * BM < b.sinks) {
      slot = 0;
    }
  }
  if (kt * BM >= q.n || tok0 >= tok1) return;
  const int kw = kt * BM + key_wave * 32, key = kw + c;
  const int M = q.n * G, m0 = tok0 * G, m1 = tok1 * G, n_tiles = (m1 - m0 + BQ - 1) / BQ;
  // the last position that sees this lane's key, from the key on (a position of -1 is beyond any)
  const uint32_t seen_by = a.window && key >= a.sinks ? a.window - 1 : 0x7fffffff - key;
  // parts beyond the window concern the sinks alone
  const bool idle = kw >= q.n || (slot > 0 && kw >= b.sinks);

  [[maybe_unused]] Peaks dout_peaks, near, far;      // of the queries walked; of the values in their sight, which delta is made of
  if constexpr (__is_same(T, TypeF16)) {
    const int lo = a.window ? max(tok0 - a.window + 1, 0) : 0;
    dout_peaks = peaks_of(b, b.dout_peak, s, tok0, tok1);
    near = peaks_of(b, b.v_peak, s, lo, tok1);
    far = peaks_of(b, b.v_peak, s, 0, min(a.sinks, lo));
  }
  vec8 kf[KS], vf[V_IN_LDS ? 1 : KS];
  {
    const long long row = q.row0 + min(key, q.n - 1);
    const uint16_t* kp = (const uint16_t*)a.k + row * a.k_stride + (long long)kvh * a.h;
    const uint16_t* vp = (const uint16_t*)a.v + row * a.v_stride + (long long)kvh * a.h;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int d = 16 * i + 8 * g;
      kf[i] = d < a.h ? *(const vec8*)(kp + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0});
      if constexpr (!V_IN_LDS) vf[i] = d < a.h ? *(const vec8*)(vp + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0});
    }
    if constexpr (V_IN_LDS)
      request_pieces(row_source(a.v, q.row0, a.v_stride, kvh, 1, a.h).tile(kt * BM, min(q.n - kt * BM, BM)),
                             piece_offsets<HD, BM, WAVES>(wave, lane, a.v_stride, a.h), lds_address(v_tile), wave);
  }
  // where tiles begin with a group's first head they all have the same offsets
  const bool even = BQ % G == 0;
  P q_off = flat_offsets<HD, BQ, WAVES>(wave, lane, a.q_stride, a.h, G, 0), o_off = flat_offsets<HD, BQ, WAVES>(wave, lane, a.dout_stride, a.h, G, 0);
  const RowSource q_rows = row_source(a.q, q.row0, a.q_stride, kvh * G, G, a.h), o_rows = row_source(a.dout, q.row0, a.dout_stride, kvh * G, G, a.h);
  const lds_t tiles0 = lds_address(lds[0][0]), stats0 = lds_address(stat[0][0]);
  auto request = [&](int t, int buf) {
    const int base = m0 + t * BQ, tok_base = even ? tok0 + t * (BQ / G) : base / G;
    if (!even) {
      q_off = flat_offsets<HD, BQ, WAVES>(wave, lane, a.q_stride, a.h, G, base - tok_base * G);
      o_off = flat_offsets<HD, BQ, WAVES>(wave, lane, a.dout_stride, a.h, G, base - tok_base * G);
    }
    const int rows = min(q.n - tok_base, BQ);
    request_pieces(q_rows.tile(tok_base, rows), q_off, tiles0 + buf * 4 * TILE, wave);
    request_pieces(o_rows.tile(tok_base, rows), o_off, tiles0 + buf * 4 * TILE + 2 * TILE, wave);
    if (wave < 3) {
      const int m = min(base + lane, M - 1), tok = m / G, head = kvh * G + m - tok * G;
      const long long at = (long long)(q.row0 + tok) * a.Hq + head;
      if (wave == 2) stat[buf][2][lane] = __int_as_float(base + lane < m1 ? tok : -1);      // (a row past the job's sees nothing)
      else request_word((wave ? b.delta : b.lse2) + at, stats0 + (buf * 3 + wave) * 256);
    }
  };

  f32x16 dk[DT], dv[BY_GRADIENT ? 1 : DT];     // (by gradient: a wave's own one in dk)
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) dk[t][i] = dv[BY_GRADIENT ? 0 : t][i] = 0.f;
  const float scale2 = a.scale * LOG2E;
  const int sub0 = BY_GRADIENT ? 0 : half * SUB;
  const lds_t tiles = tiles0 + sub0 * 32 * HD * 2, by_row = row_base<HD>(lane), v_row = lds_address(v_tile) + key_wave * 32 * HD * 2 + by_row;
  const ColumnBase<HD> by_column = column_base<HD>(lane);
  if (n_tiles > 0) request(0, 0);
  settle(kf);                                  // (behind the first request: one wait for both)
  if constexpr (!V_IN_LDS) settle(vf);
  float factor = 1.f;
  if constexpr (__is_same(T, TypeF16)) factor = ds_factor(a.h, largest(dout_peaks), fmaxf(largest(near), largest(far)));
  const float p_factor = factor * (1.f / P_SIZE<T>);
  scalars_landed();
  const bool few_keys = sees_few(a, q.n);
  auto walk = [&](auto few) {
    constexpr bool FEW = decltype(few)::value;
    for (int t = 0; t < n_tiles; ++t) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 1 < n_tiles) request(t + 1, (t + 1) & 1);
      if (idle) continue;
      const lds_t qt = tiles + (t & 1) * 4 * TILE, ot = qt + 2 * TILE;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const int base = m0 + t * BQ + 32 * (sub0 + u);
        if (base >= m1) break;
        const int p_lo = base / G, p_hi = min(base + 31, M - 1) / G;
        if (p_hi < kw || (a.window && kw + 31 <= p_lo - a.window && kw >= a.sinks)) continue;
        const bool whole = base + 31 < m1 && kw + 31 <= p_lo && (a.window == 0 || kw > p_hi - a.window || kw + 31 < a.sinks);
        f32x16 sc, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) sc = T::mfma32(row_frag<HD, vec8>(qt + by_row, 32 * u, i), kf[i], sc);
        if (!BY_GRADIENT || half)
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          if constexpr (V_IN_LDS) dp = T::mfma32(row_frag<HD, vec8>(ot + by_row, 32 * u, i), row_frag<HD, vec8>(v_row, 0, i), dp);
          else dp = T::mfma32(row_frag<HD, vec8>(ot + by_row, 32 * u, i), vf[i], dp);
        }
        if constexpr (!V_IN_LDS) order_products<1, 6, 2 * KS>();
        u32x4 pw[2], sw[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 32 * (sub0 + u) + 8 * j + 4 * g;
          const f32x4 lse2 = *(const f32x4*)&stat[t & 1][0][r], delta = *(const f32x4*)&stat[t & 1][1][r];
          float p[4], ds[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(sc[4 * j + e], scale2, -lse2[e]));
          }
          if (!whole) {
            const f32x4 where = *(const f32x4*)&stat[t & 1][2][r];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = (uint32_t)(__float_as_int(where[e]) - key) <= seen_by ? p[e] : 0.f;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) ds[e] = p[e] * (dp[4 * j + e] - delta[e]) * p_factor;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            pw[j >> 1][2 * (j & 1) + e] = T::pack(p[2 * e], p[2 * e + 1]);
            sw[j >> 1][2 * (j & 1) + e] = T::pack(ds[2 * e], ds[2 * e + 1]);
          }
          if constexpr (FEW) {
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * j + e] = ds[e];
          }
        }
        const ColumnBase<HD> oc = {ot + by_column.all, ot + by_column.last}, qc = {qt + by_column.all, qt + by_column.last};
        if (FEW && (!BY_GRADIENT || (half && few_keys))) {
          // (as on the queries' side: with what the rounding of dS loses)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            u32x4 rest;
#pragma unroll
            for (int e = 0; e < 4; ++e) rest[e] = rest_of<T>(dp[8 * v + 2 * e], dp[8 * v + 2 * e + 1], sw[v][e]);
#pragma unroll
            for (int d = 0; d < DT; ++d) dk[d] = T::mfma32(column_frag<HD, vec8>(qc, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, rest), dk[d]);
          }
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          if constexpr (BY_GRADIENT) {
            const ColumnBase<HD> mine = {half ? qc.all : oc.all, half ? qc.last : oc.last};
            const u32x4 w = half ? sw[v] : pw[v];
#pragma unroll
            for (int d = 0; d < DT; ++d) dk[d] = T::mfma32(column_frag<HD, vec8>(mine, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, w), dk[d]);
          } else {
#pragma unroll
            for (int d = 0; d < DT; ++d) dv[d] = T::mfma32(column_frag<HD, vec8>(oc, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, pw[v]), dv[d]);
#pragma unroll
            for (int d = 0; d < DT; ++d) dk[d] = T::mfma32(column_frag<HD, vec8>(qc, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, sw[v]), dk[d]);
          }
        }
      }
    }
  };
  // (by gradient one walk asks at every tile: a wave's registers do not hold two)
  if (BY_GRADIENT || few_keys) walk(std::true_type{});
  else walk(std::false_type{});
  if constexpr (HALVES > 1 && !BY_GRADIENT) {
    // the second half's sums through LDS, first those of dv, then those of dk: a register of 64 lanes a 256-byte row
    static_assert(sizeof(lds) >= 4 * DT * 16 * 64 * sizeof(float), "the tiles' place holds one gradient of four waves");
    float* meet = (float*)lds + key_wave * DT * 16 * 64 + lane;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      f32x16(&x)[DT] = which ? dk : dv;
      __syncthreads();
      if (half == 1) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) meet[(t * 16 + i) * 64] = x[t][i];
      }
      __syncthreads();
      if (half == 0) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[t][i] += meet[(t * 16 + i) * 64];
      }
    }
    if (half == 1) return;
  }
  const float back = a.scale / factor;
  const bool parted = slot >= 0 && key < b.sinks, in_runs = slot < 0 && b.runs > 1;
  const long long row = q.row0 + key;
  if ((parted || in_runs) && key < q.n) {
    float* to = in_runs ? b.run_part + (((long long)run * a.rows + row) * a.Hkv + kvh) * 2 * a.h
                        : b.part + ((((long long)unit * (b.chunks + 1) + slot) * 2) * b.sinks + key) * a.h;
    const long long to_values = in_runs ? a.h : (long long)b.sinks * a.h;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * t + 8 * j + 4 * g;
        if (d >= a.h) continue;
        if constexpr (BY_GRADIENT) {
          *(f32x4*)(to + (half ? 0 : to_values) + d) = f32x4{dk[t][4 * j], dk[t][4 * j + 1], dk[t][4 * j + 2], dk[t][4 * j + 3]} * (half ? back : 1.f / P_SIZE<T>);
        } else {
          *(f32x4*)(to + d) = f32x4{dk[t][4 * j], dk[t][4 * j + 1], dk[t][4 * j + 2], dk[t][4 * j + 3]} * back;
          *(f32x4*)(to + to_values + d) = f32x4{dv[t][4 * j], dv[t][4 * j + 1], dv[t][4 * j + 2], dv[t][4 * j + 3]} * (1.f / P_SIZE<T>);
        }
      }
  }
  const bool whole_sum = key < q.n && slot <= 0 && !parted && !in_runs;
  if constexpr (BY_GRADIENT) {
    store_row<T, DT>((uint16_t*)(half ? a.dk : a.dv) + row * (half ? a.dk_stride : a.dv_stride) + (long long)kvh * a.h, dk, half ? back : 1.f / P_SIZE<T>, a.h, g, whole_sum);
  } else {
    store_row<T, DT>((uint16_t*)a.dk + row * a.dk_stride + (long long)kvh * a.h, dk, back, a.h, g, whole_sum);
    store_row<T, DT>((uint16_t*)a.dv + row * a.dv_stride + (long long)kvh * a.h, dv, 1.f / P_SIZE<T>, a.h, g, whole_sum);
  }
}

// Adds up the parts of SUM_KEYS of a tile's keys (tile blockIdx.y), always in the same order.
constexpr int SUM_KEYS = 16;
template <class T>
__global__ __launch_bounds__(TPB) void parts_sum_kernel(Backward b) {
  const WindowArgs& a = b.a;
  const int unit = blockIdx.x, kt = blockIdx.y, s = unit / a.Hkv, kvh = unit - s * a.Hkv;
  const Seq q = load_seq(a, s, false);
  const int quads = a.h / 4, key0 = kt * BM + blockIdx.z * SUM_KEYS, n = min(min(b.runs > 1 ? key0 + SUM_KEYS : b.sinks, key0 + SUM_KEYS), q.n) - key0;
  if (n <= 0) return;
  const int runs = b.runs > 1 ? (last_seer(b, kt, q.n) - kt * BM + b.run - 1) / b.run : 0;
  const long long beyond = (long long)q.n - (kt * BM + BM - 1 + (long long)a.window);
  const int slots = 1 + (beyond > 0 ? (int)((beyond + b.chunk - 1) / b.chunk) : 0);
  for (int at = threadIdx.x; at < 2 * n * quads; at += TPB) {
    const int which = at / (n * quads), rest = at - which * n * quads, key = key0 + rest / quads, d = rest % quads * 4;
    const long long row = q.row0 + key;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int r = 0; r < runs; ++r) y += *(const f32x4*)(b.run_part + ((((long long)r * a.rows + row) * a.Hkv + kvh) * 2 + which) * a.h + d);
    if (key < b.sinks)
      for (int p = runs > 0 ? 1 : 0; p < slots; ++p) y += *(const f32x4*)(b.part + ((((long long)unit * (b.chunks + 1) + p) * 2 + which) * b.sinks + key) * a.h + d);
    uint16_t* to = (uint16_t*)(which ? a.dv : a.dk) + row * (which ? a.dv_stride : a.dk_stride) + (long long)kvh * a.h + d;
    *(u32x2*)to = u32x2{T::pack(y[0], y[1]), T::pack(y[2], y[3])};
  }
}

// ------------------------------------------------------------------ queries' side
// The forward pass's walk: a block owns 128 rows of a group's queries, a wave 32 of them with q and dout in registers; keys and values pass
// through LDS (K by rows and transposed, V by rows).
template <class T, int HD>
__global__ __launch_bounds__(TPB, HD > 128 ? 1 : HD > 96 ? 2 : 3) void queries_backward_kernel(Backward b, int tiles) {
  typedef typename T::vec8 vec8;
  const WindowArgs& a = b.a;
  constexpr int BN = HD > 128 ? 32 : 64, SUB = BN / 32, KS = HD / 16, DT = (HD + 31) / 32, TILE = BN * HD;
  __shared__ __attribute__((aligned(256))) uint16_t lds[2][2][TILE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, g = lane >> 5;
  const int G = a.Hq / a.Hkv;
  int unit, mt;
  if (!map_block(blockIdx.x, a.S * a.Hkv, tiles, unit, mt)) return;
  mt = tiles - 1 - mt;
  const int s = unit / a.Hkv, kvh = unit - s * a.Hkv;
  const Seq q = load_seq(a, s, false);
  const int m0 = mt * BM, M = q.n * G;
  if (m0 >= M) return;
  const int p_lo = m0 / G, p_hi = min(m0 + BM - 1, M - 1) / G, key_end = p_hi + 1;
  const int w_lo = a.window ? max(p_lo - a.window + 1, 0) : 0;
  const int sink_tiles = (min(min(a.sinks, w_lo), key_end) + BN - 1) / BN;
  const int w_base = max(w_lo, sink_tiles * BN);
  const int n_tiles = sink_tiles + (key_end > w_base ? (key_end - w_base + BN - 1) / BN : 0);
  auto tile_key = [&](int t) { return t < sink_tiles ? t * BN : w_base + (t - sink_tiles) * BN; };
  const int m = m0 + wave * 32 + c;
  const bool live = m < M;
  const int tok = min(m, M - 1) / G, head = kvh * G + min(m, M - 1) % G, pos = tok;
  const int wp_lo = min(m0 + wave * 32, M - 1) / G, wp_hi = min(m0 + wave * 32 + 31, M - 1) / G;
  const long long row = q.row0 + tok;
  [[maybe_unused]] Peaks near, far;            // of the values in the window, of those of the sinks
  if constexpr (__is_same(T, TypeF16)) {
    near = peaks_of(b, b.v_peak, s, w_lo, key_end);
    far = peaks_of(b, b.v_peak, s, 0, min(a.sinks, w_lo));
  }
  vec8 qf[KS], of[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    const int d = 16 * i + 8 * g;
    qf[i] = d < a.h ? *(const vec8*)((const uint16_t*)a.q + row * a.q_stride + (long long)head * a.h + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0});
    of[i] = d < a.h ? *(const vec8*)((const uint16_t*)a.dout + row * a.dout_stride + (long long)head * a.h + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0});
  }
  float of_row[2] = {b.lse2[row * a.Hq + head], b.delta[row * a.Hq + head]};
  const Pieces<HD, BN> k_off = piece_offsets<HD, BN>(wave, lane, a.k_stride, a.h), v_off = piece_offsets<HD, BN>(wave, lane, a.v_stride, a.h);
  const RowSource k_rows = row_source(a.k, q.row0, a.k_stride, kvh, 1, a.h), v_rows = row_source(a.v, q.row0, a.v_stride, kvh, 1, a.h);
  const lds_t tiles0 = lds_address(lds[0][0]);
  auto request = [&](int t, int buf) {
    const int base = tile_key(t);
    const int rows = min(q.n - base, BN);
    request_pieces(k_rows.tile(base, rows), k_off, tiles0 + buf * 4 * TILE, wave);
    request_pieces(v_rows.tile(base, rows), v_off, tiles0 + buf * 4 * TILE + 2 * TILE, wave);
  };
  f32x16 dq[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[t][i] = 0.f;
  const float scale2 = a.scale * LOG2E;
  const lds_t by_row = row_base<HD>(lane);
  const ColumnBase<HD> by_column = column_base<HD>(lane);
  if (n_tiles > 0) request(0, 0);
  settle(qf);
  settle(of);
  settle_words(of_row);
  float factor = 1.f;
  if constexpr (__is_same(T, TypeF16)) {
    float dout_peak = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = __builtin_bit_cast(u32x4, of[i])[e];
        const float lo = fabsf(T::low(w)), hi = fabsf(T::high(w));
        dout_peak = fmaxf(dout_peak, fmaxf(lo < INFINITY ? lo : 0.f, hi < INFINITY ? hi : 0.f));
      }
    factor = ds_factor(a.h, max_halves(dout_peak), fmaxf(largest(near), largest(far)));
  }
  const float lse2 = of_row[0];
  float delta = of_row[1];
  // This lane's row against 32 keys of the tile in buffer `buf`: scores (of the products' scale) and dP
  auto products = [&](int buf, int u, f32x16& sc, f32x16& dp) {
    const lds_t kt = tiles0 + buf * 4 * TILE, vt = kt + 2 * TILE;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) sc = T::mfma32(row_frag<HD, vec8>(kt + by_row, 32 * u, i), qf[i], sc);
#pragma unroll
    for (int i = 0; i < KS; ++i) dp = T::mfma32(row_frag<HD, vec8>(vt + by_row, 32 * u, i), of[i], dp);
    order_products<1, 6, 2 * KS>();
  };
  // out was rounded, and where a row sees few keys its delta is nearly as large as its dP: there the rounding shows in dS.  Such rows
  // take delta from the sum over their keys of P dP and leave it for the keys' side: a sequence's first 32 rows from the 32 keys that they
  // see at most, which begin the first tile; all rows, in a pass of its own, where every row sees few (FEW: a window of up to FEW_KEYS, or
  // a sequence of up to FEW_ROWS).  There dS also takes part with what its rounding loses, on both sides: over few keys, whose dS add up to
  // nothing, such errors do not average out (28 calls of 1 to 64 tokens or windows up to 25, against the formulas in 64 bits: 1.22 to 1.47
  // times the error of gradients that are rounded once, 1.00 with it).  Long sequences come to 1.45 without, and would pay 15 % of the keys'
  // side for it.
  auto own_delta = [&](int buf, int u, int kb) {
    f32x16 sc, dp;
    products(buf, u, sc, dp);
    const uint32_t bits = group_bits(seen_keys(pos, kb, a.window, a.sinks), g);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += or_else(__builtin_amdgcn_exp2f(fmaf(sc[i], scale2, -lse2)) * dp[i], element_mask(bits, i), 0u);
    return sum * (1.f / P_SIZE<T>);
  };
  const float p_factor = factor * (1.f / P_SIZE<T>);
  auto walk = [&](auto few) {
    constexpr bool FEW = decltype(few)::value;
    if constexpr (FEW) {
      float sum = 0.f;
      for (int t = 0; t < n_tiles; ++t) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + 1 < n_tiles) request(t + 1, (t + 1) & 1);
        for (int u = 0; u < SUB; ++u) sum += own_delta(t & 1, u, tile_key(t) + 32 * u);
      }
      delta = sum_halves(sum);
      if (live && g == 0) b.delta[row * a.Hq + head] = delta;
      __syncthreads();                           // (the tiles are filled again)
      if (n_tiles > 0) request(0, 0);
    } else if (p_lo < FEW_KEYS) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (wp_lo < FEW_KEYS) {
        const float sum = sum_halves(own_delta(0, 0, tile_key(0)));
        delta = pos < FEW_KEYS ? sum : delta;
        if (live && g == 0 && pos < FEW_KEYS) b.delta[row * a.Hq + head] = sum;
      }
    }
    scalars_landed();
    for (int t = 0; t < n_tiles; ++t) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 1 < n_tiles) request(t + 1, (t + 1) & 1);
      const lds_t kt = tiles0 + (t & 1) * 4 * TILE;
      const ColumnBase<HD> kc = {kt + by_column.all, kt + by_column.last};
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const int kb = tile_key(t) + 32 * u;
        if (kb > wp_hi || (a.window && kb + 31 <= wp_lo - a.window && kb >= a.sinks)) continue;
        const bool whole = kb + 31 <= wp_lo && (a.window == 0 || kb > wp_hi - a.window || kb + 31 < a.sinks);
        uint32_t bits = ~0u;
        if (!whole) bits = group_bits(seen_keys(pos, kb, a.window, a.sinks), g);
        f32x16 sc, dp;
        products(t & 1, u, sc, dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float ds = __builtin_amdgcn_exp2f(fmaf(sc[i], scale2, -lse2)) * (dp[i] - delta) * p_factor;
          dp[i] = or_else(ds, element_mask(bits, i), 0u);
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = T::pack(dp[8 * v + 2 * e], dp[8 * v + 2 * e + 1]);
          if constexpr (FEW) {
            u32x4 rest;
#pragma unroll
            for (int e = 0; e < 4; ++e) rest[e] = rest_of<T>(dp[8 * v + 2 * e], dp[8 * v + 2 * e + 1], w[e]);
#pragma unroll
            for (int d = 0; d < DT; ++d) dq[d] = T::mfma32(column_frag<HD, vec8>(kc, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, rest), dq[d]);
          }
#pragma unroll
          for (int d = 0; d < DT; ++d) dq[d] = T::mfma32(column_frag<HD, vec8>(kc, 32 * u + 16 * v, d), __builtin_bit_cast(vec8, w), dq[d]);
        }
        order_products<2, 3, 2 * DT>();
      }
    }
  };
  if (sees_few(a, q.n)) walk(std::true_type{});
  else walk(std::false_type{});
  store_row<T, DT>((uint16_t*)a.dq + row * a.dq_stride + (long long)head * a.h, dq, a.scale / factor, a.h, g, live);
}

// A walk of a tile of keys over the tokens that see it is long or short beside an even share of all such walks (512 blocks, two to a CU;
// one where h > 128), but no part has less than 512 rows.
int even_walk(const WindowArgs& a, long long walk) {
  const long long tiles = (long long)a.rows * a.Hkv / BM + (long long)a.S * a.Hkv / 2 + 1, blocks = a.h > 128 ? 256 : 512;
  const int G = a.Hq / a.Hkv, least = (512 + G - 1) / G;
  const long long even = (tiles * walk + blocks - 1) / blocks;
  return (int)(even < least ? least : even < a.max_new ? even : a.max_new);
}
// Sinks are parted while their partial sums (two fp32 vectors a sink, kv head and part) stay below 64 MB: into even shares.
void part_sinks(Backward& b) {
  const WindowArgs& a = b.a;
  b.sinks = b.chunks = 0;
  b.chunk = 1;
  const int sinks = a.sinks < a.max_new ? a.sinks : a.max_new;
  const long long beyond = (long long)a.max_new - (BM - 1 + (long long)a.window);
  if (!a.window || sinks < 1 || beyond < 1) return;
  const int chunk = even_walk(a, (long long)a.window + BM - 1);
  long long chunks = (beyond + chunk - 1) / chunk;
  const long long slot = (long long)a.S * a.Hkv * sinks * a.h * 2 * 4;
  if (chunks > 63) chunks = 63;
  if (slot * (chunks + 1) > (64ll << 20)) chunks = (64ll << 20) / slot - 1;
  if (chunks < 1) return;
  b.sinks = sinks;
  b.chunks = (int)chunks;
  b.chunk = (int)((beyond + chunks - 1) / chunks);
}
// The queries that see a tile of keys are parted where the longest such walk would take well over an even share: few kv heads with many
// query heads each, a long sequence.  Partial sums stay below 256 MB.
// Measured on six sequences of 500 to 2000 tokens, 12 heads over 2 of 96: 476 us in one walk, 220 parted with 11 for the sums; 16 over 4 of
// 64: 222 us, 118 with 11.
void part_runs(Backward& b) {
  const WindowArgs& a = b.a;
  b.runs = 1;
  b.run = a.max_new;
  long long longest = a.max_new;
  const bool bounded = a.window > 0 && (b.sinks > 0 || a.sinks == 0) && (long long)a.window + BM - 1 < longest;
  if (bounded) longest = (long long)a.window + BM - 1;
  const long long run = even_walk(a, bounded ? longest : longest / 2);
  if (2 * longest <= 3 * run) return;
  long long runs = (longest + run - 1) / run;
  if (runs > 8) runs = 8;
  const long long part = (long long)a.rows * a.Hkv * 2 * a.h * 4;
  if (part * runs > (256ll << 20)) runs = (256ll << 20) / part;
  if (runs < 2) return;
  b.runs = (int)runs;
  b.run = (int)((longest + runs - 1) / runs);
}
Backward parted(const WindowArgs& a) {
  Backward b;
  b.a = a;
  if (b.a.max_new > a.rows) b.a.max_new = a.rows < 1 ? 1 : a.rows;
  // A block has 64 (token, head) pairs at once, or as many times that as keep the blocks, of which those past a short sequence's end do nothing,
  // to 8192 and one a sequence (8250 tokens of 32 heads of 128 in bf16 in one step 22 us, 23 in two, 24 in four).
  const long long even = ((long long)a.S * b.a.max_new + 8191) / 8192, steps = (64 + a.Hq - 1) / a.Hq;
  b.delta_tokens = (int)(even > steps ? even : steps);
  b.delta_chunks = (int)(((long long)b.a.max_new + b.delta_tokens - 1) / b.delta_tokens);
  part_sinks(b);
  part_runs(b);
  return b;
}
size_t round_up(size_t n) { return (n + 255) / 256 * 256; }
// places the buffers and returns their size
size_t place(Backward& b, char* ws) {
  const WindowArgs& a = b.a;
  size_t at = 0;
  b.lse2 = (float*)(ws + at);
  at += round_up((size_t)a.rows * a.Hq * sizeof(float));
  b.delta = (float*)(ws + at);
  at += round_up((size_t)a.rows * a.Hq * sizeof(float));
  b.dout_peak = (float*)(ws + at);
  b.v_peak = b.dout_peak + (size_t)a.S * b.delta_chunks;
  at += round_up(2 * (size_t)a.S * b.delta_chunks * sizeof(float));
  b.part = (float*)(ws + at);
  at += round_up((size_t)a.S * a.Hkv * (b.chunks + 1) * 2 * b.sinks * a.h * sizeof(float));
  b.run_part = (float*)(ws + at);
  if (b.runs > 1) at += (size_t)b.runs * a.rows * a.Hkv * 2 * a.h * sizeof(float);
  return at;
}

struct Tiles { int keys, sinks, jobs, queries; };
Tiles tiles_of(const Backward& b) {
  const WindowArgs& a = b.a;
  Tiles t{(int)(((long long)a.max_new + BM - 1) / BM), (b.sinks + BM - 1) / BM, 0, (int)(((long long)a.max_new * (a.Hq / a.Hkv) + BM - 1) / BM)};
  t.jobs = t.keys * b.runs + t.sinks * b.chunks;
  return t;
}
template <class T, int HD>
hipError_t launch(const Backward& b, hipStream_t s) {
  const WindowArgs& a = b.a;
  const int units = a.S * a.Hkv;
  const Tiles t = tiles_of(b);
  hipLaunchKernelGGL((delta_kernel<T, (HD > 128 ? 2 : 1)>), dim3((unsigned)(a.S * b.delta_chunks)), dim3(TPB), 0, s, b);
  hipLaunchKernelGGL((queries_backward_kernel<T, HD>), dim3((unsigned)mapped_blocks(units, t.queries)), dim3(TPB), 0, s, b, t.queries);
  hipLaunchKernelGGL((keys_backward_kernel<T, HD>), dim3((unsigned)mapped_blocks(units, t.jobs)), dim3(TPB * KEYS_HALVES<HD>), 0, s, b, t.keys, t.jobs);
  if (b.sinks > 0 || b.runs > 1) hipLaunchKernelGGL((parts_sum_kernel<T>), dim3((unsigned)units, b.runs > 1 ? t.keys : t.sinks, BM / SUM_KEYS), dim3(TPB), 0, s, b);
  return hipGetLastError();
}
template <class T>
hipError_t by_head(const Backward& b, hipStream_t s) {
  const int h = b.a.h;
  if (h <= 32) return launch<T, 32>(b, s);
  if (h <= 64) return launch<T, 64>(b, s);
  if (h <= 80) return launch<T, 80>(b, s);
  if (h <= 96) return launch<T, 96>(b, s);
  if (h <= 128) return launch<T, 128>(b, s);
  return launch<T, 256>(b, s);
}

}  // namespace

size_t rl_window_backward_bytes(const WindowArgs& a) {
  Backward b = parted(a);
  return place(b, nullptr);
}
long long rl_window_backward_blocks(const WindowArgs& a) {
  const Backward b = parted(a);
  const Tiles t = tiles_of(b);
  const long long keys = (long long)t.jobs * (a.h > 96 ? KEYS_HALVES<128> : 1);          // (heads of more than 96 dims run as 128 or 256)
  return mapped_blocks((long long)a.S * a.Hkv, keys > t.queries ? keys : t.queries);
}
hipError_t rl_window_backward(const WindowArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  Backward b = parted(a);
  place(b, (char*)a.ws);
  return a.dtype == RLGEN_DTYPE_F16 ? by_head<TypeF16>(b, s) : by_head<TypeBf16>(b, s);
}
