// Attention with a sliding window and first tokens that stay visible, over packed sequences: keys and values as rows (training, fresh
// prompts) or out of the cache's pages (a chunk of new tokens behind a context).
//
// A query at position p sees key j if j <= p and (j > p - window, or j < sinks, or there is no window).  The keys that a tile of
// queries sees are two runs, the sinks and the window; tiles of keys walk the one and then the other, so the work follows the window
// and not the context.  Softmax in one pass over the keys with a running maximum and sum in 32 bits.
//
// The query heads of a kv head and the tokens make one axis (row m: token m / G, head m % G of the group), so a tile of 128 rows spans
// 128 / G tokens: grouped heads read a key once, and the diagonal and the window's edge waste less.
//   S^T[key, m] = K q^T             32x32x16 matrix instructions, K fragments from LDS, q in registers
//   O^T[d, m]  += V^T[d, key] P^T   the probabilities leave the first product in the layout the second wants; V is read transposed
// The probabilities are rounded to the inputs' type for the second product (the sum that they are divided by is of the unrounded ones):
// an error of the order of the output's own rounding.
#include "../../include/rlgen.h"
#include "window_tiles.h"

namespace {

constexpr int TPB = 256, BM = 128;

// Rows m_first .. m_first + 31 of a group's queries by one wave, key by key: what the matrix products cannot give where a value is infinite
// or NaN, since a probability of zero times it is NaN for every query of the tile, not only for those that see it.  Reached only by
// waves that found such a result.  64 keys at a time, one to a lane for the scores; for the sums a lane owns every 64th dim.
template <class T, bool PAGED>
__device__ void rows_key_by_key(const WindowArgs& a, const Seq& q, int s, int kvh, int m_first, int M, int lane) {
  const int G = a.Hq / a.Hkv;
  auto key_row = [&](int key, bool value) {
    if constexpr (PAGED) {
      const unsigned entry = a.page_table[(size_t)s * a.table_stride + (key >> a.page_shift)], page = entry < (unsigned)a.n_pages ? entry : 0;
      const long long row = ((((long long)page * 2 + (value ? 1 : 0)) * a.Hkv + kvh) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
      return (const uint16_t*)a.pages + row * a.h;
    } else {
      return (const uint16_t*)(value ? a.v : a.k) + (long long)(q.row0 + key) * (value ? a.v_stride : a.k_stride) + (long long)kvh * a.h;
    }
  };
  for (int m = m_first; m < min(m_first + 32, M); ++m) {
    const int tok = m / G, head = kvh * G + m - tok * G, pos = q.ctx + tok, end = min(pos + 1, q.total);
    const int w_lo = a.window ? max(pos - a.window + 1, 0) : 0, sinks = max(min(min(a.sinks, w_lo), end), 0);
    const uint16_t* qp = (const uint16_t*)a.q + (long long)(q.row0 + tok) * a.q_stride + (long long)head * a.h;
    float mx = -INFINITY, sum = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    const int seen = sinks + max(end - w_lo, 0);
    for (int i0 = 0; i0 < seen; i0 += 64) {
      const int i = i0 + lane;
      float sc = -INFINITY;
      if (i < seen) {
        const uint16_t* kp = key_row(i < sinks ? i : w_lo + i - sinks, false);
        sc = 0.f;
        for (int d = 0; d < a.h; d += 2) {
          const uint32_t kw = *(const uint32_t*)(kp + d), qw = *(const uint32_t*)(qp + d);
          sc = fmaf(T::low(kw), T::low(qw), sc);
          sc = fmaf(T::high(kw), T::high(qw), sc);
        }
        sc *= a.scale * 1.4426950408889634f;
      }
      const float now = fmaxf(mx, wave_max(sc)), base = now == -INFINITY ? 0.f : now;
      const float shrink = __builtin_amdgcn_exp2f(mx - base), p = __builtin_amdgcn_exp2f(sc - base);
      mx = now;
      sum = sum * shrink + wave_sum(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= shrink;
      for (int j = 0; j < min(64, seen - i0); ++j) {
        const float pj = __shfl(p, j, WAVE);
        const uint16_t* vp = key_row(i0 + j < sinks ? i0 + j : w_lo + i0 + j - sinks, true);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (lane + 64 * e < a.h) y[e] = fmaf(pj, T::low(vp[lane + 64 * e]), y[e]);
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const long long row = q.row0 + tok;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (lane + 64 * e < a.h) ((uint16_t*)a.out)[row * a.out_stride + (long long)head * a.h + lane + 64 * e] = (uint16_t)T::pack(y[e] * inv, 0.f);
    if (a.lse && lane == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

template <class T, int HD, bool PAGED>
__global__ __launch_bounds__(TPB, HD > 128 ? (PAGED ? 1 : 2) : HD > 96 ? 3 : 4) void window_rows_kernel(WindowArgs a, int tiles) {
  typedef typename T::vec8 vec8;
  constexpr int BN = 32, KS = HD / 16, DT = (HD + 31) / 32, TILE = BN * HD;
  constexpr int AHEAD = 6;
  typedef Pieces<HD, BN> P;
  __shared__ __attribute__((aligned(256))) uint16_t lds[2][2][TILE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, g = lane >> 5;
  const int G = a.Hq / a.Hkv;
  int unit, mt;
  if (!map_block(blockIdx.x, a.S * a.Hkv, tiles, unit, mt)) return;
  mt = tiles - 1 - mt;                                             // (late rows see most)
  const int s = unit / a.Hkv, kvh = unit - s * a.Hkv;
  const Seq q = load_seq(a, s, PAGED);
  const int m0 = mt * BM, M = q.n * G;
  if (m0 >= M) return;
  const int p_lo = q.ctx + m0 / G, p_hi = q.ctx + min(m0 + BM - 1, M - 1) / G;
  const int key_end = min(p_hi + 1, q.total);                      // keys from here on are seen by nobody
  const int w_lo = a.window ? max(p_lo - a.window + 1, 0) : 0;
  const int sink_tiles = (min(min(a.sinks, w_lo), key_end) + BN - 1) / BN;
  const int w_base = max(w_lo, sink_tiles * BN);
  const int n_tiles = sink_tiles + (key_end > w_base ? (key_end - w_base + BN - 1) / BN : 0);
  auto tile_key = [&](int t) { return t < sink_tiles ? t * BN : w_base + (t - sink_tiles) * BN; };

  // this lane's row
  const int m = m0 + wave * 32 + c;
  const bool live = m < M;
  const int tok = min(m, M - 1) / G, head = kvh * G + min(m, M - 1) % G, pos = q.ctx + tok;
  const int wp_lo = q.ctx + min(m0 + wave * 32, M - 1) / G, wp_hi = q.ctx + min(m0 + wave * 32 + 31, M - 1) / G;
  vec8 qf[KS];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (long long)(q.row0 + tok) * a.q_stride + (long long)head * a.h;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int d = 16 * i + 8 * g;
      qf[i] = signed_query(d < a.h ? *(const vec8*)(qp + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0}), a.scale);
    }
  }

  const int key_max = q.total - 1;
  [[maybe_unused]] P k_off, v_off;                                 // rows: a lane's offsets behind the tile's first row
  [[maybe_unused]] int page_of[P::PER];                            // pages: of the tile that is requested next
  if constexpr (!PAGED) {
    k_off = piece_offsets<HD, BN>(wave, lane, a.k_stride, a.h);
    v_off = piece_offsets<HD, BN>(wave, lane, a.v_stride, a.h);
  }
  const RowSource k_rows = row_source(a.k, q.row0, a.k_stride, kvh, 1, a.h), v_rows = row_source(a.v, q.row0, a.v_stride, kvh, 1, a.h);
  auto fetch_pages = [&](int t) {
    if constexpr (PAGED) {
#pragma unroll
      for (int n = 0; n < P::PER; ++n) {
        int row, dim;
        P::place(n, wave, lane, row, dim);
        page_of[n] = a.page_table[(size_t)s * a.table_stride + (min(tile_key(t) + row, key_max) >> a.page_shift)];
      }
    }
  };
  auto request = [&](int t, int buf) {
    const int base = tile_key(t);
    if constexpr (PAGED) {
#pragma unroll
      for (int n = 0; n < P::PER; ++n) {
        if (P::ALL % 4 != 0 && n * 4 + wave >= P::ALL) break;
        int row, dim;
        P::place(n, wave, lane, row, dim);
        const int key = min(base + row, key_max);                  // (rows past the last are masked)
        const unsigned page = (unsigned)page_of[n] < (unsigned)a.n_pages ? page_of[n] : 0;      // (an entry outside is not followed)
        const long long at = (((long long)page * 2 * a.Hkv + kvh) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
        const uint16_t* ks = (const uint16_t*)a.pages + at * a.h + dim;
        const uint16_t* vs = ks + ((long long)a.Hkv << a.page_shift) * a.h;
        if (dim >= a.h) ks = vs = (const uint16_t*)&zero_chunk;
        const int to = (n * 4 + wave) * 512;
        ::request(ks, lds[buf][0] + to);
        ::request(vs, lds[buf][1] + to);
      }
    } else {
      const int rows = min(q.n - base, BN);
      request_pieces(k_rows.tile(base, rows), k_off, lds[buf][0], wave);
      request_pieces(v_rows.tile(base, rows), v_off, lds[buf][1], wave);
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  // Of the scores times scale log2 e.  The maximum that the sums refer to follows the true one only when that is more than RISE ahead:
  // probabilities up to 2^RISE keep the type's relative precision, and most tiles then rescale nothing.
  constexpr float RISE = 8.f;
  float mx = -INFINITY, sum = 0.f;
  const float scale2 = score_factor(a.scale);
  const lds_t k_base = lds_address(lds[0][0]) + row_base<HD>(lane);
  ColumnBase<HD> v_base = column_base<HD>(lane);
  v_base.all += lds_address(lds[0][1]);
  v_base.last += lds_address(lds[0][1]);
  if (n_tiles > 0) {
    fetch_pages(0);
    request(0, 0);
    if (n_tiles > 1) fetch_pages(1);
  }
  settle(qf);                                  // (behind the first request: one wait for both)
  for (int t = 0; t < n_tiles; ++t) {
    // this tile has landed, and nobody reads the other buffer any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if constexpr (PAGED) settle_words(page_of);
    if (t + 1 < n_tiles) request(t + 1, (t + 1) & 1);
    if (t + 2 < n_tiles) fetch_pages(t + 2);
    const int kb = tile_key(t);
    if (kb > wp_hi || (a.window && kb + BN - 1 <= wp_lo - a.window && kb >= a.sinks)) continue;
    const lds_t buffer = (t & 1) * 4 * TILE;
    const ColumnBase<HD> vb = {v_base.all + buffer, v_base.last + buffer};
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) sc = T::mfma32(row_frag<HD, vec8>(k_base + buffer, 0, i), qf[i], sc);
    order_products<1, AHEAD, KS>();
    const bool whole = kb + BN - 1 <= wp_lo && (a.window == 0 || kb > wp_hi - a.window || kb + BN - 1 < a.sinks);
    float top = -INFINITY;
    if (!whole) {
      const uint32_t bits = group_bits(seen_keys(pos, kb, a.window, a.sinks), g);
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = or_else(sc[i], element_mask(bits, i), 0xff800000u);      // -infinity
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[i]);
    top = max_halves(top) * scale2;
    if (__any(top > mx + RISE)) {
      const float now = fmaxf(mx, top), shrink = __builtin_amdgcn_exp2f(mx - (now == -INFINITY ? 0.f : now));
      mx = now;
      sum *= shrink;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= shrink;
    }
    const float base = mx == -INFINITY ? 0.f : mx;            // a row that has seen no key yet keeps zeros
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], scale2, -base));
      part += sc[i];
    }
    sum += part;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = T::pack(sc[8 * u + 2 * e], sc[8 * u + 2 * e + 1]);
      const vec8 pf = __builtin_bit_cast(vec8, w);
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] = T::mfma32(column_frag<HD, vec8>(vb, 16 * u, d), pf, o[d]);
    }
  }
  sum = sum_halves(sum);
  const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);      // (NaN stays)
  bool finite = fabsf(sum) < INFINITY;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite &= fabsf(o[t][i]) < INFINITY;
  if (__any(live && !finite)) {
    rows_key_by_key<T, PAGED>(a, q, s, kvh, m0 + wave * 32, M, lane);
    return;
  }
  const long long row = q.row0 + tok;
  if (live && a.lse && g == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  store_row<T, DT>((uint16_t*)a.out + row * a.out_stride + (long long)head * a.h, o, inv, a.h, g, live);
}

template <class T, int HD>
hipError_t launch_rows(const WindowArgs& a, hipStream_t s) {
  const int tiles = (int)(((long long)a.max_new * (a.Hq / a.Hkv) + BM - 1) / BM);
  const dim3 grid(mapped_blocks(a.S * a.Hkv, tiles));
  if (a.pages) hipLaunchKernelGGL((window_rows_kernel<T, HD, true>), grid, dim3(TPB), 0, s, a, tiles);
  else hipLaunchKernelGGL((window_rows_kernel<T, HD, false>), grid, dim3(TPB), 0, s, a, tiles);
  return hipGetLastError();
}
template <class T>
hipError_t by_head(const WindowArgs& a, hipStream_t s) {
  // the smallest of the compiled sizes that holds the head; dims past it are zeros in LDS
  if (a.h <= 32) return launch_rows<T, 32>(a, s);
  if (a.h <= 64) return launch_rows<T, 64>(a, s);
  if (a.h <= 80) return launch_rows<T, 80>(a, s);
  if (a.h <= 96) return launch_rows<T, 96>(a, s);
  if (a.h <= 128) return launch_rows<T, 128>(a, s);
  return launch_rows<T, 256>(a, s);
}

}  // namespace

hipError_t rl_window_rows(WindowArgs a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (a.max_new > a.rows) a.max_new = a.rows;
  return a.dtype == RLGEN_DTYPE_F16 ? by_head<TypeF16>(a, s) : by_head<TypeBf16>(a, s);
}
