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
// an error of the order of the output's own rounding.  In fp16 they are taken 2^9 times as large, so that those down to 2^-23 of the largest are
// normal numbers: beside a first token that takes nearly all mass and has next to no value, an output is made of such.
//
// Tiles: 128 rows to a block and 32 of them to a wave, so that q stays in registers and a wave's sums are four (eight at 256 dims)
// accumulators; 32 keys to a tile, so that K and V of two tiles take 32 KB at 128 dims and three blocks share a CU (tiles of 64 keys: 33 us
// where these take 27, 48 sequences of up to 512 tokens, window 128).  Bound by neither memory nor the matrix unit alone: at 128 dims the
// exponentials, masks and conversions of a tile take as many cycles as its products, 46 and 39 % of the launch, and three waves to a SIMD
// overlap them only in part.  Measured: 8250 rows, 32 heads over 8 of 128, window 1024: 137 us for 0.11 TFLOP; 9985 rows, 32 heads of
// 80 in fp16: 77 us; a chunk of 500 rows on each of six contexts over pages: 71 us (on other cards 133 to 149, 76 to 84, 70 to 79).
#include "../../include/rlgen.h"
#include "window_tiles.h"

namespace {

constexpr int TPB = 256, BM = 128;

// Rows m_first .. m_end - 1 of a group's queries by one wave, key by key: what the matrix products cannot give where a value is infinite
// or NaN, since a probability of zero times it is NaN for every query of the tile, not only for those that see it.  Reached only by
// waves that found such a result.  64 keys at a time, one to a lane for the scores; for the sums a lane owns every 64th dim.
template <class T, bool PAGED>
__device__ void rows_key_by_key(const WindowArgs& a, const Seq& q, int s, int kvh, int m_first, int m_end, int lane) {
  const int G = a.Hq / a.Hkv;
  auto key_row = [&](int key, bool value) -> const uint16_t* {     // (null: the key's page lies outside the cache)
    if constexpr (PAGED) {
      const unsigned page = a.page_table[(size_t)s * a.table_stride + (key >> a.page_shift)];
      if (page >= (unsigned)a.n_pages) return nullptr;
      const long long row = ((((long long)page * 2 + (value ? 1 : 0)) * a.Hkv + kvh) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
      return (const uint16_t*)a.pages + row * a.h;
    } else {
      return (const uint16_t*)(value ? a.v : a.k) + (long long)(q.row0 + key) * (value ? a.v_stride : a.k_stride) + (long long)kvh * a.h;
    }
  };
  for (int m = m_first; m < m_end; ++m) {
    const int tok = m / G, head = kvh * G + m - tok * G, pos = q.ctx + tok, end = min(pos + 1, q.total);
    const int w_lo = a.window ? max(pos - a.window + 1, 0) : 0, sinks = max(min(min(a.sinks, w_lo), end), 0);
    const uint16_t* qp = (const uint16_t*)a.q + (long long)(q.row0 + tok) * a.q_stride + (long long)head * a.h;
    float mx = -INFINITY, sum = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    const int seen = sinks + max(end - w_lo, 0);
    for (int i0 = 0; i0 < seen; i0 += 64) {
      const int i = i0 + lane;
      float sc = -INFINITY;
      const uint16_t* kp = i < seen ? key_row(i < sinks ? i : w_lo + i - sinks, false) : nullptr;
      if (kp) {
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
        if (!vp) continue;
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

// Where blocks leave their part of the keys: [sequence, kv head, row of its group, part] the largest score and the sum, and h dims that
// are not yet divided by it.
struct RowParts { float2* stats; float* out; };
__device__ __forceinline__ RowParts row_parts(const WindowArgs& a, int parts) {
  return {(float2*)a.ws, (float*)((float2*)a.ws + ((long long)a.S * a.max_new * a.Hq * parts + 1) / 2 * 2)};
}

template <class T, int HD, bool PAGED>
__global__ __launch_bounds__(TPB, HD > 128 ? (PAGED ? 1 : 2) : HD > 96 ? 3 : 4) void window_rows_kernel(WindowArgs a, int tiles, int parts) {
  typedef typename T::vec8 vec8;
  constexpr int BN = 32, KS = HD / 16, DT = (HD + 31) / 32, TILE = BN * HD;
  constexpr int AHEAD = 6;
  typedef Pieces<HD, BN> P;
  __shared__ __attribute__((aligned(256))) uint16_t lds[2][2][TILE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, g = lane >> 5;
  const int G = a.Hq / a.Hkv;
  int unit, mt;
  if (!map_block(blockIdx.x, a.S * a.Hkv, tiles * parts, unit, mt)) return;
  const int part = PAGED ? mt % parts : 0;
  mt = tiles - 1 - (PAGED ? mt / parts : mt);                      // (late rows see most)
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
  const int t0 = PAGED ? (int)((long long)n_tiles * part / parts) : 0, t1 = PAGED ? (int)((long long)n_tiles * (part + 1) / parts) : n_tiles;
  // Pages outside the cache, which nobody sees, are looked for once in front of the walk: where there are none, as a rule, no tile asks.
  // Of the table's entries that the walk reads, first the sinks', then the window's; a thread's first is under way while tiles are requested.
  const int* table = PAGED ? a.page_table + (size_t)s * a.table_stride : nullptr;
  auto entries_of = [&](int ta, int tb) {      // first, and how many
    const int e = tile_key(ta) >> a.page_shift;
    return int2{e, ta < tb ? ((min(tile_key(tb - 1) + BN, q.total) - 1) >> a.page_shift) - e + 1 : 0};
  };
  [[maybe_unused]] int2 near, far;
  [[maybe_unused]] int page_seen = 0;
  auto entry = [&](int i) { return table[i < far.y ? far.x + i : near.x + i - far.y]; };
  if constexpr (PAGED) {
    const int mid = min(max(sink_tiles, t0), max(t0, t1));
    far = entries_of(t0, mid);
    near = entries_of(mid, t1);
    if ((int)threadIdx.x < far.y + near.y) page_seen = entry(threadIdx.x);
  }

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
        page_of[n] = table[min(tile_key(t) + row, key_max) >> a.page_shift];
      }
    }
  };
  const lds_t tiles0 = lds_address(lds[0][0]);
  auto request = [&](int t, int buf) {
    const int base = tile_key(t);
    if constexpr (PAGED) {
#pragma unroll
      for (int n = 0; n < P::PER; ++n) {
        if (P::ALL % 4 != 0 && n * 4 + wave >= P::ALL) break;
        int row, dim;
        P::place(n, wave, lane, row, dim);
        const int key = min(base + row, key_max);                  // (rows past the last are masked)
        const unsigned page = (unsigned)page_of[n] < (unsigned)a.n_pages ? page_of[n] : 0;      // (an entry outside is not followed, its keys are masked)
        const long long at = (((long long)page * 2 * a.Hkv + kvh) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
        const uint16_t* ks = (const uint16_t*)a.pages + at * a.h + dim;
        const uint16_t* vs = ks + ((long long)a.Hkv << a.page_shift) * a.h;
        if (dim >= a.h) ks = vs = (const uint16_t*)&zero_chunk;
        const lds_t to = tiles0 + buf * 4 * TILE + (n * 4 + wave) * 1024;
        ::request(ks, to);
        ::request(vs, to + 2 * TILE);
      }
    } else {
      const int rows = min(q.n - base, BN);
      request_pieces(k_rows.tile(base, rows), k_off, tiles0 + buf * 4 * TILE, wave);
      request_pieces(v_rows.tile(base, rows), v_off, tiles0 + buf * 4 * TILE + 2 * TILE, wave);
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  // Of the scores times scale log2 e.  The maximum that the sums refer to follows the true one only when that is more than RISE ahead:
  // probabilities up to 2^RISE (times 2^UP) keep the type's relative precision, and most tiles then rescale nothing (48 sequences of up to 512
  // tokens in fp16, RISE 8, 6 and 4: 23.8, 24.2 and 24.6 us).
  constexpr float RISE = __is_same(T, TypeF16) ? 6.f : 8.f, UP = __is_same(T, TypeF16) ? 9.f : 0.f;
  float mx = -INFINITY, sum = 0.f;
  const float scale2 = score_factor(a.scale);
  const lds_t k_base = tiles0 + row_base<HD>(lane);
  ColumnBase<HD> v_base = column_base<HD>(lane);
  v_base.all += tiles0 + 2 * TILE;
  v_base.last += tiles0 + 2 * TILE;
  if (t0 < t1) {
    fetch_pages(t0);
    request(t0, t0 & 1);
    if (t0 + 1 < t1) fetch_pages(t0 + 1);
  }
  bool holes = false;
  if constexpr (PAGED) {
    holes = (unsigned)page_seen >= (unsigned)a.n_pages;
    for (int i = threadIdx.x + TPB; i < far.y + near.y; i += TPB) holes |= (unsigned)entry(i) >= (unsigned)a.n_pages;
    holes = __syncthreads_or(holes);
  }
  settle(qf);                                  // (behind the first request: one wait for both)
  scalars_landed();
  for (int t = t0; t < t1; ++t) {
    // this tile has landed, and nobody reads the other buffer any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if constexpr (PAGED) settle_words(page_of);
    if (t + 1 < t1) request(t + 1, (t + 1) & 1);
    if (t + 2 < t1) fetch_pages(t + 2);
    const int kb = tile_key(t);
    if (m0 + wave * 32 >= M || kb > wp_hi || (a.window && kb + BN - 1 <= wp_lo - a.window && kb >= a.sinks)) continue;
    const lds_t buffer = (t & 1) * 4 * TILE;
    const ColumnBase<HD> vb = {v_base.all + buffer, v_base.last + buffer};
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) sc = T::mfma32(row_frag<HD, vec8>(k_base + buffer, 0, i), qf[i], sc);
    order_products<1, AHEAD, KS>();
    const bool whole = kb + BN - 1 <= wp_lo && (a.window == 0 || kb > wp_hi - a.window || kb + BN - 1 < a.sinks) && !holes;
    float top = -INFINITY;
    if (!whole) {
      uint32_t seen = seen_keys(pos, kb, a.window, a.sinks);
      if constexpr (PAGED) {
        if (holes) {
          const unsigned page = table[min(kb + c, key_max) >> a.page_shift];
          seen &= (uint32_t)__ballot(page < (unsigned)a.n_pages);
        }
      }
      const uint32_t bits = group_bits(seen, g);
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
    const float base = mx == -INFINITY ? 0.f : mx - UP;       // a row that has seen no key yet keeps zeros
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
  mx -= UP;                                    // (what the sums refer to)
  const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);      // (NaN stays)
  bool finite = fabsf(sum) < INFINITY;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) finite &= fabsf(o[t][i]) < INFINITY;
  if (PAGED && parts > 1) {
    if (!live) return;
    const RowParts to = row_parts(a, parts);
    const long long slot = ((long long)unit * a.max_new * G + m) * parts + part;
    if (g == 0) to.stats[slot] = float2{mx, sum};
    // (a value that is not finite is told by a sum that is none: its row is computed again where the parts are joined)
    if (__shfl_xor(finite ? 1 : 0, 32, WAVE) == 0) finite = false;
    if (g == 0 && !finite) to.stats[slot].y = __builtin_nanf("");
    float* y = to.out + slot * a.h;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (32 * t + 8 * j + 4 * g < a.h) *(f32x4*)(y + 32 * t + 8 * j + 4 * g) = f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
    return;
  }
  if (__any(live && !finite)) {
    rows_key_by_key<T, PAGED>(a, q, s, kvh, m0 + wave * 32, min(m0 + wave * 32 + 32, M), lane);
    return;
  }
  const long long row = q.row0 + tok;
  if (live && a.lse && g == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  store_row<T, DT>((uint16_t*)a.out + row * a.out_stride + (long long)head * a.h, o, inv, a.h, g, live);
}

// Adds up the parts of a row in their order: a row to 16, 32 or 64 lanes (`lanes`), four dims to a lane.
template <class T>
__global__ __launch_bounds__(TPB) void rows_join_kernel(WindowArgs a, int parts, int lanes) {
  const int lane = threadIdx.x & 63, G = a.Hq / a.Hkv;
  const long long rows = (long long)a.max_new * G, all = (long long)a.S * a.Hkv * rows, first = ((long long)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / lanes);
  const long long at = first + lane / lanes;
  if (first >= all) return;
  const int unit = (int)(min(at, all - 1) / rows), m = (int)(min(at, all - 1) - unit * rows), s = unit / a.Hkv, kvh = unit - s * a.Hkv;
  const Seq q = load_seq(a, s, true);
  const bool live = at < all && m < q.n * G;
  const RowParts from = row_parts(a, parts);
  const float2* stats = from.stats + ((long long)unit * rows + m) * parts;
  const float* out = from.out + ((long long)unit * rows + m) * parts * a.h;
  const int d = lane % lanes * 4, tok = m / G, head = kvh * G + m - tok * G;
  float mx = -INFINITY, sum = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (live) {
    for (int p = 0; p < parts; ++p) mx = fmaxf(mx, stats[p].x);
    const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) {
      const float2 part = stats[p];
      const float f = __builtin_amdgcn_exp2f(part.x - base);
      sum = fmaf(part.y, f, sum);
      if (d < a.h) y += *(const f32x4*)(out + (long long)p * a.h + d) * f;
    }
    const float inv = sum > 0.f ? 1.0f / sum : 0.f;
    const long long row = q.row0 + tok;
    if (d < a.h) *(u32x2*)((uint16_t*)a.out + row * a.out_stride + (long long)head * a.h + d) = u32x2{T::pack(y[0] * inv, y[1] * inv), T::pack(y[2] * inv, y[3] * inv)};
    if (a.lse && d == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
  for (int i = 0; i < 64; i += lanes) {
    if (!__shfl(live && sum != sum ? 1 : 0, i, WAVE)) continue;
    const int s1 = __shfl(s, i, WAVE), kvh1 = __shfl(kvh, i, WAVE), m1 = __shfl(m, i, WAVE);
    rows_key_by_key<T, true>(a, load_seq(a, s1, true), s1, kvh1, m1, m1 + 1, lane);
  }
}

// Parts of the keys of a call over pages: those whose walk, with what writing and reading the partial results adds, is estimated to be the
// shortest, a part having at least eight tiles and partial results staying below 128 MB.  A tile of keys costs a block about 0.9 us alone on its CU and 0.45 us for each other block
// there; partial results pass at 4 TB/s and the second launch costs 5 us.  Measured whole and parted: 8 new tokens on 12000, 32 heads over
// 8 of 128, 338 us and 46; 500 on 8000, 234 and 118; 3 on each of seven of 1067 to 6375, 32 heads of 80, 189 and 59; but 200 on each of
// four with a window of 1024, 38 and 53: those stay whole.
int rows_parts(const WindowArgs& a) {
  const int G = a.Hq / a.Hkv, at_once = a.h > 128 ? 1 : a.h > 96 ? 3 : 4;
  const double blocks = (double)(((long long)a.max_new * G + BM - 1) / BM) * a.S * a.Hkv, row_us = (double)a.S * a.max_new * a.Hq * (a.h + 2) * 8 / 4e6;
  long long seen = a.max_total;
  if (a.window && (long long)a.window + BM / G + a.sinks < seen) seen = (long long)a.window + BM / G + a.sinks;
  const double tiles = (double)((seen + 31) / 32);
  int best = 1;
  double best_us = 0;
  for (int parts = 1; parts <= 64 && (parts == 1 || (parts * 8 <= tiles && parts * row_us < 64)); ++parts) {
    const double on_cu = ceil(blocks * parts / 256), rounds = ceil(on_cu / at_once);
    const double us = ceil(tiles / parts) * rounds * 0.45 * (1 + (on_cu < at_once ? on_cu : at_once)) + (parts > 1 ? 5 + parts * row_us : 0);
    if (parts == 1 || us < best_us) {
      best = parts;
      best_us = us;
    }
  }
  return best;
}
size_t parts_bytes(const WindowArgs& a, int parts) {
  return parts > 1 ? ((size_t)a.S * a.max_new * a.Hq * parts + 1) / 2 * 2 * (sizeof(float2) + (size_t)a.h * sizeof(float)) : 0;
}

struct Rows { int max_new, tiles, parts; };
Rows rows_launch(const WindowArgs& a) {
  Rows r{a.pages || a.max_new < a.rows ? a.max_new : a.rows, 0, 1};          // (packed sequences have no more rows than there are)
  r.tiles = (int)(((long long)r.max_new * (a.Hq / a.Hkv) + BM - 1) / BM);
  if (a.pages) {
    r.parts = rows_parts(a);
    if (r.parts > 1 && (!a.ws || a.ws_bytes < parts_bytes(a, r.parts))) r.parts = 1;
  }
  return r;
}

template <class T, int HD>
hipError_t launch_rows(WindowArgs a, hipStream_t s) {
  const Rows r = rows_launch(a);
  const int tiles = r.tiles, parts = r.parts;
  a.max_new = r.max_new;
  const dim3 grid((unsigned)mapped_blocks((long long)a.S * a.Hkv, (long long)tiles * parts));
  if (!a.pages) {
    hipLaunchKernelGGL((window_rows_kernel<T, HD, false>), grid, dim3(TPB), 0, s, a, tiles, 1);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((window_rows_kernel<T, HD, true>), grid, dim3(TPB), 0, s, a, tiles, parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int lanes = a.h <= 64 ? 16 : a.h <= 128 ? 32 : 64;
  const long long waves = ((long long)a.S * a.max_new * a.Hq + 64 / lanes - 1) / (64 / lanes);
  hipLaunchKernelGGL((rows_join_kernel<T>), dim3((unsigned)((waves + 3) / 4)), dim3(TPB), 0, s, a, parts, lanes);
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

long long rl_window_rows_blocks(const WindowArgs& a) {
  const Rows r = rows_launch(a);
  return mapped_blocks((long long)a.S * a.Hkv, (long long)r.tiles * r.parts);
}
hipError_t rl_window_rows(const WindowArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return a.dtype == RLGEN_DTYPE_F16 ? by_head<TypeF16>(a, s) : by_head<TypeBf16>(a, s);
}
size_t rl_window_rows_bytes(const WindowArgs& a) { return parts_bytes(a, rows_parts(a)); }
