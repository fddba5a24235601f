// Windowed attention of single tokens over the paged cache: the bandwidth-bound step of serving.
//
// One wave takes 32 keys of one kv head at a time, the query heads of its group in the columns of 16x16x32 matrix instructions:
//   S^T[key, col] = K q^T          a lane reads 16 bytes of a key: the fragment as it lies in the page
//   O^T[dim, col] += V^T P^T       a lane reads the same eight (four) dims of eight keys; their words change places in registers, which
//                                  gives the fragments of V^T without a pass through LDS
// The scores leave the first product where the second wants its probabilities (key 8 g + 4 t + j in lane group g).  Visible keys are two
// runs, sinks and window, so a step's cost follows the window.  Eight keys in a row share a page, so a lane looks up two pages for
// 32 keys, one iteration before it needs them; the next 32 keys are requested before the present ones are used.
// In fp16 the probabilities are taken 2^15 times as large, which keeps those down to 2^-29 of the largest normal numbers.
// Values that are not seen are zeroed, not multiplied by zero; a page outside the cache is not seen (a lane's scores and values are those of the
// eight keys that it looked up together).
//
// Bound by HBM: 4 h bytes a visible key and kv head.  Measured: 512 sequences of 257 to 576 tokens, 32 heads of 80 in fp16: 443 us, 4.9 TB/s;
// one of 32001, 32 heads over 8 of 128: 25 us and 4 for the join, 5.2 TB/s without it; 64 of up to 9000, window 1024: 46 us, 5.5 TB/s (in
// part out of the last-level cache).
#include "../../include/rlgen.h"
#include "window_tiles.h"

namespace {

constexpr int TPB = 256;

struct Part { float m, l; };

// JW waves share a job (a sequence's kv head and up to CB of its query heads), each taking every JW-th group of 32 keys; the
// maxima, sums and outputs meet in LDS.  PARTS: several blocks share it as well and leave their share for window_join_kernel.
template <class T, int HD, int JW>
__global__ __launch_bounds__(TPB, HD > 128 ? 1 : 2) void window_decode_kernel(WindowArgs a, int parts, int col_blocks) {
  typedef typename T::vec8 vec8;
  constexpr int KS = (HD + 31) / 32, VW = HD > 64 ? 8 : 4, CH = HD > 128 ? 2 : 1, CB = HD > 128 ? 8 : 16;
  extern __shared__ float joined[];            // JW > 1: [JW][columns][h]
  __shared__ Part part_of[4][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int G = a.Hq / a.Hkv;
  long long job = JW > 1 ? blockIdx.x : (long long)blockIdx.x * 4 + wave;
  const int part = (int)(job % parts);
  job /= parts;
  if (job >= (long long)a.S * a.Hkv * col_blocks) return;
  const int cb = (int)(job % col_blocks), kvh = (int)(job / col_blocks % a.Hkv), s = (int)(job / col_blocks / a.Hkv);
  const Seq q = load_seq(a, s, true);
  if (q.n < 1) return;
  const int cols = min(G - cb * CB, CB), head0 = kvh * G + cb * CB;
  const int pos = q.ctx, key_end = min(pos + 1, q.total);
  const int w_lo = a.window ? max(pos - a.window + 1, 0) : 0;
  const int sink_groups = (max(min(min(a.sinks, w_lo), key_end), 0) + 31) >> 5;
  const int w_base = max(w_lo & ~7, sink_groups * 32);
  const int groups = sink_groups + (key_end > w_base ? (key_end - w_base + 31) >> 5 : 0);
  auto group_key = [&](int i) { return i < sink_groups ? i * 32 : w_base + (i - sink_groups) * 32; };
  const int i0 = (int)((long long)groups * part / parts) + (JW > 1 ? wave : 0), i1 = (int)((long long)groups * (part + 1) / parts);

  vec8 qf[KS];
  {
    const uint16_t* qp = (const uint16_t*)a.q + (long long)q.row0 * a.q_stride + (long long)(head0 + min(c, cols - 1)) * a.h;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int d = 32 * i + 8 * g;
      qf[i] = signed_query(d < a.h ? *(const vec8*)(qp + d) : __builtin_bit_cast(vec8, u32x4{0, 0, 0, 0}), a.scale);
    }
  }
  const int last8 = (key_end - 1) & ~7, in_page = (1 << a.page_shift) - 1;
  const int* table = a.page_table + (size_t)s * a.table_stride;
  const long long plane = ((long long)a.Hkv << a.page_shift) * a.h;      // from a page's keys to its values
  auto key8 = [&](int i, int quad) { return min(group_key(i) + 8 * quad, last8); };
  auto lookup = [&](int i, int& pk, int& pv) {
    pk = table[key8(i, c >> 2) >> a.page_shift];
    pv = table[key8(i, g) >> a.page_shift];
  };
  auto inside = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
  auto page_row = [&](int page, int key) {            // (an entry outside the cache is not followed, its keys are masked)
    const unsigned p = inside(page) ? page : 0;
    return (const uint16_t*)a.pages + ((((long long)p * 2 * a.Hkv + kvh) << a.page_shift) + (key & in_page)) * a.h;
  };
  typedef uint32_t vraw_t __attribute__((ext_vector_type(VW / 2)));
  auto load = [&](int i, int pk, int pv, u32x4 (&k)[2][KS], vraw_t (&v)[CH][8]) {
    const uint16_t* kp = page_row(pk, key8(i, c >> 2)) + (c & 3) * a.h + 8 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        if (32 * j + 8 * g < a.h) k[t][j] = __builtin_nontemporal_load((const u32x4*)(kp + 4 * t * a.h + 32 * j));
        else k[t][j] = u32x4{0, 0, 0, 0};
      }
    const uint16_t* vp = page_row(pv, key8(i, g)) + plane + VW * c;
#pragma unroll
    for (int x = 0; x < CH; ++x)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (128 * x + VW * c < a.h) v[x][e] = __builtin_nontemporal_load((const vraw_t*)(vp + e * a.h + 128 * x));
        else
#pragma unroll
          for (int w = 0; w < VW / 2; ++w) v[x][e][w] = 0;
  };

  f32x4 o[CH][VW];
#pragma unroll
  for (int x = 0; x < CH; ++x)
#pragma unroll
    for (int e = 0; e < VW; ++e) o[x][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr float UP = __is_same(T, TypeF16) ? 15.f : 0.f;
  float mx = -INFINITY, sum = 0.f;
  const float scale2 = score_factor(a.scale);
  u32x4 k[2][KS], k_next[2][KS];
  vraw_t v[CH][8], v_next[CH][8];
  int pk, pv;
  bool there = true, there_next = true;
  if (i0 < i1) {
    lookup(i0, pk, pv);
    load(i0, pk, pv, k, v);
    there = inside(pv);
    lookup(min(i0 + JW, i1 - 1), pk, pv);
  }
  for (int i = i0; i < i1; i += JW) {
    if (i + JW < i1) {
      load(i + JW, pk, pv, k_next, v_next);
      there_next = inside(pv);
      lookup(min(i + 2 * JW, i1 - 1), pk, pv);
    }
    const int kb = group_key(i);
    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) sc[t] = T::mfma16(__builtin_bit_cast(vec8, k[t][j]), qf[j], sc[t]);
    }
    const int key0 = kb + 8 * g;
    if (kb + 31 >= key_end || (kb < w_lo && kb + 31 >= a.sinks) || __any(!there)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + e;
        // (selections, not a branch: of a branch that writes single elements of these vectors the compiler lost one)
        const bool seen = (key < key_end) & ((key >= w_lo) | (key < a.sinks)) & there;
        const uint32_t keep = seen ? 0xffffffffu : 0u;
        sc[e >> 2][e & 3] = seen ? sc[e >> 2][e & 3] : -INFINITY;
#pragma unroll
        for (int x = 0; x < CH; ++x)
#pragma unroll
          for (int w = 0; w < VW / 2; ++w) v[x][e][w] &= keep;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, sc[e >> 2][e & 3]);
    top = fmaxf(top, __shfl_xor(top, 16, WAVE));
    top = fmaxf(top, __shfl_xor(top, 32, WAVE)) * scale2;
    const float now = fmaxf(mx, top), base = (now == -INFINITY ? 0.f : now) - UP;
    if (__any(now > mx)) {
      const float shrink = __builtin_amdgcn_exp2f(mx - UP - base);
      sum *= shrink;
#pragma unroll
      for (int x = 0; x < CH; ++x)
#pragma unroll
        for (int e = 0; e < VW; ++e) o[x][e] *= shrink;
    }
    mx = now;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(sc[e >> 2][e & 3], scale2, -base));
      sum += p[e];
    }
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = T::pack(p[2 * e], p[2 * e + 1]);
    const vec8 pf = __builtin_bit_cast(vec8, w);
#pragma unroll
    for (int x = 0; x < CH; ++x)
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        u32x4 f;                                   // dim VW c + e of the eight keys
#pragma unroll
        for (int y = 0; y < 4; ++y) f[y] = __builtin_amdgcn_perm(v[x][2 * y + 1][e >> 1], v[x][2 * y][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
        o[x][e] = T::mfma16(__builtin_bit_cast(vec8, f), pf, o[x][e]);
      }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < KS; ++j) k[t][j] = k_next[t][j];
#pragma unroll
    for (int x = 0; x < CH; ++x)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[x][e] = v_next[x][e];
    there = there_next;
  }
  sum += __shfl_xor(sum, 16, WAVE);
  sum += __shfl_xor(sum, 32, WAVE);
  mx -= UP;                                        // (what the sums refer to)
  // lane (c, g) holds of column c the dims VW (4 g + j) + e, j = 0..3
  const long long row = q.row0;
  if constexpr (JW == 1) {
    if (c >= cols) return;
    const float inv = sum > 0.f ? 1.0f / sum : (sum == 0.f ? 0.f : sum);
    const int head = head0 + c;
    if (a.lse && g == 0) a.lse[row * a.Hq + head] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    uint16_t* op = (uint16_t*)a.out + row * a.out_stride + (long long)head * a.h;
#pragma unroll
    for (int x = 0; x < CH; ++x)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 128 * x + VW * (4 * g + j);
        if (d >= a.h) continue;
        vraw_t y;
#pragma unroll
        for (int e = 0; e < VW / 2; ++e) y[e] = T::pack(o[x][2 * e][j] * inv, o[x][2 * e + 1][j] * inv);
        *(vraw_t*)(op + d) = y;
      }
    return;
  } else {
    if (g == 0) part_of[wave][c] = Part{mx, sum};
    if (c < cols) {
      float* mine = joined + ((size_t)wave * cols + c) * a.h;
#pragma unroll
      for (int x = 0; x < CH; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = 128 * x + VW * (4 * g + j);
          if (d >= a.h) continue;
#pragma unroll
          for (int e = 0; e < VW; ++e) mine[d + e] = o[x][e][j];
        }
    }
    __syncthreads();
    float* po = (float*)a.ws;                                            // partial outputs, then their maxima and sums
    Part* pm = (Part*)(po + (long long)a.S * a.Hq * parts * a.h);
    for (int at = threadIdx.x * 2; at < cols * a.h; at += TPB * 2) {
      const int col = at / a.h, d = at - col * a.h;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < JW; ++w) m = fmaxf(m, part_of[w][col].m);
      const float base = m == -INFINITY ? 0.f : m;
      float l = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
      for (int w = 0; w < JW; ++w) {
        const float f = __builtin_amdgcn_exp2f(part_of[w][col].m - base);
        l = fmaf(part_of[w][col].l, f, l);
        y0 = fmaf(joined[((size_t)w * cols + col) * a.h + d], f, y0);
        y1 = fmaf(joined[((size_t)w * cols + col) * a.h + d + 1], f, y1);
      }
      const int head = head0 + col;
      if (parts > 1) {
        const long long slot = ((long long)s * a.Hq + head) * parts + part;
        *(float2*)(po + slot * a.h + d) = make_float2(y0, y1);
        if (d == 0) pm[slot] = Part{m, l};
      } else {
        const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
        *(uint32_t*)((uint16_t*)a.out + row * a.out_stride + (long long)head * a.h + d) = T::pack(y0 * inv, y1 * inv);
        if (d == 0 && a.lse) a.lse[row * a.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
      }
    }
  }
}

// Adds up the parts of a query head, in their order: a block takes 64 dims, lane d one of them, the waves a part each in turn.  A part's
// share of the sum depends on its maximum alone, so all loads of eight parts are on their way at once.
template <class T>
__global__ __launch_bounds__(TPB) void window_join_kernel(WindowArgs a, int parts) {
  __shared__ float part_sum[4][64];
  const int s = blockIdx.x / a.Hq, head = blockIdx.x - s * a.Hq;
  const Seq q = load_seq(a, s, true);
  if (q.n < 1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.y * 64 + lane;
  const float* po = (const float*)a.ws;
  const Part* pm = (const Part*)(po + (long long)a.S * a.Hq * parts * a.h);
  const long long slot = ((long long)s * a.Hq + head) * parts;
  // (at most 64 parts)
  const Part mine = lane < parts ? pm[slot + lane] : Part{-INFINITY, 0.f};
  float y = 0.f;
  constexpr int AHEAD = 8;
  float v[2][AHEAD];
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int p = wave + 4 * (half * AHEAD + i);
      v[half][i] = p < parts && d < a.h ? po[(slot + p) * a.h + d] : 0.f;
    }
  const float m = wave_max(mine.m), base = m == -INFINITY ? 0.f : m, f = __builtin_amdgcn_exp2f(mine.m - base);
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) y = fmaf(v[half][i], __shfl(f, min(wave + 4 * (half * AHEAD + i), 63), WAVE), y);
  part_sum[wave][lane] = y;
  const float l = wave_sum(mine.l * f);
  __syncthreads();
  if (wave == 0 && d < a.h) {
    const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
    const float sum = (part_sum[0][lane] + part_sum[1][lane] + part_sum[2][lane] + part_sum[3][lane]) * inv;
    ((uint16_t*)a.out)[(long long)q.row0 * a.out_stride + (long long)head * a.h + d] = (uint16_t)T::pack(sum, 0.f);
    if (d == 0 && a.lse) a.lse[(long long)q.row0 * a.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

// Waves to a job and blocks to a job.  Where jobs alone fill the card a wave takes one, which spares the join in LDS (512 sequences of up to
// 576 tokens, 32 kv heads of 80, 16384 jobs: 447 us, 506 with four waves to a job); else four waves share it (64 sequences, 8 kv heads of
// 128, window 1024, 512 jobs: 46 us, 77 with one).  At the border, sequences of 257 to 576 tokens, one wave and four: 1024 jobs 40 and 36 us (80
// dims), 46.1 and 45.6 (128), 33 and 24 (64); 2048 jobs 63 and 68, 82 and 83, 46 and 44; 4096 jobs 120 and 127, 156 and 158, 86 and 82.  Longer
// contexts gain from four beyond it too (1000 to 4000 tokens, 2048 jobs: 371 and 353 us, 504 and 436, 269 and 239).
// Few jobs are parted over blocks until there are 512 of these, each with eight groups of keys or more (one sequence of 32000 tokens, 8 jobs:
// 24 us and 4 for the join with 256, 512 or 1024 blocks, 1250 unparted by single waves; the 512 jobs above in 1024 blocks: 50 us and 8).
constexpr int MAX_PARTS = 64;                 // (window_join_kernel's lanes)
struct Split { int waves, parts, col_blocks; };
Split decode_split(const WindowArgs& a) {
  const int G = a.Hq / a.Hkv, cb = a.h > 128 ? 8 : 16;
  Split r{1, 1, (G + cb - 1) / cb};
  const long long jobs = (long long)a.S * a.Hkv * r.col_blocks;
  long long seen = a.max_total;
  if (a.window && (long long)a.window + a.sinks < seen) seen = (long long)a.window + a.sinks;
  const long long groups = (seen + 31) / 32;
  if (jobs >= 2048 || groups < 2) return r;
  r.waves = 4;
  long long parts = (512 + jobs - 1) / jobs, most = (groups + 7) / 8;
  if (parts > most) parts = most;
  if (parts > MAX_PARTS) parts = MAX_PARTS;
  r.parts = parts < 1 ? 1 : (int)parts;
  return r;
}

long long blocks(const WindowArgs& a, const Split& r) {
  const long long jobs = (long long)a.S * a.Hkv * r.col_blocks * r.parts;
  return r.waves == 1 ? (jobs + 3) / 4 : jobs;
}

template <class T, int HD>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  const Split r = decode_split(a);
  const dim3 grid((unsigned)blocks(a, r));
  const int G = a.Hq / a.Hkv, cb = HD > 128 ? 8 : 16;
  if (r.waves == 1) {
    hipLaunchKernelGGL((window_decode_kernel<T, HD, 1>), grid, dim3(TPB), 0, s, a, r.parts, r.col_blocks);
  } else {
    const size_t lds = (size_t)4 * (G < cb ? G : cb) * a.h * sizeof(float);
    hipLaunchKernelGGL((window_decode_kernel<T, HD, 4>), grid, dim3(TPB), lds, s, a, r.parts, r.col_blocks);
    if (r.parts > 1) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((window_join_kernel<T>), dim3((unsigned)(a.S * a.Hq), (a.h + 63) / 64), dim3(TPB), 0, s, a, r.parts);
    }
  }
  return hipGetLastError();
}
template <class T>
hipError_t by_head(const WindowArgs& a, hipStream_t s) {
  if (a.h <= 64) return launch<T, 64>(a, s);
  if (a.h <= 96) return launch<T, 96>(a, s);
  if (a.h <= 128) return launch<T, 128>(a, s);
  return launch<T, 256>(a, s);
}

}  // namespace

size_t rl_window_decode_bytes(const WindowArgs& a) {
  const Split r = decode_split(a);
  return r.parts > 1 ? (size_t)a.S * a.Hq * r.parts * ((size_t)a.h * sizeof(float) + sizeof(Part)) : 0;
}
long long rl_window_decode_blocks(const WindowArgs& a) { return blocks(a, decode_split(a)); }
hipError_t rl_window_decode(const WindowArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return a.dtype == RLGEN_DTYPE_F16 ? by_head<TypeF16>(a, s) : by_head<TypeBf16>(a, s);
}
