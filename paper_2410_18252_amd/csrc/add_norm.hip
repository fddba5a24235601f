// Residual addition with dropout and a root-mean-square norm over rows, and its gradients.
//   h = residual + m x,  y = h / sqrt(mean h^2 + eps) gain
//   d = dh + r (t - h r^2 mean(t h)),  r = 1 / sqrt(mean h^2 + eps),  t = dy gain;   dresidual = d,  dx = m d,  dgain = sum over rows of dy h r
// with m = 0 for a dropped element, else 65536 / (65536 - drop).
#include "learner.h"
#include "../../include/rlgen.h"

namespace {

// The dropout mask is never stored: both passes make it from (seed, offset, row, column) with Philox4x32 of ten rounds (Salmon, Moraes, Dror
// and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).  One call gives 128 bits, 16 for each of eight columns: key = the
// seed's two words, counter = (column / 8, row, the offset's two words).  16 bits an element quantise the drop probability to 2^-16, and
// the factor is the quantised one's, so the expectation is exact; 32 bits would take twice the multiplications.
struct Bits { uint32_t w[4]; };
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ Bits philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = xor3((uint32_t)(b >> 32), c1, k0);
    c1 = (uint32_t)b;
    c2 = xor3((uint32_t)(a >> 32), c3, k1);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}
struct Generator {
  uint32_t k0, k1, o0, o1;
  __device__ __forceinline__ void begin(const unsigned long long* rng) {
    k0 = (uint32_t)rng[0]; k1 = (uint32_t)(rng[0] >> 32);
    o0 = (uint32_t)rng[1]; o1 = (uint32_t)(rng[1] >> 32);
  }
  // the eight elements' factors, applied
  __device__ __forceinline__ void apply(float* x, int vec, int row, unsigned drop, float scale) const {
    const Bits r = philox((uint32_t)vec, (uint32_t)row, o0, o1, k0, k1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = e & 1 ? r.w[e >> 1] >> 16 : r.w[e >> 1] & 0xffffu;
      x[e] = bits >= drop ? x[e] * scale : 0.f;
    }
  }
};

// Sum or maximum over a row's waves: `slot` is the row's own part of LDS
template <bool MAX> __device__ __forceinline__ float over_row(float v, float* slot, int wave, int waves) {
  v = MAX ? lanes_max(v) : lanes_sum(v);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) slot[wave] = v;
  __syncthreads();
  float t = slot[0];
  for (int w = 1; w < waves; ++w) t = MAX ? fmaxf(t, slot[w]) : t + slot[w];
  return t;
}

constexpr int MOST_WAVES = 8;

__device__ __forceinline__ uint32_t pack_e4m3x4(const float* y) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}
constexpr float E4M3_MAX = 448.f;
// A group whose largest magnitude is below this counts as zeros: chosen, far below what a norm gives, so that its scale (from 2^-109 on) and 448 over the
// magnitude (up to 2^109) are normal numbers with room to spare
constexpr float E4M3_LEAST = 7.8886090522101181e-31f;       // 2^-100

// Forward.  A row lies in the registers of `waves` waves, thread t of them holding its 16-byte pieces t, t + 64 waves, ...: read once, written once, the norm
// taken of the 32-bit sum before it is rounded.  Bound by HBM: 16384 rows of 4096 in bf16 with dropout 94 us, 5.7 TB/s (the generator's multiplications
// hide behind it); 7001 of 2560 in fp16 over 32 bits 43.8 us, 4.9 TB/s; 128 rows of 4096 into 8 bits 4.5 us, a launch and two waits.
template <class TX, class TR, int NV>
__global__ __launch_bounds__(512) void add_norm_kernel(AddNormArgs a, int waves) {
  __shared__ float red[2][MOST_WAVES];
  const int wave_all = threadIdx.x >> 6, wave = wave_all % waves, sub = wave_all / waves;
  const int t = wave * 64 + (threadIdx.x & 63), step = waves * 64;
  const int rows_here = blockDim.x / step;
  const int row = blockIdx.x * rows_here + sub;
  if (row >= a.rows) return;                   // only where a row has one wave: no barrier follows
  const int n8 = a.width >> 3;
  float h[NV][8];
  {
    Vec8<TX> x[NV];
    Vec8<TR> r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = t + i * step;
      x[i] = v < n8 ? Vec8<TX>::load(a.x, row * a.x_stride + 8ll * v) : Vec8<TX>::zero();
      r[i] = a.residual && v < n8 ? Vec8<TR>::load(a.residual, row * a.residual_stride + 8ll * v) : Vec8<TR>::zero();
    }
    Generator rng{};
    if (a.drop) rng.begin(a.rng);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float y[8];
      x[i].to(y);
      r[i].to(h[i]);
      if (a.drop) rng.apply(y, t + i * step, row, a.drop, a.keep_scale);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += y[e];
    }
  }
  if (a.h) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (t + i * step < n8) Vec8<TR>::store(a.h, row * a.h_stride + 8ll * (t + i * step), h[i]);
  }
  if (!a.gain) return;
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e], h[i][e], ss);
  ss = over_row<false>(ss, red[0] + sub * waves, wave, waves);
  const float inv = 1.0f / sqrtf(ss / (float)a.width + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = t + i * step;
    if (v >= n8) continue;
    const Vec8<TypeF32> g8 = Vec8<TypeF32>::load(a.gain, 8ll * v);
    float g[8];
    g8.to(g);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * inv * g[e];
  }
  if (a.y_dtype != RLGEN_DTYPE_E4M3) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = t + i * step;
      if (v >= n8) continue;
      const long long at = row * a.y_stride + 8ll * v;
      if (a.y_dtype == RLGEN_DTYPE_BF16) Vec8<TypeBf16>::store(a.y, at, h[i]);
      else if (a.y_dtype == RLGEN_DTYPE_F16) Vec8<TypeF16>::store(a.y, at, h[i]);
      else Vec8<TypeF32>::store(a.y, at, h[i]);
    }
    return;
  }
  // 8 bits: scale = largest magnitude / 448, of the row or of scale_group columns (4, 8 or 16 lanes next to each other)
  float most[NV], row_most = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    most[i] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most[i] = fmaxf(most[i], fabsf(h[i][e]));
    row_most = fmaxf(row_most, most[i]);
  }
  if (a.scale_group == 0) {
    row_most = over_row<true>(row_most, red[1] + sub * waves, wave, waves);
#pragma unroll
    for (int i = 0; i < NV; ++i) most[i] = row_most;
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      for (int o = 1; o < a.scale_group / 8; o <<= 1) most[i] = fmaxf(most[i], __shfl_xor(most[i], o, WAVE));
  }
  const int groups = a.scale_group ? (a.width + a.scale_group - 1) / a.scale_group : 1;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = t + i * step;
    if (v >= n8) continue;
    const bool some = most[i] >= E4M3_LEAST;
    const float f = some ? E4M3_MAX / most[i] : 0.f;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = h[i][e] * f;
    u32x2 w;
    w[0] = pack_e4m3x4(y);
    w[1] = pack_e4m3x4(y + 4);
    *(u32x2*)((uint8_t*)a.y + row * a.y_stride + 8ll * v) = w;
    const float scale = some ? most[i] / E4M3_MAX : 0.f;
    if (a.scale_group == 0) {
      if (v == 0) a.scales[row] = scale;
    } else if (v % (a.scale_group / 8) == 0) {
      a.scales[(long long)row * groups + v / (a.scale_group / 8)] = scale;
    }
  }
}

// The backward pass: a block walks rows in turn (rows_here of them beside each other where a row takes few waves), the next ones requested ahead, its
// threads on the same columns throughout, so that the gain's gradient is summed in registers; the rows beside each other meet in LDS, and a
// second launch adds up the blocks in their order.  Bound by HBM: 16384 rows of 4096 in bf16 with dropout 112 us, 3001 of 2048 in fp16 over 32 bits 19 us, 5 us
// more for the second launch.
template <class TX, class TR, int NV, bool ONCE>
__global__ __launch_bounds__(512) void add_norm_backward_kernel(AddNormArgs a, int waves) {
  __shared__ float red[2][2][MOST_WAVES];
  __shared__ __attribute__((aligned(16))) float sums[NV == 1 ? 512 * 8 : 1];
  const int wave_all = threadIdx.x >> 6, wave = wave_all % waves, sub = wave_all / waves;
  const int t = wave * 64 + (threadIdx.x & 63), step = waves * 64;
  const int rows_here = blockDim.x / step;
  const int n8 = a.width >> 3;
  const float inv_width = 1.0f / (float)a.width;
  Generator rng{};
  if (a.drop) rng.begin(a.rng);
  float gain[NV][8], sum[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = t + i * step;
    (a.gain && v < n8 ? Vec8<TypeF32>::load(a.gain, 8ll * v) : Vec8<TypeF32>::zero()).to(gain[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[i][e] = 0.f;
  }
  struct Raw { Vec8<TR> h[NV], dh[NV]; Vec8<TX> dy[NV]; };
  auto load = [&](int row, Raw& w) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = t + i * step;
      const bool on = v < n8 && row < a.rows;
      w.h[i] = on && a.gain ? Vec8<TR>::template load<ONCE>(a.h, row * a.h_stride + 8ll * v) : Vec8<TR>::zero();
      w.dy[i] = on && a.gain ? Vec8<TX>::template load<ONCE>(a.dy, row * a.dy_stride + 8ll * v) : Vec8<TX>::zero();
      w.dh[i] = on && a.dh ? Vec8<TR>::template load<ONCE>(a.dh, row * a.dh_stride + 8ll * v) : Vec8<TR>::zero();
    }
  };
  const int row_step = gridDim.x * rows_here;
  int turn = 0;
  Raw now, next;
  load(blockIdx.x * rows_here + sub, now);
  for (int first = blockIdx.x * rows_here; first < a.rows; first += row_step, turn ^= 1) {
    const int row = first + sub;
    load(row + row_step, next);
    float inv = 0.f, back = 0.f;
    if (a.gain) {
      float ss = 0.f, th = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float h[8], dy[8];
        now.h[i].to(h);
        now.dy[i].to(dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss = fmaf(h[e], h[e], ss);
          th = fmaf(dy[e] * gain[i][e], h[e], th);
        }
      }
      ss = lanes_sum(ss);
      th = lanes_sum(th);
      if (waves > 1) {
        if ((threadIdx.x & 63) == 0) { red[turn][0][wave_all] = ss; red[turn][1][wave_all] = th; }
        __syncthreads();
        ss = th = 0.f;
        for (int w = sub * waves; w < (sub + 1) * waves; ++w) { ss += red[turn][0][w]; th += red[turn][1][w]; }
      }
      if (row < a.rows) {                        // (past the last row there are zeros, and eps may be 0)
        inv = 1.0f / sqrtf(ss * inv_width + a.eps);
        back = inv * inv * (th * inv_width);
      }
    }
    // (the values are widened again: kept as they are they would take twice the registers, and half the waves)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      now.h[i].opaque();
      now.dy[i].opaque();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float h[8], dy[8], d[8];
      now.h[i].to(h);
      now.dy[i].to(dy);
      now.dh[i].to(d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum[i][e] = fmaf(dy[e], h[e] * inv, sum[i][e]);
        d[e] = fmaf(inv, dy[e] * gain[i][e] - h[e] * back, d[e]);
      }
      const int v = t + i * step;
      if (v >= n8 || row >= a.rows) continue;
      if (a.dres) Vec8<TR>::template store<ONCE>(a.dres, row * a.dres_stride + 8ll * v, d);
      if (a.dx) {
        if (a.drop) rng.apply(d, v, row, a.drop, a.keep_scale);
        Vec8<TX>::template store<ONCE>(a.dx, row * a.dx_stride + 8ll * v, d);
      }
    }
    now = next;
  }
  if (!a.dgain) return;
  float* to = gridDim.x == 1 ? a.dgain : a.partial + (long long)blockIdx.x * a.width;
  if (NV == 1 && rows_here > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x * 8 + e] = sum[0][e];
    __syncthreads();
    for (int d = threadIdx.x; d < a.width; d += blockDim.x) {
      float v = 0.f;
      for (int r = 0; r < rows_here; ++r) v += sums[r * step * 8 + d];
      to[d] = v;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = t + i * step;
    if (v < n8) Vec8<TypeF32>::store(to, 8ll * v, sum[i]);
  }
}

// dgain over the parts: 32 columns to a block, 32 runs of parts at once and then the runs, in one order
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* partial, int parts, int width, float* dgain) {
  __shared__ float red[32][33];
  const int col = threadIdx.x & 31, run = threadIdx.x >> 5, d = blockIdx.x * 32 + col;
  float v = 0.f;
  if (d < width)
#pragma unroll 8
    for (int p = run; p < parts; p += 32) v += partial[(long long)p * width + d];
  red[run][col] = v;
  __syncthreads();
  if (run == 0 && d < width) {
    for (int p = 1; p < 32; ++p) v += red[p][col];
    dgain[d] = v;
  }
}

// 16-byte pieces of a thread, waves to a row and rows to a block: by the width alone, so that a row's sums do not depend on how many rows there are.
// Forward (16384 rows of 4096 in bf16 with dropout, us): one piece 97, two 95, four 98, eight 110.  Backward, whose sums and requests ahead take
// 88 to 111 registers with one piece to a thread, 143 to 185 with two and all 256 with four (63 more in scratch where the residual stream is fp32, 113 where x
// is too): one piece while eight waves hold a row.  4000 rows of bf16 over bf16 | bf16 over fp32 | fp32 with dh, us, and their bytes at 5.08 TB/s: 4096
// columns 38 | 57 | 72 (32 | 52 | 65), 5120 50 | 74 | 90 (40 | 65 | 81), 8192 70 | 110 | 139 (65 | 103 | 129), 8200 76 | 181 | 222 (65 | 103 | 129),
// 16384 126 | 253 | 337 (129 | 206 | 258).
struct Shape { int nv, waves, rows_here; };
Shape shape_of(int width, bool backward) {
  const int n8 = (width + 7) / 8;
  Shape s;
  if (backward) s.nv = n8 <= 512 ? 1 : n8 <= 1024 ? 2 : 4;
  else s.nv = n8 <= 64 ? 1 : n8 <= 1024 ? 2 : 4;
  s.waves = (n8 + 64 * s.nv - 1) / (64 * s.nv);
  s.rows_here = backward ? (s.nv == 1 ? 8 / s.waves : 1) : s.waves == 1 ? 4 : 1;
  return s;
}
// The same number of blocks on every CU: as many as it holds at once with one piece to a thread, one with two or four pieces (16384 rows of 4096 in bf16 with dropout: 108 us with two blocks of eight waves to a
// CU, 145, 126, 125 and 113 with one, 1.5, three and four; 2560: 97 to 80 with 410 to 614 blocks of five waves, 95 with 819)
// Up to four walks of rows one block takes alone: its sums are the gain's gradient, and there is neither a second launch nor a workspace (a call of 24
// rows of 128 or 4 of 4096: 8.4 us, 13 with them; 8 of 4096 13.4 in one block, 64 of 512 10.5, 16 of 4096 25).
int backward_blocks(int rows, const Shape& s) {
  if (rows <= 4 * s.rows_here) return 1;
  const int here = s.waves * s.rows_here, per_cu = s.nv == 1 ? 16 / here : s.nv == 2 ? 8 / here : 1;
  const int blocks = (rows + s.rows_here - 1) / s.rows_here, most = 256 * (per_cu < 1 ? 1 : per_cu);
  return blocks < most ? blocks : most;
}

template <class TX, class TR>
hipError_t launch(const AddNormArgs& a, bool backward, hipStream_t s) {
  const Shape f = shape_of(a.width, backward);
  const dim3 block(64 * f.waves * f.rows_here), grid(backward ? backward_blocks(a.rows, f) : (a.rows + f.rows_here - 1) / f.rows_here);
  // backward past the caches (16384 rows of 4096 in bf16, 671 MB: 130 us without, 118 with; forward it is 94 without, 101 with)
  const double bytes = (double)a.rows * a.width * (2 * (a.dtype == RLGEN_DTYPE_F32 ? 4 : 2) + 3 * (a.res_dtype == RLGEN_DTYPE_F32 ? 4 : 2));
#define ADD_NORM(NV) do { \
    if (backward && bytes > CACHE_BYTES) hipLaunchKernelGGL((add_norm_backward_kernel<TX, TR, NV, true>), grid, block, 0, s, a, f.waves); \
    else if (backward) hipLaunchKernelGGL((add_norm_backward_kernel<TX, TR, NV, false>), grid, block, 0, s, a, f.waves); \
    else hipLaunchKernelGGL((add_norm_kernel<TX, TR, NV>), grid, block, 0, s, a, f.waves); } while (0)
  if (f.nv == 1) ADD_NORM(1);
  else if (f.nv == 2) ADD_NORM(2);
  else ADD_NORM(4);
#undef ADD_NORM
  return hipGetLastError();
}
hipError_t by_type(const AddNormArgs& a, bool backward, hipStream_t s) {
  switch (a.dtype) {
    case RLGEN_DTYPE_F32: return launch<TypeF32, TypeF32>(a, backward, s);
    case RLGEN_DTYPE_BF16: return a.res_dtype == RLGEN_DTYPE_F32 ? launch<TypeBf16, TypeF32>(a, backward, s) : launch<TypeBf16, TypeBf16>(a, backward, s);
    case RLGEN_DTYPE_F16: return a.res_dtype == RLGEN_DTYPE_F32 ? launch<TypeF16, TypeF32>(a, backward, s) : launch<TypeF16, TypeF16>(a, backward, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t rl_add_norm(const AddNormArgs& a, hipStream_t s) { return a.rows <= 0 ? hipSuccess : by_type(a, false, s); }
size_t rl_add_norm_backward_bytes(int rows, int width) {
  const Shape f = shape_of(width, true);
  const int blocks = backward_blocks(rows, f);
  return blocks == 1 ? 0 : (size_t)blocks * width * sizeof(float);
}
hipError_t rl_add_norm_backward(const AddNormArgs& a, hipStream_t s) {
  const Shape f = shape_of(a.width, true);
  const int blocks = a.rows > 0 ? backward_blocks(a.rows, f) : 0;
  if (blocks > 0) {
    const hipError_t e = by_type(a, true, s);
    if (e != hipSuccess) return e;
  }
  if (a.dgain && blocks != 1) hipLaunchKernelGGL(gain_sum_kernel, dim3((a.width + 31) / 32), dim3(1024), 0, s, a.partial, blocks, a.width, a.dgain);
  return hipGetLastError();
}
