// The loss of pairs of packed sequences, and the C entry points of the learner's operators: what the host can check is checked here, then
// launched.  A pass without rows has no tensors of rows, so their pointers may be null.
#include "../../include/rlgen.h"
#include "learner.h"

#include <cmath>

#define HIPCHK(expr) do { if ((expr) != hipSuccess) return RLGEN_ERR_DEVICE; } while (0)

namespace {

// One block to a prompt: the sums of log pi - log pi_ref over the chosen and the rejected sequence (in 64 bits: thousands of terms of which
// small differences count), the loss, and its gradient on the rows of all k sequences.  Bound by the launch and four waits for memory behind
// each other (index, row start, log-probs, the other sequence's): 512 prompts with two sequences of 64 to 576 rows 4.8 us, 16 with four of 300 to 9000
// 6.6; both sums in one loop and a block to each sequence of few prompts took as long.
template <int T> __global__ __launch_bounds__(T) void dpo_pairs_kernel(PairArgs a) {
  __shared__ double part[2][T / 64];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int* starts = a.row_starts + (long long)b * a.k;
  auto from = [&](int i) { return min(max(starts[i], 0), a.rows); };
  const int which[2] = {min(max(a.pos[b], 0), a.k - 1), min(max(a.neg[b], 0), a.k - 1)};
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int end = from(which[q] + 1);
    double v = 0.0;
#pragma unroll 4
    for (int i = from(which[q]) + threadIdx.x; i < end; i += T) v += (double)a.pol[i] - (double)a.ref[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
    if (lane == 0) part[q][wave] = v;
  }
  __syncthreads();
  double sums[2] = {0.0, 0.0};
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    sums[0] += part[0][w];
    sums[1] += part[1][w];
  }
  const bool same = which[0] == which[1];       // no difference, whatever the log-probs are
  const double x = same ? 0.0 : (double)a.beta * (sums[0] - sums[1]);
  if (threadIdx.x == 0) a.loss[b] = (float)(fmax(-x, 0.0) + log1p(exp(-fabs(x))));
  const float step = (float)((double)a.weight * a.beta / (1.0 + exp(x)));
  for (int i = 0; i < a.k; ++i) {
    // (chosen, not multiplied: a step of NaN or infinity is the pair's alone)
    const float g = same ? 0.f : i == which[0] ? -step : i == which[1] ? step : 0.f;
    const int end = from(i + 1);
    for (int r = from(i) + threadIdx.x; r < end; r += T) a.grad[r] = g;
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
bool type_ok(int dtype) { return dtype >= RLGEN_DTYPE_F32 && dtype <= RLGEN_DTYPE_F16; }
// rows of `width` elements with 16-byte accesses (8 bytes of 8-bit elements)
bool rows_ok(const void* p, int64_t stride, int width, int dtype) {
  return aligned16(p) && stride >= width && stride % (dtype == RLGEN_DTYPE_F32 ? 4 : 8) == 0 && stride <= INT32_MAX;
}
constexpr int MOST_ROWS = 1 << 23;           // (of up to 512 threads, which have to stay below 2^32)
int add_norm_args(AddNormArgs& a, int dtype, int res_dtype, int rows, int width, double drop_p, const int64_t* rng, const float* gain, float eps) {
  if (drop_p > 0.0 && !rng) return RLGEN_ERR_NULL;
  if (!type_ok(dtype) || (res_dtype != RLGEN_DTYPE_F32 && res_dtype != dtype) || rows < 0 || width < 8 || width % 8 != 0 || width > MOST_WIDTH ||
      !(drop_p >= 0.0 && drop_p <= 1.0) || ((uintptr_t)rng & 7) != 0 || !aligned16(gain) || !std::isfinite(eps) || eps < 0.f || rows >= MOST_ROWS)
    return RLGEN_ERR_BAD_ARG;
  a.dtype = dtype; a.res_dtype = res_dtype; a.rows = rows; a.width = width;
  a.drop = (unsigned)std::lround(drop_p * 65536.0);
  a.keep_scale = a.drop < 65536u ? (float)(65536.0 / (65536.0 - a.drop)) : 0.f;
  a.rng = (const unsigned long long*)rng; a.gain = gain; a.eps = eps;
  return RLGEN_OK;
}
bool logits_ok(const void* p, int64_t stride, int vocab, int dtype) {
  return type_ok(dtype) && ((uintptr_t)p & (dtype == RLGEN_DTYPE_F32 ? 3 : 1)) == 0 && stride >= vocab && stride <= INT32_MAX;
}
constexpr int MOST_VOCAB = 1 << 24;
bool temperature_ok(float t) { return std::isfinite(t) && t >= 1e-6f; }

}  // namespace

hipError_t rl_dpo_pairs(const PairArgs& a, hipStream_t s) {
  if (a.rows / a.B > 2048) hipLaunchKernelGGL((dpo_pairs_kernel<1024>), dim3(a.B), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((dpo_pairs_kernel<256>), dim3(a.B), dim3(256), 0, s, a);
  return hipGetLastError();
}

extern "C" {

int rlgen_add_rms_norm(const void* x, int64_t x_stride, int32_t dtype, const void* residual, int64_t residual_stride, int32_t residual_dtype,
                       int32_t rows, int32_t width, double drop_p, const int64_t* rng, const float* gain, float eps, void* h, int64_t h_stride,
                       void* y, int64_t y_stride, int32_t y_dtype, float* scales, int32_t scale_group, void* hip_stream) {
  AddNormArgs a{};
  const int rc = add_norm_args(a, dtype, residual_dtype, rows, width, drop_p, rng, gain, eps);
  const bool eight = y && y_dtype == RLGEN_DTYPE_E4M3;
  if (rc == RLGEN_ERR_NULL || (rows > 0 && (!x || (!h && !y) || (eight && !scales))) || (y && !gain)) return RLGEN_ERR_NULL;
  if (rc != RLGEN_OK || !rows_ok(x, x_stride, width, dtype) || (residual && !rows_ok(residual, residual_stride, width, residual_dtype)) ||
      (h && !rows_ok(h, h_stride, width, residual_dtype)) || (y && !rows_ok(y, y_stride, width, y_dtype)))
    return RLGEN_ERR_BAD_ARG;
  if (y && !eight && !(dtype == RLGEN_DTYPE_F32 ? type_ok(y_dtype) : y_dtype == dtype)) return RLGEN_ERR_BAD_ARG;
  if (eight && ((scale_group != 0 && scale_group != 32 && scale_group != 64 && scale_group != 128) || !aligned4(scales))) return RLGEN_ERR_BAD_ARG;
  if (!y) a.gain = nullptr;
  a.x = x; a.x_stride = x_stride; a.residual = residual; a.residual_stride = residual_stride;
  a.h = h; a.h_stride = h_stride; a.y = y; a.y_stride = y_stride; a.y_dtype = y_dtype; a.scales = scales; a.scale_group = scale_group;
  HIPCHK(rl_add_norm(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

size_t rlgen_add_rms_norm_backward_workspace(int32_t rows, int32_t width) {
  return rows < 0 || rows >= MOST_ROWS || width < 8 || width % 8 != 0 || width > MOST_WIDTH ? 0 : rl_add_norm_backward_bytes(rows, width);
}
int rlgen_add_rms_norm_backward(const void* h, int64_t h_stride, int32_t residual_dtype, const void* dy, int64_t dy_stride, int32_t dtype,
                                const void* dh, int64_t dh_stride, int32_t rows, int32_t width, double drop_p, const int64_t* rng,
                                const float* gain, float eps, void* dresidual, int64_t dresidual_stride, void* dx, int64_t dx_stride,
                                float* dgain, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AddNormArgs a{};
  const int rc = add_norm_args(a, dtype, residual_dtype, rows, width, drop_p, rng, gain, eps);
  if (rc == RLGEN_ERR_NULL || (gain && (!dgain || (rows > 0 && (!h || !dy)))) || (!gain && (dgain || dy)) ||
      (rows > 0 && ((!dresidual && !dx) || (!gain && !dh))))
    return RLGEN_ERR_NULL;
  if (rc != RLGEN_OK || (h && !rows_ok(h, h_stride, width, residual_dtype)) || (dy && !rows_ok(dy, dy_stride, width, dtype)) ||
      (dh && !rows_ok(dh, dh_stride, width, residual_dtype)) || (dresidual && !rows_ok(dresidual, dresidual_stride, width, residual_dtype)) ||
      (dx && !rows_ok(dx, dx_stride, width, dtype)) || !aligned16(dgain))
    return RLGEN_ERR_BAD_ARG;
  const size_t need = gain ? rl_add_norm_backward_bytes(rows, width) : 0;
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return RLGEN_ERR_WORKSPACE;
  a.h = const_cast<void*>(h); a.h_stride = h_stride; a.dy = dy; a.dy_stride = dy_stride; a.dh = dh; a.dh_stride = dh_stride;
  a.dres = dresidual; a.dres_stride = dresidual_stride; a.dx = dx; a.dx_stride = dx_stride;
  a.dgain = dgain; a.partial = (float*)workspace;
  HIPCHK(rl_add_norm_backward(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

size_t rlgen_token_logprobs_workspace(int32_t dtype, int32_t rows, int32_t vocab, int32_t n_top) {
  if (!type_ok(dtype) || rows < 0 || rows >= MOST_BLOCKS || vocab < 1 || vocab > MOST_VOCAB || n_top < 0 || n_top > MOST_TOP || n_top > vocab) return 0;
  LogprobArgs a{};
  a.dtype = dtype; a.rows = rows; a.vocab = vocab; a.n_top = n_top;
  return rl_token_logprobs_bytes(a);
}
int rlgen_token_logprobs(const void* logits, int64_t stride, int32_t dtype, int32_t rows, int32_t vocab, const int32_t* tokens,
                         float temperature, float* logprobs, float* stats, float* entropy, int32_t n_top, int32_t* top_tokens,
                         float* top_logprobs, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (rows > 0 && (!logits || !stats || (n_top > 0 && (!top_tokens || !top_logprobs)) || !tokens != !logprobs)) return RLGEN_ERR_NULL;
  if (rows < 0 || rows >= MOST_BLOCKS || vocab < 1 || vocab > MOST_VOCAB || n_top < 0 || n_top > MOST_TOP || n_top > vocab ||
      !logits_ok(logits, stride, vocab, dtype) || !temperature_ok(temperature))
    return RLGEN_ERR_BAD_ARG;
  LogprobArgs a{};
  a.dtype = dtype; a.rows = rows; a.vocab = vocab; a.logits = logits; a.stride = stride; a.tokens = tokens; a.temperature = temperature;
  a.logprobs = logprobs; a.stats = stats; a.entropy = entropy; a.n_top = n_top; a.top_tokens = top_tokens; a.top_logprobs = top_logprobs;
  const size_t need = rl_token_logprobs_bytes(a);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return RLGEN_ERR_WORKSPACE;
  HIPCHK(rl_token_logprobs(a, workspace, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

int rlgen_token_logprobs_backward(const void* logits, int64_t stride, int32_t dtype, int32_t rows, int32_t vocab, const int32_t* tokens,
                                  float temperature, const float* stats, const float* entropy, const float* dlogprobs, const float* dentropy,
                                  void* dlogits, int64_t dlogits_stride, void* hip_stream) {
  if (rows > 0 && (!logits || !stats || !dlogits || (!dlogprobs && !dentropy) || (dlogprobs && !tokens) || (dentropy && !entropy))) return RLGEN_ERR_NULL;
  LogprobArgs a{};
  a.dtype = dtype; a.rows = rows; a.vocab = vocab; a.logits = logits; a.stride = stride; a.tokens = tokens; a.temperature = temperature;
  a.stats = const_cast<float*>(stats); a.entropy = const_cast<float*>(entropy); a.g = dlogprobs; a.g_entropy = dentropy;
  a.dlogits = dlogits; a.d_stride = dlogits_stride;
  if (rows < 0 || vocab < 1 || vocab > MOST_VOCAB || !logits_ok(logits, stride, vocab, dtype) || !logits_ok(dlogits, dlogits_stride, vocab, dtype) ||
      !temperature_ok(temperature) || rl_token_logprobs_backward_blocks(a) >= MOST_BLOCKS)
    return RLGEN_ERR_BAD_ARG;
  HIPCHK(rl_token_logprobs_backward(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

int rlgen_dpo_pairs(const float* token_logprobs, const float* ref_logprobs, int32_t rows, const int32_t* row_starts, int32_t B, int32_t k,
                    const int32_t* idx_pos, const int32_t* idx_neg, float beta, float weight, float* loss, float* dlogprobs,
                    void* hip_stream) {
  if ((rows > 0 && (!token_logprobs || !ref_logprobs || !dlogprobs)) || !row_starts || !idx_pos || !idx_neg || !loss) return RLGEN_ERR_NULL;
  if (rows < 0 || rows > INT32_MAX - 1024 || B < 1 || B >= MOST_BLOCKS / 4 || k < 1 || (int64_t)B * k >= INT32_MAX || !std::isfinite(beta) ||
      !std::isfinite(weight))
    return RLGEN_ERR_BAD_ARG;
  PairArgs a{};
  a.pol = token_logprobs; a.ref = ref_logprobs; a.rows = rows; a.row_starts = row_starts; a.B = B; a.k = k;
  a.pos = idx_pos; a.neg = idx_neg; a.beta = beta; a.weight = weight; a.loss = loss; a.grad = dlogprobs;
  HIPCHK(rl_dpo_pairs(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

}  // extern "C"
