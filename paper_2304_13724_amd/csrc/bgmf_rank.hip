// Log probabilities of given items with entropy and top alternatives
// (bgmf_log_probs), and their gradient (bgmf_log_probs_grad).
#include <algorithm>
#include <cmath>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// Score of item j, -inf where it is excluded.
template <class T>
__device__ __forceinline__ float score(const T *x, const uint8_t *ex, int64_t j) {
  return ex && ex[j] ? -INFINITY : to_float(x[j]);
}

template <class Op>
__device__ float block_reduce(float v, float *lds, Op op) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = op(v, __shfl_xor(v, o));
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  float r = lds[0];
  for (int w = 1; w < kThreads / 64; ++w) r = op(r, lds[w]);
  return r;
}

struct LogProbs {
  const void *x;
  const uint8_t *ex;
  const int32_t *given;
  int64_t rows, cols, stride, ex_stride;
  float temperature;
  int32_t top;
  float *log_prob, *entropy, *row_max, *row_sum;
  int32_t *top_item;
  float *top_log_prob;
};

template <class T>
__global__ void __launch_bounds__(kThreads) k_log_probs(LogProbs P) {
  __shared__ float lds[kThreads / 64];
  const auto add = [](float a, float b) { return a + b; };
  const auto most = [](float a, float b) { return fmaxf(a, b); };
  const float c = kLog2e / P.temperature;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(P.x) + r * P.stride;
    const uint8_t *ex = P.ex ? P.ex + r * P.ex_stride : nullptr;
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < P.cols; j += kThreads) m = fmaxf(m, score(x, ex, j));
    m = block_reduce(m, lds, most);
    const float m0 = m == -INFINITY ? 0.0f : m;
    double ts = 0.0, tw = 0.0;  // of many equal terms: 32 bits would lose a unit at each
    for (int64_t j = threadIdx.x; j < P.cols; j += kThreads) {
      const float d = (score(x, ex, j) - m0) * c, e = exp2f(d);
      ts += e;
      tw += e * fmaxf(d, -200.0f);
    }
    const float s = block_reduce((float)ts, lds, add), w = block_reduce((float)tw, lds, add);
    const float log_s = logf(s);
    if (threadIdx.x == 0) {
      if (P.row_max) P.row_max[r] = m;
      if (P.row_sum) P.row_sum[r] = s;
      if (P.entropy) P.entropy[r] = s == 0.0f ? 0.0f : log_s - w * kLn2 / s;
      if (P.log_prob) {
        const int64_t g = P.given[r];
        float lp = 0.0f;
        if (g < -1 || g >= P.cols) lp = NAN;
        else if (g >= 0)
          lp = s == 0.0f ? -INFINITY : (score(x, ex, g) - m) / P.temperature - log_s;
        P.log_prob[r] = lp;
      }
    }
    // alternatives one by one: the largest score after the last one taken
    float last = INFINITY;
    int64_t last_j = -1;
    for (int i = 0; i < P.top; ++i) {
      float best = -INFINITY;
      int64_t at = P.cols;
      for (int64_t j = threadIdx.x; j < P.cols; j += kThreads) {
        const float v = score(x, ex, j);
        if ((v < last || (v == last && j > last_j)) && v > best) best = v, at = j;
      }
      const float all = block_reduce(best, lds, most);
      __shared__ int first;
      if (threadIdx.x == 0) first = 0x7FFFFFFF;
      __syncthreads();
      if (best == all && all > -INFINITY) atomicMin(&first, (int)at);
      __syncthreads();
      last = all, last_j = first;
      if (threadIdx.x == 0) {
        const bool some = all > -INFINITY;
        P.top_item[r * P.top + i] = some ? first : -1;
        P.top_log_prob[r * P.top + i] = some ? (all - m) / P.temperature - log_s : -INFINITY;
      }
      __syncthreads();
    }
  }
}

struct LogProbsGrad {
  const void *x;
  const uint8_t *ex;
  const int32_t *given;
  int64_t rows, cols, stride, ex_stride, out_stride;
  float temperature;
  const float *row_max, *row_sum, *entropy, *g_log_prob, *g_entropy;
  void *out;
};

template <class T>
__global__ void __launch_bounds__(kThreads) k_log_probs_grad(LogProbsGrad P) {
  const float c = kLog2e / P.temperature;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(P.x) + r * P.stride;
    const uint8_t *ex = P.ex ? P.ex + r * P.ex_stride : nullptr;
    T *out = static_cast<T *>(P.out) + r * P.out_stride;
    const float m = P.row_max[r], s = P.row_sum[r];
    const int64_t g = P.given ? P.given[r] : -1;
    float gl = P.g_log_prob && g != -1 ? P.g_log_prob[r] / P.temperature : 0.0f;
    if (g < -1 || g >= P.cols) gl = NAN;
    const float gh = P.g_entropy ? P.g_entropy[r] / P.temperature : 0.0f;
    const float h = P.g_entropy ? P.entropy[r] : 0.0f, log_s = logf(s);
    for (int64_t j = threadIdx.x; j < P.cols; j += kThreads) {
      float v = 0.0f;
      if (!(ex && ex[j]) && s != 0.0f) {
        const float d = (to_float(x[j]) - m) * c, p = exp2f(d) / s;
        v = -gl * p;
        if (P.g_entropy) v -= gh * p * (fmaxf(d, -200.0f) * kLn2 - log_s + h);
        if (j == g) v += gl;
      }
      out[j] = from_float<T>(v);
    }
  }
}

constexpr int64_t kMostGroups = 1 << 20;

template <template <class> class Launch, class P>
hipError_t by_type(int32_t type, const P &p, hipStream_t stream) {
  if (type == BGMF_TYPE_F32) Launch<float>::go(p, stream);
  else if (type == BGMF_TYPE_BF16) Launch<bf16_t>::go(p, stream);
  else Launch<f16_t>::go(p, stream);
  return hipGetLastError();
}

template <class T>
struct RunLogProbs {
  static void go(const LogProbs &p, hipStream_t stream) {
    const unsigned groups = (unsigned)std::min(p.rows, kMostGroups);
    hipLaunchKernelGGL(k_log_probs<T>, dim3(groups), dim3(kThreads), 0, stream, p);
  }
};
template <class T>
struct RunLogProbsGrad {
  static void go(const LogProbsGrad &p, hipStream_t stream) {
    const unsigned groups = (unsigned)std::min(p.rows, kMostGroups);
    hipLaunchKernelGGL(k_log_probs_grad<T>, dim3(groups), dim3(kThreads), 0, stream, p);
  }
};

// The checks both calls share; 0 if the arguments are valid.
int check_scores(const char *call, const void *scores, int32_t type, int64_t rows, int64_t cols,
                 int64_t stride, const uint8_t *excluded, int64_t excluded_stride, float t) {
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: rows and cols must be in [0, 2^31): %lld x %lld", call,
                     (long long)rows, (long long)cols);
  if (!(t > 0.0f) || !std::isfinite(t) || !std::isfinite(kLog2e / t))
    return fail_call(BGMF_E_ARG, "%s: the temperature must be positive and finite: %g", call, t);
  if (bad_matrix(scores, rows, cols, stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad scores (pointer, alignment or row stride %lld)", call,
                     (long long)stride);
  if (excluded && bad_matrix(excluded, rows, cols, excluded_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad excluded (row stride %lld)", call,
                     (long long)excluded_stride);
  return 0;
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int64_t bgmf_log_probs_workspace(int64_t rows, int64_t cols, int32_t top) {
  (void)rows, (void)cols, (void)top;
  return 0;
}

int bgmf_log_probs(const void *scores, int32_t type, int64_t rows, int64_t cols,
                   int64_t row_stride, const uint8_t *excluded, int64_t excluded_stride,
                   const int32_t *given, float temperature, int32_t top, float *log_prob,
                   float *entropy, float *row_max, float *row_sum, int32_t *top_item,
                   float *top_log_prob, void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_log_probs";
  if (const int rc = check_scores(call, scores, type, rows, cols, row_stride, excluded,
                                  excluded_stride, temperature))
    return rc;
  if (top < 0 || top > BGMF_TOP_MAX)
    return fail_call(BGMF_E_ARG, "%s: top must be in [0, %d]: %d", call, BGMF_TOP_MAX, top);
  if (rows == 0) return BGMF_OK;
  if (log_prob && !given) return fail_call(BGMF_E_ARG, "%s: log_prob needs given", call);
  if (top && (!top_item || !top_log_prob))
    return fail_call(BGMF_E_ARG, "%s: top needs top_item and top_log_prob", call);
  (void)ws, (void)ws_bytes;
  const LogProbs p{scores, excluded, given, rows, cols, row_stride, excluded_stride, temperature,
                   top, log_prob, entropy, row_max, row_sum, top_item, top_log_prob};
  const hipError_t e = by_type<RunLogProbs>(type, p, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int bgmf_log_probs_grad(const void *scores, int32_t type, int64_t rows, int64_t cols,
                        int64_t row_stride, const uint8_t *excluded, int64_t excluded_stride,
                        const int32_t *given, float temperature, const float *row_max,
                        const float *row_sum, const float *entropy, const float *grad_log_prob,
                        const float *grad_entropy, void *grad_scores, int64_t grad_stride,
                        void *hip_stream) {
  const char *call = "bgmf_log_probs_grad";
  if (const int rc = check_scores(call, scores, type, rows, cols, row_stride, excluded,
                                  excluded_stride, temperature))
    return rc;
  if (bad_matrix(grad_scores, rows, cols, grad_stride, cols, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad grad_scores (pointer, alignment or row stride %lld)",
                     call, (long long)grad_stride);
  if (rows == 0 || cols == 0) return BGMF_OK;
  if (!row_max || !row_sum) return fail_call(BGMF_E_ARG, "%s: null row_max or row_sum", call);
  if (grad_log_prob && !given) return fail_call(BGMF_E_ARG, "%s: grad_log_prob needs given", call);
  if (grad_entropy && !entropy)
    return fail_call(BGMF_E_ARG, "%s: grad_entropy needs entropy", call);
  if (grad_scores == scores && grad_stride != row_stride && rows > 1)
    return fail_call(BGMF_E_ARG, "%s: in place, the row strides must be equal", call);
  const LogProbsGrad p{scores, excluded, given, rows, cols, row_stride, excluded_stride,
                       grad_stride, temperature, row_max, row_sum, entropy, grad_log_prob,
                       grad_entropy, grad_scores};
  const hipError_t e = by_type<RunLogProbsGrad>(type, p, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
