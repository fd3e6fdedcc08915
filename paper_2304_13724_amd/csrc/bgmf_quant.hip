// Rows in 8-bit integers (bgmf_quantize_rows) and the product of two such
// matrices with their scales (bgmf_quantized_scores).
#include <algorithm>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostGroups = 1 << 20;

// One wave per row.
template <class T>
__global__ void __launch_bounds__(kThreads) k_quantize(const T *x, int64_t rows, int64_t k,
                                                       int64_t stride, int8_t *q, int64_t q_stride,
                                                       float *scale) {
  const int lane = threadIdx.x % 64;
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64; r < rows;
       r += (int64_t)gridDim.x * (kThreads / 64)) {
    const T *row = x + r * stride;
    float most = 0.0f;
    bool bad = false;
    for (int64_t i = lane; i < k; i += 64) {
      const float v = fabsf(to_float(row[i]));
      bad |= !(v < INFINITY);
      most = fmaxf(most, v);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    bad = __any(bad);
    const float s = most / 127.0f;
    if (lane == 0) scale[r] = bad ? NAN : s;
    for (int64_t i = lane; i < k; i += 64) {
      const float v = s > 0.0f && !bad ? rintf(to_float(row[i]) / s) : 0.0f;
      q[r * q_stride + i] = (int8_t)fminf(fmaxf(v, -127.0f), 127.0f);
    }
  }
}

template <class T>
hipError_t quantize(const void *x, int64_t rows, int64_t k, int64_t stride, int8_t *q,
                    int64_t q_stride, float *scale, hipStream_t stream) {
  const unsigned groups =
      (unsigned)std::min<int64_t>((rows + kThreads / 64 - 1) / (kThreads / 64), kMostGroups);
  hipLaunchKernelGGL(k_quantize<T>, dim3(groups), dim3(kThreads), 0, stream,
                     static_cast<const T *>(x), rows, k, stride, q, q_stride, scale);
  return hipGetLastError();
}

hipError_t quantize_by_type(int32_t type, const void *x, int64_t rows, int64_t k, int64_t stride,
                            int8_t *q, int64_t q_stride, float *scale, hipStream_t stream) {
  if (type == BGMF_TYPE_F32) return quantize<float>(x, rows, k, stride, q, q_stride, scale, stream);
  if (type == BGMF_TYPE_BF16)
    return quantize<bf16_t>(x, rows, k, stride, q, q_stride, scale, stream);
  return quantize<f16_t>(x, rows, k, stride, q, q_stride, scale, stream);
}

struct Product {
  const int8_t *a;  // rows x k
  const float *a_scale;
  int64_t rows, k, a_stride;
  const int8_t *b;  // items x k
  const float *b_scale;
  int64_t items, b_stride;
  void *out;
  int64_t out_stride;
};

// One thread per score.
template <class O>
__global__ void __launch_bounds__(kThreads) k_product(Product P) {
  const int64_t tiles = (P.items + kThreads - 1) / kThreads;
  for (int64_t t = blockIdx.x; t < tiles * P.rows; t += gridDim.x) {
    const int64_t r = t / tiles, j = t % tiles * kThreads + threadIdx.x;
    if (j >= P.items) continue;
    const int8_t *a = P.a + r * P.a_stride, *b = P.b + j * P.b_stride;
    int32_t sum = 0;
    for (int64_t i = 0; i < P.k; ++i) sum += (int32_t)a[i] * b[i];
    static_cast<O *>(P.out)[r * P.out_stride + j] =
        from_float<O>((float)sum * P.a_scale[r] * P.b_scale[j]);
  }
}

template <class O>
hipError_t product(const Product &p, hipStream_t stream) {
  const int64_t tiles = (p.items + kThreads - 1) / kThreads * p.rows;
  hipLaunchKernelGGL(k_product<O>, dim3((unsigned)std::min(tiles, kMostGroups)), dim3(kThreads), 0,
                     stream, p);
  return hipGetLastError();
}

// The workspace of rows quantised within a call: bytes, then scales.
int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int bgmf_quantize_rows(const void *x, int32_t type, int64_t rows, int64_t k, int64_t row_stride,
                       int8_t *q, int64_t q_stride, float *scale, void *hip_stream) {
  const char *call = "bgmf_quantize_rows";
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (rows < 0 || rows >= (1ll << 31) || k < 1 || k >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: rows must be in [0, 2^31) and k in [1, 2^31): %lld x %lld",
                     call, (long long)rows, (long long)k);
  if (bad_matrix(x, rows, k, row_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (bad_matrix(q, rows, k, q_stride, k, 1))
    return fail_call(BGMF_E_ARG, "%s: bad q (pointer or row stride %lld)", call,
                     (long long)q_stride);
  if (rows == 0) return BGMF_OK;
  if (!scale) return fail_call(BGMF_E_ARG, "%s: null scale", call);
  const hipError_t e = quantize_by_type(type, x, rows, k, row_stride, q, q_stride, scale,
                                        static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int64_t bgmf_quantized_scores_workspace(int64_t rows, int64_t item_count, int64_t k,
                                        int32_t type) {
  if (type == BGMF_TYPE_I8 || rows <= 0 || k <= 0 || item_count <= 0 || rows >= (1ll << 31) ||
      k > BGMF_PRODUCT_K_MAX)
    return 0;
  return padded(rows * k) + padded(rows * 4);
}

int bgmf_quantized_scores(const void *x, int32_t type, int64_t rows, int64_t k,
                          int64_t row_stride, const float *row_scale, const int8_t *items,
                          int64_t item_count, int64_t items_stride, const float *item_scale,
                          void *out, int32_t out_type, int64_t out_stride, void *ws,
                          int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_quantized_scores";
  if (type != BGMF_TYPE_I8 && !is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be I8, F32, BF16 or F16: %d", call, type);
  if (!is_float_type(out_type))
    return fail_call(BGMF_E_ARG, "%s: out_type must be F32, BF16 or F16: %d", call, out_type);
  if (rows < 0 || item_count < 0 || rows >= (1ll << 31) || item_count >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: rows and item_count must be in [0, 2^31): %lld, %lld", call,
                     (long long)rows, (long long)item_count);
  if (k < 1 || k > BGMF_PRODUCT_K_MAX)
    return fail_call(BGMF_E_ARG, "%s: k must be in [1, %d]: %lld", call, BGMF_PRODUCT_K_MAX,
                     (long long)k);
  if (rows == 0 || item_count == 0) return BGMF_OK;
  if (bad_matrix(x, rows, k, row_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (bad_matrix(items, item_count, k, items_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad items (pointer or row stride %lld)", call,
                     (long long)items_stride);
  if (bad_matrix(out, rows, item_count, out_stride, item_count, type_bytes(out_type)))
    return fail_call(BGMF_E_ARG, "%s: bad out (pointer, alignment or row stride %lld)", call,
                     (long long)out_stride);
  if (!item_scale) return fail_call(BGMF_E_ARG, "%s: null item_scale", call);
  if ((type == BGMF_TYPE_I8) != (row_scale != nullptr))
    return fail_call(BGMF_E_ARG, "%s: row_scale goes with rows of type I8 and with no other", call);
  const int64_t need = bgmf_quantized_scores_workspace(rows, item_count, k, type);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 256))
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  Product p{static_cast<const int8_t *>(x), row_scale, rows, k, row_stride, items, item_scale,
            item_count, items_stride, out, out_stride};
  hipError_t e = hipSuccess;
  if (type != BGMF_TYPE_I8) {
    int8_t *q = static_cast<int8_t *>(ws);
    float *scale = reinterpret_cast<float *>(q + padded(rows * k));
    e = quantize_by_type(type, x, rows, k, row_stride, q, k, scale, stream);
    p.a = q, p.a_scale = scale, p.a_stride = k;
  }
  if (e == hipSuccess)
    e = out_type == BGMF_TYPE_F32    ? product<float>(p, stream)
        : out_type == BGMF_TYPE_BF16 ? product<bf16_t>(p, stream)
                                     : product<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
