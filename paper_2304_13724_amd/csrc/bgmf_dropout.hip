// Dropout from a counter-based generator (bgmf_dropout): no mask is stored, the
// gradient draws the same words again.
#include <algorithm>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;

// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, 2011): four words
// for a counter, whose two upper words are 0 here.  The round keys depend on
// the seed alone (scalar registers).
struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t counter, uint64_t seed) {
  uint32_t x0 = (uint32_t)counter, x1 = (uint32_t)(counter >> 32), x2 = 0, x3 = 0;
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
    x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
    x1 = (uint32_t)b;
    x3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{x0, x1, x2, x3}};
}

struct Dropout {
  const void *x;
  void *out;
  int64_t rows, cols, stride, out_stride;
  uint64_t seed, offset;
  const uint64_t *more;  // added to offset
  uint32_t least;        // words below are dropped
  bool all;              // p = 1
  float factor;
};

template <class T>
__device__ __forceinline__ T dropped(const Dropout &P, uint32_t word, T x) {
  return from_float<T>(word >= P.least && !P.all ? to_float(x) * P.factor : 0.0f);
}

// Elements in one row (a dense tensor): a thread takes 16-byte vectors, one or
// two counters each.  Bound: 480,000 x 64 bf16 take 24.5 us: HBM, 5.0 TB/s, a large
// copy's rate, and the vector units, at work 92% of the cycles (23 instructions an
// element, 15 of them a quarter of a counter's ten rounds).  4,096 x 64 fp32 2.4 us:
// latency.
template <class T>
__global__ void __launch_bounds__(kThreads) k_dropout(Dropout P) {
  constexpr int N = Vec<T>::N;
  const uint64_t offset = P.offset + (P.more ? *P.more : 0);
  const T *x = static_cast<const T *>(P.x);
  T *out = static_cast<T *>(P.out);
  const int64_t vecs = P.cols / N;
  for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v <= vecs;
       v += (int64_t)gridDim.x * kThreads) {
    const int64_t i = v * N;
    if (v < vecs) {
      Vec<T> a = load_vec(x + i);
#pragma unroll
      for (int h = 0; h < N / 4; ++h) {
        const Words w = philox(offset + (uint64_t)(i / 4 + h), P.seed);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.v[h * 4 + e] = dropped<T>(P, w.w[e], a.v[h * 4 + e]);
      }
      store_vec(out + i, a);
    } else {
      for (int64_t j = i; j < P.cols; j += 4) {
        const Words w = philox(offset + (uint64_t)(j / 4), P.seed);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < P.cols) out[j + e] = dropped<T>(P, w.w[e], x[j + e]);
      }
    }
  }
}

// Rows that are apart: a thread takes a counter's four elements, which may lie
// in several rows (element by element, with two 64-bit divisions a counter).
template <class T>
__global__ void __launch_bounds__(kThreads) k_dropout_rows(Dropout P) {
  const uint64_t offset = P.offset + (P.more ? *P.more : 0);
  const int64_t count = P.rows * P.cols, counters = (count + 3) / 4;
  for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v < counters;
       v += (int64_t)gridDim.x * kThreads) {
    const Words w = philox(offset + (uint64_t)v, P.seed);
    int64_t r = v * 4 / P.cols, c = v * 4 % P.cols;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (r < P.rows)
        static_cast<T *>(P.out)[r * P.out_stride + c] =
            dropped<T>(P, w.w[e], static_cast<const T *>(P.x)[r * P.stride + c]);
      if (++c == P.cols) c = 0, ++r;
    }
  }
}

template <class T>
hipError_t dropout(Dropout p, hipStream_t stream) {
  constexpr int64_t kMost = 1 << 20;
  if (p.rows > 1 && p.stride == p.cols && p.out_stride == p.cols) p.cols *= p.rows, p.rows = 1;
  if (p.rows == 1) {
    const int64_t groups = (p.cols / Vec<T>::N + kThreads) / kThreads;  // one more vector: the end
    hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)std::min(groups, kMost)), dim3(kThreads), 0,
                       stream, p);
  } else {
    const int64_t groups = ((p.rows * p.cols + 3) / 4 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(k_dropout_rows<T>, dim3((unsigned)std::min(groups, kMost)),
                       dim3(kThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int bgmf_dropout(const void *x, int32_t type, int64_t rows, int64_t cols, int64_t row_stride,
                 double p, uint64_t seed, uint64_t offset, const uint64_t *offset_on_device,
                 void *out, int64_t out_stride, void *hip_stream) {
  const char *call = "bgmf_dropout";
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 40))
    return fail_call(BGMF_E_ARG, "%s: rows must be in [0, 2^31) and cols in [0, 2^40): %lld x %lld",
                     call, (long long)rows, (long long)cols);
  if (!(p >= 0.0 && p <= 1.0))
    return fail_call(BGMF_E_ARG, "%s: p must be in [0, 1]: %g", call, p);
  if (rows == 0 || cols == 0) return BGMF_OK;
  if (bad_matrix(x, rows, cols, row_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (bad_matrix(out, rows, cols, out_stride, cols, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad out (pointer, alignment or row stride %lld)", call,
                     (long long)out_stride);
  if (reinterpret_cast<uintptr_t>(offset_on_device) % 8)
    return fail_call(BGMF_E_ARG, "%s: offset_on_device must be aligned to 8 bytes", call);
  if (out == x && out_stride != row_stride && rows > 1)
    return fail_call(BGMF_E_ARG, "%s: in place, the row strides must be equal", call);
  if ((out != x && share(out, type, rows, cols, out_stride, x, type, rows, cols, row_stride)) ||
      share(out, type, rows, cols, out_stride, offset_on_device, BGMF_TYPE_F32, 1, 2, 2))
    return fail_call(BGMF_E_ARG, "%s: out shares memory with an input", call);
  const Dropout d{x, out, rows, cols, row_stride, out_stride, seed, offset, offset_on_device,
                  p < 1.0 ? (uint32_t)(p * 4294967296.0) : 0, p == 1.0,
                  p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = type == BGMF_TYPE_F32    ? dropout<float>(d, stream)
                       : type == BGMF_TYPE_BF16 ? dropout<bf16_t>(d, stream)
                                                : dropout<f16_t>(d, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
