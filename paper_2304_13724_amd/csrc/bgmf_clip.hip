// Clipping of many gradients by their global norm (bgmf_clip_grad_norm).
#include <algorithm>
#include <cmath>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int kPartials = 1024;  // workgroups of the norm's first pass, at most
constexpr int kTable = 60;       // gradients that travel in one kernel's arguments (under 4 KB)

// A workgroup works on whole chunks of kChunk elements of one gradient;
// gradient i has chunks [first_chunk of i, first_chunk of i + 1).
constexpr int64_t kChunk = 8192;
struct Entry {
  const void *in;
  void *out;
  int64_t rows, cols, in_stride, out_stride;
  int64_t first_chunk;
  int64_t type;
};
struct Batch {
  Entry e[kTable];
};

__global__ void __launch_bounds__(kTable) k_table(Batch b, int count, Entry *table) {
  if ((int)threadIdx.x < count) table[threadIdx.x] = b.e[threadIdx.x];
}

// The gradient of chunk c: the last entry whose first chunk is at most c.
__device__ __forceinline__ Entry find(const Entry *table, int64_t count, int64_t c) {
  int64_t lo = 0, hi = count - 1;
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) / 2;
    if (table[mid].first_chunk <= c) lo = mid;
    else hi = mid - 1;
  }
  return table[lo];
}

__device__ __forceinline__ float load(const Entry &e, int64_t i) {
  const int64_t at = i / e.cols * e.in_stride + i % e.cols;
  if (e.type == BGMF_TYPE_F32) return static_cast<const float *>(e.in)[at];
  if (e.type == BGMF_TYPE_BF16) return to_float(static_cast<const bf16_t *>(e.in)[at]);
  return to_float(static_cast<const f16_t *>(e.in)[at]);
}
__device__ __forceinline__ void store(const Entry &e, int64_t i, float v) {
  const int64_t at = i / e.cols * e.out_stride + i % e.cols;
  if (e.type == BGMF_TYPE_F32) static_cast<float *>(e.out)[at] = v;
  else if (e.type == BGMF_TYPE_BF16) static_cast<bf16_t *>(e.out)[at] = from_float<bf16_t>(v);
  else static_cast<f16_t *>(e.out)[at] = from_float<f16_t>(v);
}

// Sum over the workgroup, the same order at every call.
__device__ double block_sum(double v) {
  __shared__ double lds[kThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
  return s;
}

__global__ void __launch_bounds__(kThreads) k_norm(const Entry *table, int64_t count,
                                                   int64_t chunks, double *partial) {
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Entry e = find(table, count, c);
    const int64_t lo = (c - e.first_chunk) * kChunk, end = e.rows * e.cols;
    const int64_t hi = lo + kChunk < end ? lo + kChunk : end;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
      const double v = load(e, i);
      s += v * v;
    }
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreads) k_clip(const Entry *table, int64_t count,
                                                   int64_t chunks, const double *partial,
                                                   int partials, float max_norm, float *norm) {
  double s = 0.0;
  for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
  const float n = (float)sqrt(block_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  const bool clips = n > max_norm && n < INFINITY;
  const float factor = clips ? max_norm / n : 1.0f;
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Entry e = find(table, count, c);
    if (!clips && e.in == e.out) continue;
    const int64_t lo = (c - e.first_chunk) * kChunk, end = e.rows * e.cols;
    const int64_t hi = lo + kChunk < end ? lo + kChunk : end;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) store(e, i, load(e, i) * factor);
  }
}

int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int64_t bgmf_clip_grad_norm_workspace(int64_t count) {
  if (count < 0 || count >= (1ll << 31)) return 0;
  return padded(kPartials * 8) + padded(count * (int64_t)sizeof(Entry));
}

int bgmf_clip_grad_norm(const bgmf_grad_t *grads, int64_t count, float max_norm, float *norm,
                        void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_clip_grad_norm";
  if (count < 0 || count >= (1ll << 31) || (count && !grads))
    return fail_call(BGMF_E_ARG, "%s: bad grads or count %lld", call, (long long)count);
  if (!(max_norm >= 0.0f))
    return fail_call(BGMF_E_ARG, "%s: max_norm must be at least 0: %g", call, max_norm);
  if (!norm) return fail_call(BGMF_E_ARG, "%s: null norm", call);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256)
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  const int64_t need = bgmf_clip_grad_norm_workspace(count);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  for (int64_t i = 0; i < count; ++i) {
    const bgmf_grad_t &g = grads[i];
    if (!is_float_type(g.type))
      return fail_call(BGMF_E_ARG, "%s: gradient %lld: type must be F32, BF16 or F16: %d", call,
                       (long long)i, g.type);
    if (g.rows < 0 || g.cols < 0 || (g.cols && g.rows > ((int64_t)1 << 60) / g.cols))
      return fail_call(BGMF_E_ARG, "%s: gradient %lld: bad size %lld x %lld", call, (long long)i,
                       (long long)g.rows, (long long)g.cols);
    if (bad_matrix(g.in, g.rows, g.cols, g.in_stride, g.cols, type_bytes(g.type)) ||
        bad_matrix(g.out, g.rows, g.cols, g.out_stride, g.cols, type_bytes(g.type)))
      return fail_call(BGMF_E_ARG, "%s: gradient %lld: bad pointer, alignment or row stride", call,
                       (long long)i);
    if (g.in == g.out && g.rows > 1 && g.cols && g.in_stride != g.out_stride)
      return fail_call(BGMF_E_ARG, "%s: gradient %lld: in place, the row strides must be equal",
                       call, (long long)i);
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  double *partial = static_cast<double *>(ws);
  Entry *table = reinterpret_cast<Entry *>(static_cast<char *>(ws) + padded(kPartials * 8));
  int64_t chunks = 0, entries = 0;
  Batch b;
  int held = 0;
  const auto send = [&] {
    if (held)
      hipLaunchKernelGGL(k_table, dim3(1), dim3(kTable), 0, stream, b, held,
                         table + entries - held);
    held = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const bgmf_grad_t &g = grads[i];
    if (g.rows == 0 || g.cols == 0) continue;
    b.e[held++] = Entry{g.in, g.out, g.rows, g.cols, g.in_stride, g.out_stride, chunks, g.type};
    ++entries;
    chunks += (g.rows * g.cols + kChunk - 1) / kChunk;
    if (held == kTable) send();
  }
  send();
  const unsigned groups = (unsigned)std::min<int64_t>(chunks, kPartials);
  if (groups)
    hipLaunchKernelGGL(k_norm, dim3(groups), dim3(kThreads), 0, stream, table, entries, chunks,
                       partial);
  hipLaunchKernelGGL(k_clip, dim3(groups ? groups : 1), dim3(kThreads), 0, stream, table, entries,
                     chunks, partial, (int)groups, max_norm, norm);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
