// Clipping of many gradients by their global norm (bgmf_clip_grad_norm).
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2048;  // workgroups of the norm's pass, at most
constexpr int kTable = 120;    // table slots that travel in a kernel's arguments (under 4 KB)

// Gradients are worked on in chunks of kChunk elements; gradient i has chunks
// [first_chunk of i, first_chunk of the next).  It takes a slot of the table,
// and a second one if its rows are not adjacent (kMatrix): in, out and size of
// that hold cols, in_stride and out_stride, and its first_chunk is past all.
constexpr int64_t kChunk = 8192;
constexpr int32_t kMatrix = 4, kPast = 0x7FFFFFFF;
struct Slot {
  int64_t in, out, size;
  int32_t first_chunk, type;
};
struct Batch {
  Slot s[kTable];
};

__global__ void __launch_bounds__(128) k_table(Batch b, int count, Slot *table) {
  if ((int)threadIdx.x < count) table[threadIdx.x] = b.s[threadIdx.x];
}

// The gradient of chunk c: the last slot whose first chunk is at most c.
// Every wave looks at 64 slots at a time.
__device__ __forceinline__ int32_t find(const Slot *table, int32_t count, int32_t c) {
  int32_t at = 0;
  for (int32_t i0 = 0; i0 < count; i0 += 64) {
    const int32_t i = i0 + (int32_t)(threadIdx.x % 64);
    const uint64_t below = __ballot(i < count && table[i].first_chunk <= c);
    if (below) at = i0 + 63 - __builtin_clzll(below);
  }
  return __builtin_amdgcn_readfirstlane(at);
}

// A gradient as the kernels use it.
struct Entry {
  const void *in;
  void *out;
  int64_t size, cols, in_stride, out_stride;
  int32_t first_chunk, type;
  bool dense;
};
__device__ __forceinline__ Entry entry(const Slot *table, int32_t at) {
  const Slot s = table[at];
  Entry e{reinterpret_cast<const void *>(s.in), reinterpret_cast<void *>(s.out), s.size, 0, 0, 0,
          s.first_chunk, s.type & (kMatrix - 1), !(s.type & kMatrix)};
  if (!e.dense) {
    const Slot m = table[at + 1];
    e.cols = m.in, e.in_stride = m.out, e.out_stride = m.size;
  }
  return e;
}

template <class T>
__device__ __forceinline__ double square(T x) {
  const double v = to_float(x);
  return v * v;
}

// Sum over the workgroup, the same order at every call.
__device__ __forceinline__ double block_sum(double v) {
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

// Calls f(entry, type, lo, hi) for the elements [lo, hi) of each chunk that
// the workgroup has: every gridDim.x-th, so that the chunks worked on at one
// time lie next to each other.
template <class F>
__device__ __forceinline__ void for_chunks(const Slot *table, int32_t count, int32_t chunks,
                                           const F &f) {
  Entry e;
  int32_t stop = -1;  // the first chunk past e's
  for (int32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    if (c >= stop) {
      const int32_t at = find(table, count, c);
      e = entry(table, at);
      const int32_t next = at + (e.dense ? 1 : 2);
      stop = next < count ? table[next].first_chunk : chunks;
    }
    const int64_t lo = (int64_t)(c - e.first_chunk) * kChunk;
    const int64_t hi = lo + kChunk < e.size ? lo + kChunk : e.size;
    if (e.type == BGMF_TYPE_F32) f(e, float{}, lo, hi);
    else if (e.type == BGMF_TYPE_BF16) f(e, bf16_t{}, lo, hi);
    else f(e, f16_t{}, lo, hi);
  }
}

// Squares in fp64: no gradient overflows or vanishes in them, and their sum is
// better than fp32 whatever its order.  Bound: HBM, one read: 31.9M fp32 values
// take 21 us, 6.1 TB/s (with the values of two sets of gradients in the cache).
__device__ __forceinline__ void norm_part(const Slot *table, int32_t count, int32_t chunks,
                                          double *partial) {
  double s = 0.0;
  for_chunks(table, count, chunks, [&](const Entry &e, auto type, int64_t lo, int64_t hi) {
    using T = decltype(type);
    constexpr int N = Vec<T>::N, K = (int)(kChunk / (kThreads * N));
    const T *x = static_cast<const T *>(e.in);
    const int tid = threadIdx.x;
    if (e.dense && hi - lo == kChunk) {
      Vec<T> a[K];
#pragma unroll
      for (int q = 0; q < K; ++q) a[q] = load_vec(x + lo + (tid + q * kThreads) * N);
#pragma unroll
      for (int q = 0; q < K; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) s += square(a[q].v[i]);
    } else if (e.dense) {
      int64_t i = lo + tid * N;
      for (; i + N <= hi; i += kThreads * N) {
        const Vec<T> a = load_vec(x + i);
#pragma unroll
        for (int k = 0; k < N; ++k) s += square(a.v[k]);
      }
      for (; i < hi; ++i) s += square(x[i]);
    } else {
      for (int64_t i = lo + tid; i < hi; i += kThreads)
        s += square(x[i / e.cols * e.in_stride + i % e.cols]);
    }
  });
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The norm from the partial sums, by every workgroup, and the gradients times
// the factor.  Bound: HBM, one read (from the Infinity Cache where the
// gradients fit it) and one write: 31.9M fp32 values take 42 us, 6.1 TB/s.  The
// stores go past the cache: otherwise the clipped values push the gradients out
// of it and are written back under the next call's reads (76 us for both
// passes, 65 so).
__device__ __forceinline__ void clip_part(const Slot *table, int32_t count, int32_t chunks,
                                          const double *partial, int partials, float max_norm,
                                          float *norm) {
  double s = 0.0;
  for (int i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
  const float n = (float)sqrt(block_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  const bool clips = n > max_norm && n < INFINITY;
  const float factor = clips ? max_norm / n : 1.0f;
  for_chunks(table, count, chunks, [&](const Entry &e, auto type, int64_t lo, int64_t hi) {
    using T = decltype(type);
    constexpr int N = Vec<T>::N, K = (int)(kChunk / (kThreads * N));
    if (!clips && e.in == e.out) return;
    const T *x = static_cast<const T *>(e.in);
    T *y = static_cast<T *>(e.out);
    const int tid = threadIdx.x;
    const auto scaled = [&](T v) { return from_float<T>(to_float(v) * factor); };
    if (e.dense && hi - lo == kChunk) {
      Vec<T> a[K];
#pragma unroll
      for (int q = 0; q < K; ++q) a[q] = load_vec(x + lo + (tid + q * kThreads) * N);
#pragma unroll
      for (int q = 0; q < K; ++q) {
#pragma unroll
        for (int i = 0; i < N; ++i) a[q].v[i] = scaled(a[q].v[i]);
        store_vec_stream(y + lo + (tid + q * kThreads) * N, a[q]);
      }
    } else if (e.dense) {
      int64_t i = lo + tid * N;
      for (; i + N <= hi; i += kThreads * N) {
        Vec<T> a = load_vec(x + i);
#pragma unroll
        for (int k = 0; k < N; ++k) a.v[k] = scaled(a.v[k]);
        store_vec_stream(y + i, a);
      }
      for (; i < hi; ++i) y[i] = scaled(x[i]);
    } else {
      for (int64_t i = lo + tid; i < hi; i += kThreads) {
        const int64_t r = i / e.cols, k = i % e.cols;
        y[r * e.out_stride + k] = scaled(x[r * e.in_stride + k]);
      }
    }
  });
}

// The table in the kernel's arguments, or in the workspace.
__global__ void __launch_bounds__(kThreads) k_norm_few(Batch b, int32_t count, int32_t chunks,
                                                       double *partial) {
  norm_part(b.s, count, chunks, partial);
}
__global__ void __launch_bounds__(kThreads) k_norm(const Slot *table, int32_t count,
                                                   int32_t chunks, double *partial) {
  norm_part(table, count, chunks, partial);
}
__global__ void __launch_bounds__(kThreads) k_clip_few(Batch b, int32_t count, int32_t chunks,
                                                       const double *partial, int partials,
                                                       float max_norm, float *norm) {
  clip_part(b.s, count, chunks, partial, partials, max_norm, norm);
}
__global__ void __launch_bounds__(kThreads) k_clip(const Slot *table, int32_t count,
                                                   int32_t chunks, const double *partial,
                                                   int partials, float max_norm, float *norm) {
  clip_part(table, count, chunks, partial, partials, max_norm, norm);
}

int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

// ---------------------------------------------------------------------------
// Whether gradients share memory.  One that is written while another's chunks
// are read or written would come out scaled once or twice, as it happens.
// ---------------------------------------------------------------------------
struct GradRegion : Region {
  int32_t grad;
  bool written;
};

// The first pair of gradients found of which one is written where the other
// lies (or one whose out meets its own in without being it); 0 if there is
// none, -1 without memory for the check.  Gradients in the order of their
// addresses, such as the parts of a bucket, are only compared with the one
// before; others are sorted (3 us more for 211 in place).
int shared_memory(const bgmf_grad_t *grads, int64_t count, int64_t *first, int64_t *second) {
  const auto region = [&](int64_t i, bool written) {
    const bgmf_grad_t &g = grads[i];
    return GradRegion{written ? region_of(g.out, g.type, g.rows, g.cols, g.out_stride)
                              : region_of(g.in, g.type, g.rows, g.cols, g.in_stride),
                      (int32_t)i, written};
  };
  int64_t some = 0, in_lo = INT64_MAX, in_hi = 0, out_lo = INT64_MAX, out_hi = 0, last = 0;
  bool ordered = true, in_place = true;
  for (int64_t i = 0; i < count; ++i) {
    if (grads[i].rows == 0 || grads[i].cols == 0) continue;
    const GradRegion w = region(i, true);
    ordered &= w.lo >= last;
    last = w.hi;
    out_lo = std::min(out_lo, w.lo), out_hi = std::max(out_hi, w.hi);
    if (grads[i].in != grads[i].out) {
      const GradRegion r = region(i, false);
      in_lo = std::min(in_lo, r.lo), in_hi = std::max(in_hi, r.hi);
      in_place = false;
    }
    ++some;
  }
  if (ordered && (in_place || in_hi <= out_lo || out_hi <= in_lo)) return 0;
  const std::unique_ptr<GradRegion[]> all(new (std::nothrow) GradRegion[2 * some]);
  const std::unique_ptr<int64_t[]> open(new (std::nothrow) int64_t[2 * some]);
  if (!all || !open) return -1;
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (grads[i].rows == 0 || grads[i].cols == 0) continue;
    all[n++] = region(i, true);
    if (grads[i].in != grads[i].out) all[n++] = region(i, false);
  }
  std::sort(all.get(), all.get() + n, [](const Region &a, const Region &b) { return a.lo < b.lo; });
  // open: the regions before i that end past its start, the written ones from
  // the front, the others from the back
  int64_t written = 0, read = 0;
  for (int64_t i = 0; i < n; ++i) {
    const GradRegion &r = all[i];
    int64_t keep = 0;
    for (int64_t q = 0; q < written; ++q) {
      const GradRegion &w = all[open[q]];
      if (w.hi <= r.lo) continue;
      open[keep++] = open[q];
      if (meets(w, r)) {
        *first = std::min(w.grad, r.grad), *second = std::max(w.grad, r.grad);
        return 1;
      }
    }
    written = keep, keep = 0;
    if (r.written) {
      for (int64_t q = 0; q < read; ++q) {
        const int64_t at = open[2 * some - 1 - q];
        if (all[at].hi <= r.lo) continue;
        open[2 * some - 1 - keep++] = at;
        if (meets(all[at], r)) {
          *first = std::min(all[at].grad, r.grad), *second = std::max(all[at].grad, r.grad);
          return 1;
        }
      }
      read = keep;
      open[written++] = i;
    } else {
      open[2 * some - 1 - read++] = i;
    }
  }
  return 0;
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int64_t bgmf_clip_grad_norm_workspace(int64_t count) {
  if (count < 0 || count >= (1ll << 31)) return 0;
  return padded(kGroups * 8) + padded(2 * count * (int64_t)sizeof(Slot));
}

int bgmf_clip_grad_norm(const bgmf_grad_t *grads, int64_t count, float max_norm, float *norm,
                        void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_clip_grad_norm";
  if (count < 0 || count >= (1ll << 31) || (count && !grads))
    return fail_call(BGMF_E_ARG, "%s: bad grads or count %lld", call, (long long)count);
  if (!(max_norm >= 0.0f))
    return fail_call(BGMF_E_ARG, "%s: max_norm must be at least 0: %g", call, max_norm);
  if (!norm) return fail_call(BGMF_E_ARG, "%s: null norm", call);
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
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    total += (grads[i].rows * grads[i].cols + kChunk - 1) / kChunk;
    if (total >= kPast - (1 << 20) || count >= (1 << 30))
      return fail_call(BGMF_E_UNSUPPORTED, "%s: more than 2^43 elements or 2^30 gradients", call);
  }
  int64_t first = 0, second = 0;
  if (const int shared = shared_memory(grads, count, &first, &second))
    return shared < 0 ? fail_call(BGMF_E_NOMEM, "%s: out of host memory", call)
                      : fail_call(BGMF_E_ARG,
                                  "%s: gradients %lld and %lld share memory that is written", call,
                                  (long long)first, (long long)second);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256)
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  const int64_t need = bgmf_clip_grad_norm_workspace(count);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  double *partial = static_cast<double *>(ws);
  Slot *table = reinterpret_cast<Slot *>(static_cast<char *>(ws) + padded(kGroups * 8));
  int32_t chunks = 0, slots = 0, held = 0;
  Batch b;
  const auto send = [&] {
    if (held)
      hipLaunchKernelGGL(k_table, dim3(1), dim3(128), 0, stream, b, held, table + slots - held);
    held = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const bgmf_grad_t &g = grads[i];
    if (g.rows == 0 || g.cols == 0) continue;
    const bool dense = g.rows == 1 || (g.in_stride == g.cols && g.out_stride == g.cols);
    const int32_t need = dense ? 1 : 2;
    if (held + need > kTable) send();
    b.s[held] = Slot{reinterpret_cast<int64_t>(g.in), reinterpret_cast<int64_t>(g.out),
                     g.rows * g.cols, chunks, g.type | (dense ? 0 : kMatrix)};
    if (!dense) b.s[held + 1] = Slot{g.cols, g.in_stride, g.out_stride, kPast, 0};
    held += need, slots += need;
    chunks += (int32_t)((g.rows * g.cols + kChunk - 1) / kChunk);
  }
  const unsigned groups = (unsigned)std::min<int64_t>(chunks, kGroups);
  const unsigned clip_groups = (unsigned)std::max<int64_t>(std::min<int64_t>(chunks, kGroups), 1);
  if (slots == held) {
    if (groups)
      hipLaunchKernelGGL(k_norm_few, dim3(groups), dim3(kThreads), 0, stream, b, slots, chunks,
                         partial);
    hipLaunchKernelGGL(k_clip_few, dim3(clip_groups), dim3(kThreads), 0, stream, b, slots,
                       chunks, partial, (int)groups, max_norm, norm);
  } else {
    send();
    hipLaunchKernelGGL(k_norm, dim3(groups), dim3(kThreads), 0, stream, table, slots, chunks,
                       partial);
    hipLaunchKernelGGL(k_clip, dim3(clip_groups), dim3(kThreads), 0, stream, table, slots,
                       chunks, partial, (int)groups, max_norm, norm);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
