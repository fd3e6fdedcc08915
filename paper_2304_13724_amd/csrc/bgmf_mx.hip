// Rows in 4 bits with a scale for each block of 32 (bgmf_quantize_rows_mx,
// bgmf_dequantize_rows_mx) and the product of two such matrices
// (bgmf_mx_scores).
#include <algorithm>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMostGroups = 1 << 20;
constexpr int kBlock = 32;  // values that share a scale: 16 bytes
constexpr int kNaN = 255;   // the scale byte of a block that stands for NaN

using i32x4 = __attribute__((ext_vector_type(4))) int32_t;
using i32x8 = __attribute__((ext_vector_type(8))) int32_t;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using f32x2 = __attribute__((ext_vector_type(2))) float;

// Columns from c on, 8 of them; zeros at and past k.
template <class T>
__device__ __forceinline__ void load_eight(const T *row, int32_t c, int32_t k, float (&x)[8]) {
  constexpr int N = Vec<T>::N;
  if (c + 8 <= k) {
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
      const Vec<T> v = load_vec(row + c + h * N);
#pragma unroll
      for (int i = 0; i < N; ++i) x[h * N + i] = to_float(v.v[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < k ? to_float(row[c + i]) : 0.0f;
  }
}

// The largest magnitude's bits (an order of floats; at and past 0x7F800000
// where one is infinite or NaN).
template <int COUNT>
__device__ __forceinline__ uint32_t largest_bits(const float (&x)[COUNT]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  return m;
}
// Over the four lanes of a block.
__device__ __forceinline__ uint32_t over_four(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));  // lane ^ 2
}
__device__ __forceinline__ int scale_byte(uint32_t largest) {
  const int e = (int)(largest >> 23);
  return e == 255 ? kNaN : e > 2 ? e - 2 : 0;
}

// Eight values in 4 bits, by the conversion instruction (it divides by its
// scale, rounds to nearest, ties to even, and saturates).  Its scale has to be
// a normal number: values of a block with byte 0 are multiplied by 2^64 first.
__device__ __forceinline__ uint32_t eight_to_bits(float (&x)[8], int code) {
  float s = __uint_as_float((uint32_t)code << 23);
  if (code == 0) {
    s = 0x1p-63f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= 0x1p64f;
  }
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
  return code == kNaN ? 0 : r;
}
__device__ __forceinline__ void bits_to_eight(uint32_t q, int code, float (&x)[8]) {
  const float s = __uint_as_float((uint32_t)(code ? code : 64) << 23);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 0),
              b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 1),
              c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 2),
              d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 3);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (code == 0) x[i] *= 0x1p-64f;
    if (code == kNaN) x[i] = NAN;
  }
}

// ---------------------------------------------------------------------------
// A thread takes a chunk of eight columns, four neighbours a block: LANES
// threads to a row.
// ---------------------------------------------------------------------------
struct Rows {
  const void *x;
  int64_t rows, stride;
  int32_t k, chunks;  // of a row
  uint8_t *q, *scale;
  int64_t q_stride, scale_stride;
};

template <class T, int LANES>
__global__ void __launch_bounds__(kThreads) k_quantize_mx(Rows P) {
  constexpr int kRows = kThreads / LANES;
  const int lane = threadIdx.x % LANES;
  for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; r < P.rows;
       r += (int64_t)gridDim.x * kRows) {
    for (int32_t c = lane; c < P.chunks; c += LANES) {
      float x[8];
      load_eight(static_cast<const T *>(P.x) + r * P.stride, c * 8, P.k, x);
      const int code = scale_byte(over_four(largest_bits(x)));
      const uint32_t bits = eight_to_bits(x, code);
      __builtin_memcpy(P.q + r * P.q_stride + (int64_t)c * 4, &bits, 4);
      if (c % 4 == 0) P.scale[r * P.scale_stride + c / 4] = (uint8_t)code;
    }
  }
}

template <class T, int LANES>
__global__ void __launch_bounds__(kThreads) k_dequantize_mx(Rows P, T *out, int64_t out_stride) {
  constexpr int kRows = kThreads / LANES, N = Vec<T>::N;
  const int lane = threadIdx.x % LANES;
  for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; r < P.rows;
       r += (int64_t)gridDim.x * kRows) {
    for (int32_t c = lane; c < P.chunks; c += LANES) {
      uint32_t bits;
      __builtin_memcpy(&bits, P.q + r * P.q_stride + (int64_t)c * 4, 4);
      float x[8];
      bits_to_eight(bits, P.scale[r * P.scale_stride + c / 4], x);
      T *to = out + r * out_stride + (int64_t)c * 8;
      if (c * 8 + 8 <= P.k) {
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) {
          Vec<T> v;
#pragma unroll
          for (int i = 0; i < N; ++i) v.v[i] = from_float<T>(x[h * N + i]);
          store_vec(to + h * N, v);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c * 8 + i < P.k) to[i] = from_float<T>(x[i]);
      }
    }
  }
}

template <class F>
void with_lanes(int32_t chunks, const F &f) {
  if (chunks <= 4) f(std::integral_constant<int, 4>{});
  else if (chunks <= 8) f(std::integral_constant<int, 8>{});
  else if (chunks <= 16) f(std::integral_constant<int, 16>{});
  else if (chunks <= 32) f(std::integral_constant<int, 32>{});
  else if (chunks <= 64) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, kThreads>{});
}
inline dim3 groups_of(int64_t rows, int lanes) {
  const int64_t per = kThreads / lanes;
  return dim3((unsigned)std::min((rows + per - 1) / per, kMostGroups));
}

template <class T>
hipError_t quantize_mx(const Rows &p, hipStream_t stream) {
  with_lanes(p.chunks, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_quantize_mx<T, L>), groups_of(p.rows, L), dim3(kThreads), 0, stream, p);
  });
  return hipGetLastError();
}
hipError_t quantize_mx(int32_t type, const Rows &p, hipStream_t stream) {
  return type == BGMF_TYPE_F32    ? quantize_mx<float>(p, stream)
         : type == BGMF_TYPE_BF16 ? quantize_mx<bf16_t>(p, stream)
                                  : quantize_mx<f16_t>(p, stream);
}
template <class T>
hipError_t dequantize_mx(const Rows &p, void *out, int64_t out_stride, hipStream_t stream) {
  with_lanes(p.chunks, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    hipLaunchKernelGGL((k_dequantize_mx<T, L>), groups_of(p.rows, L), dim3(kThreads), 0, stream,
                       p, static_cast<T *>(out), out_stride);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The product.
// ---------------------------------------------------------------------------
struct Product {
  const uint8_t *a, *a_scale;  // users: rows of `blocks` blocks
  int64_t rows, a_stride, as_stride;
  const uint8_t *b, *b_scale;  // items
  int64_t items, b_stride, bs_stride;
  int32_t blocks;
  void *out;
  int64_t out_stride;
};

// v_mfma_scale_f32_32x32x64_f8f6f4 on 4-bit values: lane l holds block l / 32
// (of two) of row l % 32 of either side, and its scale.  Register g of a lane
// is the sum of user 8 (g / 4) + 4 (l / 32) + g % 4 and item l % 32.
__device__ __forceinline__ f32x16 multiply(i32x4 a, int a_scale, i32x4 b, int b_scale, f32x16 c) {
  const i32x8 x = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, y = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 0, a_scale, 0, b_scale);
}

__device__ __forceinline__ i32x4 block_bytes(const uint8_t *p) {
  typedef int32_t quad __attribute__((ext_vector_type(4), aligned(1)));
  return *reinterpret_cast<const quad *>(p);
}

// A wave takes tiles of 32 items and the 32 users of blockIdx.y.
template <class O>
__global__ void __launch_bounds__(kThreads) k_mx_few(Product P) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int l32 = lane % 32, half = lane / 32;
  const int64_t r0 = (int64_t)blockIdx.y * 32, tiles = (P.items + 31) / 32;
  const int64_t r = r0 + l32 < P.rows ? r0 + l32 : P.rows - 1;
  const uint8_t *a = P.a + r * P.a_stride, *as = P.a_scale + r * P.as_stride;
  for (int64_t tile = (int64_t)blockIdx.x * kWaves + wave; tile < tiles;
       tile += (int64_t)gridDim.x * kWaves) {
    const int64_t item = tile * 32 + l32, j = item < P.items ? item : P.items - 1;
    const uint8_t *b = P.b + j * P.b_stride, *bs = P.b_scale + j * P.bs_stride;
    f32x16 acc = {};
    for (int32_t s = 0; s < P.blocks; s += 2) {
      const int32_t at = s + half;
      i32x4 x = {}, y = {};
      int xs = 0, ys = 0;
      if (at < P.blocks) {
        x = block_bytes(a + (int64_t)at * 16), xs = as[at];
        y = block_bytes(b + (int64_t)at * 16), ys = bs[at];
      }
      acc = multiply(x, xs, y, ys, acc);
    }
    if (item >= P.items) continue;
#pragma unroll
    for (int g = 0; g < 16; ++g) {
      const int64_t u = r0 + 8 * (g / 4) + 4 * half + g % 4;
      if (u < P.rows) static_cast<O *>(P.out)[u * P.out_stride + item] = from_float<O>(acc[g]);
    }
  }
}

// Workgroups that fill the GPU: eight of four waves on each of 256 CUs.
constexpr int64_t kFullGpu = 2048;

template <class O>
hipError_t product(Product p, hipStream_t stream) {
  const int64_t all = (p.items + 32 * kWaves - 1) / (32 * kWaves);
  constexpr int64_t kMost = 65535ll * 32;  // users of a launch
  for (int64_t left = p.rows; left > 0; left -= kMost) {
    p.rows = std::min(left, kMost);
    const int64_t users = (p.rows + 31) / 32;
    const dim3 grid((unsigned)std::min(all, std::max(kFullGpu / users, (int64_t)1) * 4),
                    (unsigned)users);
    hipLaunchKernelGGL(k_mx_few<O>, grid, dim3(kThreads), 0, stream, p);
    p.a += kMost * p.a_stride, p.a_scale += kMost * p.as_stride;
    p.out = static_cast<O *>(p.out) + kMost * p.out_stride;
  }
  return hipGetLastError();
}

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline int64_t blocks_of(int64_t k) { return (k + kBlock - 1) / kBlock; }
constexpr int64_t kMostK = (1 << 20) - 1;  // of a product

// Workspace: the users' bytes, then their scales.
int64_t bytes_part(int64_t rows, int64_t k) { return round_up(rows * blocks_of(k) * 16, 256); }

int check_rows(const char *call, int64_t rows, int64_t k, int64_t most_k) {
  if (rows < 0 || rows >= (1ll << 31) || k < 1 || k > most_k)
    return fail_call(BGMF_E_ARG, "%s: rows must be in [0, 2^31) and k in [1, %lld]: %lld x %lld",
                     call, (long long)most_k, (long long)rows, (long long)k);
  return 0;
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int bgmf_quantize_rows_mx(const void *x, int32_t type, int64_t rows, int64_t k,
                          int64_t row_stride, uint8_t *q, int64_t q_stride, uint8_t *scale,
                          int64_t scale_stride, void *hip_stream) {
  const char *call = "bgmf_quantize_rows_mx";
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (const int rc = check_rows(call, rows, k, (1 << 30) - 1)) return rc;
  const int64_t blocks = blocks_of(k);
  if (bad_matrix(x, rows, k, row_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (bad_matrix(q, rows, blocks * 16, q_stride, blocks * 16, 1))
    return fail_call(BGMF_E_ARG, "%s: bad q (pointer or row stride %lld)", call,
                     (long long)q_stride);
  if (bad_matrix(scale, rows, blocks, scale_stride, blocks, 1))
    return fail_call(BGMF_E_ARG, "%s: bad scale (pointer or row stride %lld)", call,
                     (long long)scale_stride);
  if (rows == 0) return BGMF_OK;
  if (share(q, BGMF_TYPE_I8, rows, blocks * 16, q_stride, x, type, rows, k, row_stride) ||
      share(scale, BGMF_TYPE_I8, rows, blocks, scale_stride, x, type, rows, k, row_stride) ||
      share(scale, BGMF_TYPE_I8, rows, blocks, scale_stride, q, BGMF_TYPE_I8, rows, blocks * 16,
            q_stride))
    return fail_call(BGMF_E_ARG, "%s: q or scale shares memory with another argument", call);
  const Rows p{x, rows, row_stride, (int32_t)k, (int32_t)(blocks * 4), q, scale, q_stride,
               scale_stride};
  const hipError_t e = quantize_mx(type, p, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int bgmf_dequantize_rows_mx(const uint8_t *q, int64_t q_stride, const uint8_t *scale,
                            int64_t scale_stride, int64_t rows, int64_t k, void *out,
                            int32_t out_type, int64_t out_stride, void *hip_stream) {
  const char *call = "bgmf_dequantize_rows_mx";
  if (!is_float_type(out_type))
    return fail_call(BGMF_E_ARG, "%s: out_type must be F32, BF16 or F16: %d", call, out_type);
  if (const int rc = check_rows(call, rows, k, (1 << 30) - 1)) return rc;
  const int64_t blocks = blocks_of(k);
  if (bad_matrix(q, rows, blocks * 16, q_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad q (pointer or row stride %lld)", call,
                     (long long)q_stride);
  if (bad_matrix(scale, rows, blocks, scale_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad scale (pointer or row stride %lld)", call,
                     (long long)scale_stride);
  if (bad_matrix(out, rows, k, out_stride, k, type_bytes(out_type)))
    return fail_call(BGMF_E_ARG, "%s: bad out (pointer, alignment or row stride %lld)", call,
                     (long long)out_stride);
  if (rows == 0) return BGMF_OK;
  if (share(out, out_type, rows, k, out_stride, q, BGMF_TYPE_I8, rows, blocks * 16, q_stride) ||
      share(out, out_type, rows, k, out_stride, scale, BGMF_TYPE_I8, rows, blocks, scale_stride))
    return fail_call(BGMF_E_ARG, "%s: out shares memory with an input", call);
  const Rows p{nullptr, rows, 0, (int32_t)k, (int32_t)(blocks * 4), const_cast<uint8_t *>(q),
               const_cast<uint8_t *>(scale), q_stride, scale_stride};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = out_type == BGMF_TYPE_F32 ? dequantize_mx<float>(p, out, out_stride, stream)
                       : out_type == BGMF_TYPE_BF16
                           ? dequantize_mx<bf16_t>(p, out, out_stride, stream)
                           : dequantize_mx<f16_t>(p, out, out_stride, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int64_t bgmf_mx_scores_workspace(int64_t rows, int64_t item_count, int64_t k, int32_t type) {
  if (rows <= 0 || k <= 0 || item_count <= 0 || rows >= (1ll << 31) || k > kMostK ||
      type == BGMF_TYPE_MX4)
    return 0;
  return bytes_part(rows, k) + round_up(rows * blocks_of(k), 256);
}

int bgmf_mx_scores(const void *x, int32_t type, int64_t rows, int64_t k, int64_t row_stride,
                   const uint8_t *row_scale, int64_t row_scale_stride, const uint8_t *items,
                   int64_t item_count, int64_t items_stride, const uint8_t *item_scale,
                   int64_t item_scale_stride, void *out, int32_t out_type, int64_t out_stride,
                   void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_mx_scores";
  const bool own = type != BGMF_TYPE_MX4;  // the rows are quantised here
  if (own && !is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be MX4, F32, BF16 or F16: %d", call, type);
  if (!is_float_type(out_type))
    return fail_call(BGMF_E_ARG, "%s: out_type must be F32, BF16 or F16: %d", call, out_type);
  if (const int rc = check_rows(call, rows, k, kMostK)) return rc;
  if (item_count < 0 || item_count >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: item_count must be in [0, 2^31): %lld", call,
                     (long long)item_count);
  if (rows == 0 || item_count == 0) return BGMF_OK;
  const int64_t blocks = blocks_of(k), bytes = blocks * 16;
  if (own ? bad_matrix(x, rows, k, row_stride, 0, type_bytes(type))
          : bad_matrix(x, rows, bytes, row_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (own != (row_scale == nullptr))
    return fail_call(BGMF_E_ARG, "%s: row_scale goes with rows of type MX4 and with no other",
                     call);
  if (!own && bad_matrix(row_scale, rows, blocks, row_scale_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad row_scale (row stride %lld)", call,
                     (long long)row_scale_stride);
  if (bad_matrix(items, item_count, bytes, items_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad items (pointer or row stride %lld)", call,
                     (long long)items_stride);
  if (bad_matrix(item_scale, item_count, blocks, item_scale_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad item_scale (pointer or row stride %lld)", call,
                     (long long)item_scale_stride);
  if (bad_matrix(out, rows, item_count, out_stride, item_count, type_bytes(out_type)))
    return fail_call(BGMF_E_ARG, "%s: bad out (pointer, alignment or row stride %lld)", call,
                     (long long)out_stride);
  const int64_t need = bgmf_mx_scores_workspace(rows, item_count, k, type);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 256))
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  const auto shares = [&](const void *y, int32_t y_type, int64_t y_rows, int64_t y_cols,
                          int64_t y_stride) {
    return share(out, out_type, rows, item_count, out_stride, y, y_type, y_rows, y_cols, y_stride);
  };
  if (shares(x, own ? type : BGMF_TYPE_I8, rows, own ? k : bytes, row_stride) ||
      shares(row_scale, BGMF_TYPE_I8, rows, blocks, row_scale_stride) ||
      shares(items, BGMF_TYPE_I8, item_count, bytes, items_stride) ||
      shares(item_scale, BGMF_TYPE_I8, item_count, blocks, item_scale_stride))
    return fail_call(BGMF_E_ARG, "%s: out shares memory with an input", call);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  Product p{static_cast<const uint8_t *>(x), row_scale, rows, row_stride, row_scale_stride,
            items, item_scale, item_count, items_stride, item_scale_stride, (int32_t)blocks,
            out, out_stride};
  hipError_t e = hipSuccess;
  if (own) {
    uint8_t *q = static_cast<uint8_t *>(ws), *scale = q + bytes_part(rows, k);
    e = quantize_mx(type, Rows{x, rows, row_stride, (int32_t)k, (int32_t)(blocks * 4), q, scale,
                               bytes, blocks}, stream);
    p.a = q, p.a_scale = scale, p.a_stride = bytes, p.as_stride = blocks;
  }
  if (e == hipSuccess)
    e = out_type == BGMF_TYPE_F32    ? product<float>(p, stream)
        : out_type == BGMF_TYPE_BF16 ? product<bf16_t>(p, stream)
                                     : product<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
