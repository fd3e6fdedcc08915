// Shared by the HIP sources of the ranking operators (not part of the ABI):
// element types, vector loads and stores, and the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/bgmf.h"

namespace bgmfk {

// Sets the calling thread's message (bgmf_last_error(NULL)) and returns code.
int fail_call(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline int64_t type_bytes(int32_t type) {
  return type == BGMF_TYPE_F32 ? 4 : type == BGMF_TYPE_I8 ? 1 : 2;
}
inline bool is_float_type(int32_t type) {
  return type == BGMF_TYPE_F32 || type == BGMF_TYPE_BF16 || type == BGMF_TYPE_F16;
}

// A matrix argument: a non-null pointer aligned to its elements (unless the
// matrix is empty) and a row stride of at least min_stride whose last element
// has an offset below 2^62 bytes.
inline bool bad_matrix(const void *p, int64_t rows, int64_t cols, int64_t stride,
                       int64_t min_stride, int64_t esize) {
  if (rows <= 0 || cols <= 0) return false;
  if (!p || reinterpret_cast<uintptr_t>(p) % (uintptr_t)esize) return true;
  return rows > 1 && (stride < min_stride || stride > ((int64_t)1 << 60) / rows);
}

// Whether matrices share memory: what one workgroup writes where another has yet
// to read would make the results a matter of timing.

// Rows of `bytes` bytes, `stride` apart, from lo on; the last ends at hi.
struct Region {
  int64_t lo, hi, bytes, stride, rows;
};

// Of a matrix argument that is neither bad nor empty.  Rows that overlap each
// other are one row of all their bytes.
inline Region region_of(const void *p, int32_t type, int64_t rows, int64_t cols, int64_t stride) {
  const int64_t size = type_bytes(type), lo = reinterpret_cast<int64_t>(p);
  if (rows == 1) stride = cols;
  Region r{lo, lo + ((rows - 1) * stride + cols) * size, cols * size, stride * size, rows};
  if (stride <= cols) r.bytes = r.stride = r.hi - lo, r.rows = 1;
  return r;
}

// Whether row i of a meets a row of b: the first of b's rows that ends past its
// start begins before its end.
inline bool row_meets(const Region &a, int64_t i, const Region &b) {
  const int64_t lo = a.lo + i * a.stride, past = lo - b.lo - b.bytes;
  const int64_t row = past < 0 ? 0 : past / b.stride + 1;
  return row < b.rows && b.lo + row * b.stride < lo + a.bytes;
}

inline bool meets(const Region &a, const Region &b) {
  if (a.hi <= b.lo || b.hi <= a.lo) return false;
  if (a.rows > b.rows) return meets(b, a);
  if (a.rows > 1 && a.stride == b.stride) {
    // rows of a that lie before b's second row all look at b's first one, and
    // the last of them comes nearest; the later ones look at rows of b that
    // are as far from them as the first of them is
    const int64_t before = b.lo + b.bytes - a.lo, rows = a.rows;
    const int64_t later = before <= 0 ? 0 : (before + a.stride - 1) / a.stride;
    return (later > 0 && row_meets(a, std::min(later, rows) - 1, b)) ||
           (later < rows && row_meets(a, later, b));
  }
  for (int64_t i = 0; i < a.rows; ++i)
    if (row_meets(a, i, b)) return true;
  return false;
}

// The same for two arguments, empty ones among them.
inline bool share(const void *p, int32_t type, int64_t rows, int64_t cols, int64_t stride,
                  const void *q, int32_t q_type, int64_t q_rows, int64_t q_cols,
                  int64_t q_stride) {
  if (!p || !q || !rows || !cols || !q_rows || !q_cols) return false;
  return meets(region_of(p, type, rows, cols, stride),
               region_of(q, q_type, q_rows, q_cols, q_stride));
}

using f16_t = _Float16;
using bf16_t = __bf16;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(f16_t x) { return (float)x; }
__device__ __forceinline__ float to_float(bf16_t x) {
  return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, x) << 16);
}
// rounded to nearest, ties to even
template <class T>
__device__ __forceinline__ T from_float(float x) { return (T)x; }
// The empty statement keeps a product that is converted in two roundings (to
// fp32, then to f16): the compiler would merge both into one mixed-precision
// instruction, and the result would not be the one of fp32 arithmetic.
template <>
__device__ __forceinline__ f16_t from_float<f16_t>(float x) {
  asm("" : "+v"(x));
  return (f16_t)x;
}

// 16 bytes of elements, at any alignment that suits one element.
template <class T>
struct alignas(16) Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  T v[N];
};
template <class T>
__device__ __forceinline__ Vec<T> load_vec(const T *p) {
  Vec<T> x;
  __builtin_memcpy(&x, p, sizeof x);
  return x;
}
template <class T>
__device__ __forceinline__ void store_vec(T *p, const Vec<T> &x) {
  __builtin_memcpy(p, &x, sizeof x);
}
// The same for what is not read again soon.
template <class T>
__device__ __forceinline__ void store_vec_stream(T *p, const Vec<T> &x) {
  typedef uint32_t quad __attribute__((ext_vector_type(4), aligned(2)));
  quad q;
  __builtin_memcpy(&q, &x, sizeof q);
  __builtin_nontemporal_store(q, reinterpret_cast<quad *>(p));
}

}  // namespace bgmfk
