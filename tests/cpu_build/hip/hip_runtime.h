// Stands in for the HIP runtime's header where kernels are built for the CPU to see
// which addresses they touch (tests/cpu_build/mx_addresses.cpp): a workgroup's threads
// are contexts that take turns at __syncthreads().  What lanes pass to each other,
// conversions and matrix products are left out, so the numbers mean nothing.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#define __host__
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)

struct dim3 {
  unsigned x, y, z;
  explicit dim3(unsigned x = 1, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {}
};
inline dim3 threadIdx, blockIdx, gridDim;
void __syncthreads();

using hipStream_t = void *;
enum hipError_t { hipSuccess = 0 };
inline hipError_t hipGetLastError() { return hipSuccess; }
inline const char *hipGetErrorString(hipError_t) { return ""; }

struct uint2 {
  uint32_t x, y;
};
using std::max;
using std::min;

template <class To, class From>
To bits_as(From v) {
  static_assert(sizeof(To) == sizeof(From));
  To to;
  std::memcpy(&to, &v, sizeof to);
  return to;
}
inline float __uint_as_float(uint32_t v) { return bits_as<float>(v); }
inline float __int_as_float(int32_t v) { return bits_as<float>(v); }
inline uint32_t __float_as_uint(float v) { return bits_as<uint32_t>(v); }
inline int32_t __float_as_int(float v) { return bits_as<int32_t>(v); }
inline int32_t __double2loint(double v) { return (int32_t)bits_as<uint64_t>(v); }
inline int32_t __double2hiint(double v) { return (int32_t)(bits_as<uint64_t>(v) >> 32); }
inline double __hiloint2double(int32_t hi, int32_t lo) {
  return bits_as<double>((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}

#define __builtin_amdgcn_update_dpp(none, x, ...) (x)
#define __builtin_amdgcn_mov_dpp(x, ...) (x)
#define __builtin_amdgcn_readlane(x, lane) (x)
#define __builtin_amdgcn_perm(a, b, select) ((a) ^ (b))
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a, b, scale, part) (r)
#define __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, part) (f32x2{0.0f, 0.0f})
#define __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, ...) (c)
#define __builtin_amdgcn_wave_barrier()
#define __builtin_amdgcn_sched_barrier(mask)
#define __builtin_amdgcn_sched_group_barrier(mask, size, group)
