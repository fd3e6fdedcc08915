// Rows in 8-bit integers (bgmf_quantize_rows) and the product of two such
// matrices with their scales (bgmf_quantized_scores).
#include <algorithm>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMostGroups = 1 << 20;

using i32x4 = __attribute__((ext_vector_type(4))) int32_t;
using i32x16 = __attribute__((ext_vector_type(16))) int32_t;

// ---------------------------------------------------------------------------
// Rows to bytes.  One pass over global memory: LANES threads hold a row
// (HELD vectors of 16 bytes each), reduce its largest magnitude, and write
// the quotients; what a longer row has beyond that is read a second time.
// Bound: HBM.
// ---------------------------------------------------------------------------
constexpr int kHeld = 4;

template <class T, int LANES>
__global__ void __launch_bounds__(kThreads) k_quantize(const T *x, int64_t rows, int32_t k,
                                                       int64_t stride, int8_t *q, int64_t q_stride,
                                                       int32_t fill, float *scale) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x % LANES;
  const int32_t vecs = (k + N - 1) / N;
  __shared__ float lds[kWaves];
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES; r < rows;
       r += (int64_t)gridDim.x * (kThreads / LANES)) {
    const T *row = x + r * stride;
    const auto load = [&](int32_t v) {  // vector v of the row, zeros past its end
      Vec<T> a = {};
      const int32_t at = v * N;
      if (at + N <= k) a = load_vec(row + at);
      else
        for (int i = 0; i < N; ++i)
          if (at + i < k) a.v[i] = row[at + i];
      return a;
    };
    float most = 0.0f;
    bool bad = false;
    const auto look = [&](const Vec<T> &a) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float v = fabsf(to_float(a.v[i]));
        bad |= !(v < INFINITY);
        most = fmaxf(most, v);
      }
    };
    Vec<T> held[kHeld];
#pragma unroll
    for (int h = 0; h < kHeld; ++h) held[h] = load(lane + h * LANES);
#pragma unroll
    for (int h = 0; h < kHeld; ++h) look(held[h]);
#pragma unroll 4
    for (int32_t v = lane + kHeld * LANES; v < vecs; v += LANES) look(load(v));
    if (bad) most = INFINITY;
#pragma unroll
    for (int o = LANES < 64 ? LANES / 2 : 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if constexpr (LANES > 64) {
      if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = most;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) most = fmaxf(most, lds[w]);
      __syncthreads();
    }
    const float s = most == INFINITY ? NAN : most / 127.0f;
    if (lane == 0) scale[r] = s;
    int8_t *to = q + r * q_stride;
    const auto put = [&](int32_t v, const Vec<T> &a) {
      int8_t b[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float y = s > 0.0f ? rintf(to_float(a.v[i]) / s) : 0.0f;
        b[i] = (int8_t)fminf(fmaxf(y, -127.0f), 127.0f);
      }
      const int32_t at = v * N;
      if (at + N <= fill) __builtin_memcpy(to + at, b, N);
      else
        for (int i = 0; i < N; ++i)
          if (at + i < fill) to[at + i] = b[i];
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h) put(lane + h * LANES, held[h]);
    for (int32_t v = lane + kHeld * LANES; v * N < fill; v += LANES) put(v, load(v));
  }
}

// Fills columns [k, fill) of q with zeros.
template <class T>
hipError_t quantize(const void *x, int64_t rows, int32_t k, int64_t stride, int8_t *q,
                    int64_t q_stride, int32_t fill, float *scale, hipStream_t stream) {
  const int32_t vecs = (fill + Vec<T>::N - 1) / Vec<T>::N;
  const auto go = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const int64_t per = kThreads / L, groups = std::min((rows + per - 1) / per, kMostGroups);
    hipLaunchKernelGGL((k_quantize<T, L>), dim3((unsigned)groups), dim3(kThreads), 0,
                       stream, static_cast<const T *>(x), rows, k, stride, q, q_stride, fill,
                       scale);
  };
  // as few lanes as keep at most two vectors each, so that short rows fill a wave
  if (vecs <= 8) go(std::integral_constant<int, 4>{});
  else if (vecs <= 32) go(std::integral_constant<int, 16>{});
  else if (vecs <= 256) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, kThreads>{});
  return hipGetLastError();
}

hipError_t quantize_by_type(int32_t type, const void *x, int64_t rows, int32_t k, int64_t stride,
                            int8_t *q, int64_t q_stride, int32_t fill, float *scale,
                            hipStream_t stream) {
  if (type == BGMF_TYPE_F32)
    return quantize<float>(x, rows, k, stride, q, q_stride, fill, scale, stream);
  if (type == BGMF_TYPE_BF16)
    return quantize<bf16_t>(x, rows, k, stride, q, q_stride, fill, scale, stream);
  return quantize<f16_t>(x, rows, k, stride, q, q_stride, fill, scale, stream);
}

// ---------------------------------------------------------------------------
// The product.  Users' bytes come laid out for it: row stride kp (k rounded
// up to kUnit), zeros in [k, kp).  What an item's loads pick up past k (the
// next item's bytes, or padding) meets those zeros.
// ---------------------------------------------------------------------------
constexpr int kUnit = 64;
inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Product {
  const int8_t *a;  // users: rows x kp
  const float *a_scale;
  int64_t rows;
  int32_t k, kp;
  const int8_t *b;  // items x k
  const int8_t *b_end;  // past the last item's last byte
  const float *b_scale;
  int64_t items, b_stride;
  void *out;
  int64_t out_stride;
};

// Bytes given as they are, into the padded layout.
__global__ void __launch_bounds__(kThreads) k_pad_rows(const int8_t *x, int64_t rows, int32_t k,
                                                       int64_t stride, int8_t *q, int32_t kp) {
  const int64_t chunks = rows * (kp / 16);
  for (int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x; c < chunks;
       c += (int64_t)gridDim.x * kThreads) {
    const int64_t r = c / (kp / 16);
    const int32_t at = (int32_t)(c % (kp / 16)) * 16;
    const int8_t *p = x + r * stride + at;
    alignas(16) int8_t b[16] = {};
    if (at + 16 <= k) __builtin_memcpy(b, p, 16);
    else
      for (int i = 0; i < 16; ++i)
        if (at + i < k) b[i] = p[i];
    *reinterpret_cast<i32x4 *>(q + r * kp + at) = *reinterpret_cast<const i32x4 *>(b);
  }
}

// 16 bytes of an item from column c on, at any address.
__device__ __forceinline__ i32x4 item_bytes(const int8_t *row, int32_t c) {
  i32x4 x;
  __builtin_memcpy(&x, row + c, 16);
  return x;
}
// The same where c may be at or past the row's end: nothing is read past the
// end of the matrix.
__device__ __forceinline__ i32x4 item_bytes_tail(const int8_t *row, int32_t c, int32_t k,
                                                 const int8_t *end) {
  i32x4 x = {0, 0, 0, 0};
  if (c >= k) return x;
  if (row + c + 16 <= end) return item_bytes(row, c);
  int8_t b[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) b[i] = c + i < k ? row[c + i] : (int8_t)0;
  __builtin_memcpy(&x, b, 16);
  return x;
}

template <class O>
__device__ __forceinline__ O score_of(int32_t sum, float a, float b) {
  return from_float<O>((float)sum * a * b);
}

// Few users (rows <= 16 USERS): every item's bytes go from global memory into
// a matrix instruction once (v_mfma_i32_16x16x64_i8: 16 items x 16 users, 64
// columns of k; lane l holds 16 bytes of item l % 16 and of user l % 16).  A
// wave takes ITEMS tiles of 16 items, so that many loads are in flight.  With
// SPLIT, the workgroup's waves share the tiles and take a quarter of k each.
// Bound: HBM (the items' bytes).
template <class O, int USERS, int ITEMS, bool SPLIT>
__global__ void __launch_bounds__(kThreads) k_product_few(Product P) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int l16 = lane % 16, part = lane / 16;
  const int64_t first = SPLIT ? (int64_t)blockIdx.x * (16 * ITEMS)
                              : ((int64_t)blockIdx.x * kWaves + wave) * (16 * ITEMS);
  if (!SPLIT && first >= P.items) return;
  const int8_t *item[ITEMS], *user[USERS];
#pragma unroll
  for (int t = 0; t < ITEMS; ++t) {
    const int64_t j = first + t * 16 + l16;
    item[t] = P.b + (j < P.items ? j : P.items - 1) * P.b_stride;
  }
#pragma unroll
  for (int u = 0; u < USERS; ++u) {
    const int64_t r = u * 16 + l16;
    user[u] = P.a + (r < P.rows ? r : P.rows - 1) * P.kp + part * 16;
  }
  i32x4 acc[ITEMS][USERS] = {};
  const int steps = P.kp / 64, full = P.k / 64;
  const int begin = SPLIT ? steps * wave / kWaves : 0;
  const int end = SPLIT ? steps * (wave + 1) / kWaves : steps;
  const auto step = [&](int s, auto tail) {
    const int32_t c = s * 64 + part * 16;
    i32x4 x[ITEMS], y[USERS];
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) {
      if constexpr (decltype(tail)::value) x[t] = item_bytes_tail(item[t], c, P.k, P.b_end);
      else x[t] = item_bytes(item[t], c);
    }
#pragma unroll
    for (int u = 0; u < USERS; ++u) y[u] = *reinterpret_cast<const i32x4 *>(user[u] + s * 64);
#pragma unroll
    for (int t = 0; t < ITEMS; ++t)
#pragma unroll
      for (int u = 0; u < USERS; ++u)
        acc[t][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], y[u], acc[t][u], 0, 0, 0);
  };
#pragma unroll(SPLIT ? 4 : 1)
  for (int s = begin; s < (end < full ? end : full); ++s) step(s, std::false_type{});
  if (full < end && end == steps) step(full, std::true_type{});

  if constexpr (SPLIT) {
    __shared__ i32x4 lds[kWaves - 1][ITEMS * USERS][64];
    if (wave) {
#pragma unroll
      for (int t = 0; t < ITEMS; ++t)
#pragma unroll
        for (int u = 0; u < USERS; ++u) lds[wave - 1][t * USERS + u][lane] = acc[t][u];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int t = 0; t < ITEMS; ++t)
#pragma unroll
      for (int u = 0; u < USERS; ++u)
#pragma unroll
        for (int w = 0; w < kWaves - 1; ++w) acc[t][u] += lds[w][t * USERS + u][lane];
  }
  // lane l holds the sums of items 4 (l / 16) .. + 3 and user l % 16
#pragma unroll
  for (int t = 0; t < ITEMS; ++t) {
    const int64_t j = first + t * 16 + part * 4;
    if (j >= P.items) continue;
    const int left = P.items - j < 4 ? (int)(P.items - j) : 4;
    float b[4] = {};
    if (left == 4) __builtin_memcpy(b, P.b_scale + j, 16);
    else
      for (int i = 0; i < left; ++i) b[i] = P.b_scale[j + i];
#pragma unroll
    for (int u = 0; u < USERS; ++u) {
      const int64_t r = u * 16 + l16;
      if (r >= P.rows) continue;
      const float a = P.a_scale[r];
      O v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = score_of<O>(acc[t][u][i], a, b[i]);
      O *to = static_cast<O *>(P.out) + r * P.out_stride + j;
      if (left == 4) __builtin_memcpy(to, v, 4 * sizeof(O));
      else
        for (int i = 0; i < left; ++i) to[i] = v[i];
    }
  }
}

// Many users: a workgroup of 2 x 2 waves takes a tile of kTile items x kTile
// users, each wave 64 x 64 of it in v_mfma_i32_32x32x32_i8 (lane l holds 16
// bytes of item or user l % 32).  64 columns of k at a time pass through LDS,
// in 16-byte chunks whose place in a row is swizzled so that eight lanes
// reading eight rows meet all banks.  While a step's products are formed the
// next step's bytes are loaded into registers.
constexpr int kTile = 128;
constexpr int kStep = 64;  // bytes of k per step, 4 chunks

__device__ __forceinline__ int lds_chunk(int row, int c) {
  return row * 4 + (c ^ ((row >> 1) & 3));
}

template <class O>
__global__ void __launch_bounds__(kThreads, 2) k_product_many(Product P, int64_t item_tiles,
                                                              int64_t user_tiles) {
  __shared__ i32x4 lds_items[kTile * kStep / 16], lds_users[kTile * kStep / 16];
  __shared__ float s_item[kTile], s_user[kTile];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int wi = wave % 2, wu = wave / 2, l32 = lane % 32, half = lane / 32;
  const int64_t tile = blockIdx.x;
  const int64_t j0 = tile % item_tiles * kTile, r0 = tile / item_tiles * kTile;
  // staging: thread t moves chunk t % 4 of rows t / 4 and t / 4 + 64
  const int chunk = tid % 4, row = tid / 4;
  const int8_t *item[2], *user[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t j = j0 + row + 64 * h, r = r0 + row + 64 * h;
    item[h] = P.b + (j < P.items ? j : P.items - 1) * P.b_stride;
    user[h] = P.a + (r < P.rows ? r : P.rows - 1) * P.kp + chunk * 16;
  }
  if (tid < kTile) s_item[tid] = j0 + tid < P.items ? P.b_scale[j0 + tid] : 0.0f;
  else s_user[tid - kTile] = r0 + tid - kTile < P.rows ? P.a_scale[r0 + tid - kTile] : 0.0f;
  i32x16 acc[2][2] = {};
  const int steps = P.kp / kStep, full = P.k / kStep;
  i32x4 x[2], y[2];
  const auto load = [&](int s) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = s < full ? item_bytes(item[h], s * kStep + chunk * 16)
                      : item_bytes_tail(item[h], s * kStep + chunk * 16, P.k, P.b_end);
      y[h] = *reinterpret_cast<const i32x4 *>(user[h] + s * kStep);
    }
  };
  load(0);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      lds_items[lds_chunk(row + 64 * h, chunk)] = x[h];
      lds_users[lds_chunk(row + 64 * h, chunk)] = y[h];
    }
    __syncthreads();
    if (s + 1 < steps) load(s + 1);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      i32x4 fi[2], fu[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        fi[h] = lds_items[lds_chunk(wi * 64 + h * 32 + l32, c * 2 + half)];
        fu[h] = lds_users[lds_chunk(wu * 64 + h * 32 + l32, c * 2 + half)];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          acc[i][u] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fi[i], fu[u], acc[i][u], 0, 0, 0);
    }
  }
  // register g of a lane is the sum of item 8 (g / 4) + 4 (l / 32) + g % 4 and user l % 32
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int ru = wu * 64 + u * 32 + l32;
      const int64_t r = r0 + ru;
      if (r >= P.rows) continue;
      const float a = s_user[ru];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ji = wi * 64 + i * 32 + g * 8 + half * 4;
        const int64_t j = j0 + ji;
        O v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = score_of<O>(acc[i][u][g * 4 + e], a, s_item[ji + e]);
        O *to = static_cast<O *>(P.out) + r * P.out_stride + j;
        if (j + 4 <= P.items) __builtin_memcpy(to, v, 4 * sizeof(O));
        else
          for (int e = 0; e < 4; ++e)
            if (j + e < P.items) to[e] = v[e];
      }
    }
}

template <class O>
hipError_t product(const Product &p, hipStream_t stream) {
  const auto few = [&](auto users, auto items, auto split) {
    constexpr int U = decltype(users)::value, I = decltype(items)::value;
    constexpr bool S = decltype(split)::value;
    const int64_t per = 16 * I * (S ? 1 : kWaves);
    hipLaunchKernelGGL((k_product_few<O, U, I, S>), dim3((unsigned)((p.items + per - 1) / per)),
                       dim3(kThreads), 0, stream, p);
  };
  using std::integral_constant;
  if (p.rows <= 64) {
    // few tiles and a long k: the waves of a workgroup share a tile
    const bool split = p.items < 16 * 4096 && p.kp >= 512;
    if (p.rows <= 16 && split)
      few(integral_constant<int, 1>{}, integral_constant<int, 1>{}, std::true_type{});
    else if (p.rows <= 16)
      few(integral_constant<int, 1>{}, integral_constant<int, 4>{}, std::false_type{});
    else if (p.rows <= 32 && split)
      few(integral_constant<int, 2>{}, integral_constant<int, 1>{}, std::true_type{});
    else if (p.rows <= 32)
      few(integral_constant<int, 2>{}, integral_constant<int, 4>{}, std::false_type{});
    else if (split)
      few(integral_constant<int, 4>{}, integral_constant<int, 1>{}, std::true_type{});
    else
      few(integral_constant<int, 4>{}, integral_constant<int, 4>{}, std::false_type{});
  } else {
    const int64_t it = (p.items + kTile - 1) / kTile, ut = (p.rows + kTile - 1) / kTile;
    if (it * ut >= (1ll << 24)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(k_product_many<O>, dim3((unsigned)(it * ut)), dim3(kThreads), 0, stream, p,
                       it, ut);
  }
  return hipGetLastError();
}

// Workspace: the users' bytes in the product's layout, then their scales.
int64_t bytes_part(int64_t rows, int64_t k) { return round_up(rows * round_up(k, kUnit), 256); }

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int bgmf_quantize_rows(const void *x, int32_t type, int64_t rows, int64_t k, int64_t row_stride,
                       int8_t *q, int64_t q_stride, float *scale, void *hip_stream) {
  const char *call = "bgmf_quantize_rows";
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (rows < 0 || rows >= (1ll << 31) || k < 1 || k >= (1ll << 30))
    return fail_call(BGMF_E_ARG, "%s: rows must be in [0, 2^31) and k in [1, 2^30): %lld x %lld",
                     call, (long long)rows, (long long)k);
  if (bad_matrix(x, rows, k, row_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad x (pointer, alignment or row stride %lld)", call,
                     (long long)row_stride);
  if (bad_matrix(q, rows, k, q_stride, k, 1))
    return fail_call(BGMF_E_ARG, "%s: bad q (pointer or row stride %lld)", call,
                     (long long)q_stride);
  if (rows == 0) return BGMF_OK;
  if (!scale) return fail_call(BGMF_E_ARG, "%s: null scale", call);
  const hipError_t e = quantize_by_type(type, x, rows, (int32_t)k, row_stride, q, q_stride,
                                        (int32_t)k, scale, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int64_t bgmf_quantized_scores_workspace(int64_t rows, int64_t item_count, int64_t k,
                                        int32_t type) {
  if (rows <= 0 || k <= 0 || item_count <= 0 || rows >= (1ll << 31) || k > BGMF_PRODUCT_K_MAX)
    return 0;
  return bytes_part(rows, k) + (type == BGMF_TYPE_I8 ? 0 : round_up(rows * 4, 256));
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
  const int32_t kp = (int32_t)round_up(k, kUnit);
  int8_t *q = static_cast<int8_t *>(ws);
  Product p{q, row_scale, rows, (int32_t)k, kp, items,
            items + (items_stride * (item_count - 1) + k), item_scale, item_count, items_stride,
            out, out_stride};
  hipError_t e = hipSuccess;
  if (type == BGMF_TYPE_I8) {
    const int64_t groups = std::min<int64_t>((rows * (kp / 16) + kThreads - 1) / kThreads, 4096);
    hipLaunchKernelGGL(k_pad_rows, dim3((unsigned)groups), dim3(kThreads), 0, stream,
                       static_cast<const int8_t *>(x), rows, (int32_t)k, row_stride, q, kp);
    e = hipGetLastError();
  } else {
    float *scale = reinterpret_cast<float *>(q + bytes_part(rows, k));
    e = quantize_by_type(type, x, rows, (int32_t)k, row_stride, q, kp, kp, scale, stream);
    p.a_scale = scale;
  }
  if (e == hipSuccess)
    e = out_type == BGMF_TYPE_F32    ? product<float>(p, stream)
        : out_type == BGMF_TYPE_BF16 ? product<bf16_t>(p, stream)
                                     : product<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
