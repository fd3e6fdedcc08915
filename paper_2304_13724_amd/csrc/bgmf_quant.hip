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
// (kHeld vectors of 16 bytes each), reduce its largest magnitude, and write
// the quotients; what a longer row has beyond that is read a second time.
// Bound: HBM.
// ---------------------------------------------------------------------------
constexpr int kHeld = 4;

// Largest magnitude, +infinity where a value is NaN or infinite.
struct Largest {
  float most = 0.0f;
  bool bad = false;
  __device__ __forceinline__ void look(float x) {
    const float v = fabsf(x);
    bad |= !(v < INFINITY);
    most = fmaxf(most, v);
  }
  __device__ __forceinline__ float get() const { return bad ? INFINITY : most; }
};
// The scale of a row with that magnitude, and a value's byte; NaN and 0 bytes
// where it is infinite.
__device__ __forceinline__ float scale_of(float most) {
  return most == INFINITY ? NAN : most / 127.0f;
}
__device__ __forceinline__ int8_t byte_of(float x, float scale) {
  const float y = scale > 0.0f ? rintf(x / scale) : 0.0f;
  return (int8_t)fminf(fmaxf(y, -127.0f), 127.0f);
}

template <class T, int LANES>
__global__ void __launch_bounds__(kThreads) k_quantize(const T *x, int64_t rows, int32_t k,
                                                       int64_t stride, int8_t *q, int64_t q_stride,
                                                       int32_t fill, float *scale) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x % LANES;
  const int32_t vecs = k / N, tail = vecs * N + lane;
  __shared__ float lds[kWaves];
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES; r < rows;
       r += (int64_t)gridDim.x * (kThreads / LANES)) {
    const T *row = x + r * stride;
    Largest a;
    Vec<T> held[kHeld];
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (lane + h * LANES < vecs) held[h] = load_vec(row + (lane + h * LANES) * N);
      else held[h] = {};
    for (int32_t i = tail; i < k; i += LANES) a.look(to_float(row[i]));
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
#pragma unroll
      for (int i = 0; i < N; ++i) a.look(to_float(held[h].v[i]));
#pragma unroll 4
    for (int32_t v = lane + kHeld * LANES; v < vecs; v += LANES) {
      const Vec<T> more = load_vec(row + v * N);
#pragma unroll
      for (int i = 0; i < N; ++i) a.look(to_float(more.v[i]));
    }
    float most = a.get();
#pragma unroll
    for (int o = LANES < 64 ? LANES / 2 : 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if constexpr (LANES > 64) {
      if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = most;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) most = fmaxf(most, lds[w]);
      __syncthreads();
    }
    const float s = scale_of(most);
    if (lane == 0) scale[r] = s;
    int8_t *to = q + r * q_stride;
    const auto put = [&](int32_t v, const Vec<T> &a) {
      int8_t b[N];
#pragma unroll
      for (int i = 0; i < N; ++i) b[i] = byte_of(to_float(a.v[i]), s);
      __builtin_memcpy(to + v * N, b, N);
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (lane + h * LANES < vecs) put(lane + h * LANES, held[h]);
    for (int32_t v = lane + kHeld * LANES; v < vecs; v += LANES) put(v, load_vec(row + v * N));
    for (int32_t i = tail; i < fill; i += LANES) to[i] = i < k ? byte_of(to_float(row[i]), s) : 0;
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
  const void *x;    // users' values (own_bytes)
  int64_t x_stride;
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

// 16 bytes of an item from column c on, at any address.  STREAM: items that
// the caches cannot keep until the next call are read past them (320 MB: 6.4
// TB/s against 5.9).
template <bool STREAM = false>
__device__ __forceinline__ i32x4 item_bytes(const int8_t *row, int32_t c) {
  typedef int32_t quad __attribute__((ext_vector_type(4), aligned(1)));
  const quad *p = reinterpret_cast<const quad *>(row + c);
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
// The same where c may be at or past the row's end: nothing is read past the
// end of the matrix (of at least 16 bytes), whose last bytes are shifted into
// their place.
__device__ __forceinline__ i32x4 item_bytes_tail(const int8_t *row, int32_t c, int32_t k,
                                                 const int8_t *end) {
  i32x4 x = {0, 0, 0, 0};
  if (c < k) {
    const int64_t past = row + c + 16 - end;
    x = item_bytes(row, (int32_t)(past > 0 ? c - past : c));
    if (past > 0) {
      uint64_t w[2];
      __builtin_memcpy(w, &x, 16);
      const int bits = (int)past * 8;  // 8 to 120
      const uint64_t carried = bits < 64 ? w[1] << (64 - bits) : 0;
      w[0] = bits < 64 ? w[0] >> bits | carried : w[1] >> (bits - 64);
      w[1] = bits < 64 ? w[1] >> bits : 0;
      __builtin_memcpy(&x, w, 16);
    }
  }
  return x;
}

template <class O>
__device__ __forceinline__ O score_of(int32_t sum, float a, float b) {
  return from_float<O>((float)sum * a * b);
}

// Items of less than 16 bytes altogether: one thread per score.
template <class O>
__global__ void __launch_bounds__(kThreads) k_product_tiny(Product P) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < P.rows * P.items;
       i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / P.items, j = i % P.items;
    int32_t sum = 0;
    for (int32_t c = 0; c < P.k; ++c)
      sum += (int32_t)P.a[r * P.kp + c] * P.b[j * P.b_stride + c];
    static_cast<O *>(P.out)[r * P.out_stride + j] =
        score_of<O>(sum, P.a_scale[r], P.b_scale[j]);
  }
}

// Few users (rows <= 16 USERS): every item's bytes go from global memory into
// a matrix instruction once (v_mfma_i32_16x16x64_i8: 16 items x 16 users, 64
// columns of k; lane l holds 16 bytes of item l % 16 and of user l % 16).  A
// wave takes ITEMS tiles of 16 items at a time, and while it forms their
// products the bytes and scales of its next step or tiles are on their way.
// With SPLIT, the waves of a workgroup share the tiles and take a quarter of k
// each.  ODD: k is no multiple of 16, so that a lane's bytes may end inside
// its 16.  Bound: HBM (the items' bytes).
//
// X: int8_t, users' bytes in P.a; or the type of their values in P.x, which
// every wave then turns into bytes itself (one launch less; k <= 64 OWN).
constexpr int kOwnMost = 4;

template <class X, int OWN>
__device__ __forceinline__ float own_bytes(const Product &P, int64_t r, int part, i32x4 (&y)[OWN]) {
  const X *x = static_cast<const X *>(P.x) + r * P.x_stride;
  float v[OWN][16];
  Largest a;
#pragma unroll
  for (int s = 0; s < OWN; ++s) {
    const int32_t c = s * 64 + part * 16;
    if (c + 16 <= P.k) {
      constexpr int N = Vec<X>::N;
#pragma unroll
      for (int h = 0; h < 16 / N; ++h) {
        const Vec<X> w = load_vec(x + c + h * N);
#pragma unroll
        for (int i = 0; i < N; ++i) v[s][h * N + i] = to_float(w.v[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[s][i] = c + i < P.k ? to_float(x[c + i]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) a.look(v[s][i]);
  }
  float most = a.get();
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const float scale = scale_of(most);
#pragma unroll
  for (int s = 0; s < OWN; ++s) {
    int8_t b[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = byte_of(v[s][i], scale);
    __builtin_memcpy(&y[s], b, 16);
  }
  return scale;
}

template <class O, class X, int OWN, int USERS, int ITEMS, bool SPLIT, bool ODD, bool STREAM>
__global__ void __launch_bounds__(kThreads, 4) k_product_few(Product P) {
  static_assert(!OWN || (USERS == 1 && !SPLIT), "own bytes: one tile of users");
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int l16 = lane % 16, part = lane / 16;
  const int64_t tiles = (P.items + 16 * ITEMS - 1) / (16 * ITEMS);
  int64_t tile = SPLIT ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;
  const int64_t stride = SPLIT ? gridDim.x : (int64_t)gridDim.x * kWaves;
  if (tile >= tiles) return;  // with SPLIT, all waves or none

  const int64_t own_row = l16 < P.rows ? l16 : P.rows - 1;
  i32x4 own[OWN ? OWN : 1];
  float a_scale[USERS];
  const int8_t *user[USERS];
  if constexpr (OWN > 0) {
    a_scale[0] = own_bytes<X, OWN>(P, own_row, part, own);
  } else {
#pragma unroll
    for (int u = 0; u < USERS; ++u) {
      const int64_t r = u * 16 + l16 < P.rows ? u * 16 + l16 : P.rows - 1;
      a_scale[u] = P.a_scale[r];
      user[u] = P.a + r * P.kp + part * 16;
    }
  }
  const int steps = P.kp / 64, full = P.k / 64;
  const int begin = SPLIT ? steps * wave / kWaves : 0;
  const int end = SPLIT ? steps * (wave + 1) / kWaves : steps;

  // on its way: the bytes of the next step, and the scales of the next tiles
  // (lane l holds that of item l % 16)
  i32x4 x[ITEMS], y[USERS];
  float scale[ITEMS];
  // the last tiles of several go back so far that all of them are whole (the
  // scores that two waves then form are the same)
  const auto first_of = [&](int64_t t) {
    const int64_t j = t * (16 * ITEMS), most = P.items - 16 * ITEMS;
    return ITEMS > 1 && j > most ? most : j;
  };
  const auto load = [&](int64_t t, int s) {
    const int32_t c = s * 64 + part * 16;
    const int64_t j0 = first_of(t);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      int64_t j = j0 + i * 16 + l16;
      if (ITEMS == 1 && j >= P.items) j = P.items - 1;
      const int8_t *row = P.b + j * P.b_stride;
      if (s < full) x[i] = item_bytes<STREAM>(row, c);
      else if constexpr (ODD) x[i] = item_bytes_tail(row, c, P.k, P.b_end);
      else x[i] = c < P.k ? item_bytes<STREAM>(row, c) : i32x4{0, 0, 0, 0};
      if (s == begin) scale[i] = P.b_scale[j];
    }
    if constexpr (OWN == 0) {
#pragma unroll
      for (int u = 0; u < USERS; ++u) y[u] = *reinterpret_cast<const i32x4 *>(user[u] + s * 64);
    }
  };
  load(tile, begin);
  for (; tile < tiles; tile += stride) {
    i32x4 acc[ITEMS][USERS] = {};
    float b[ITEMS];
    const auto step = [&](int s, const i32x4 *mine) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int u = 0; u < USERS; ++u) {
          const i32x4 other = OWN ? *mine : y[u];
          acc[i][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[i], other, acc[i][u], 0, 0, 0);
        }
      const bool last = s + 1 == end;
      const int64_t next = last ? tile + stride : tile;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) b[i] = scale[i];
      if (next < tiles) load(next, last ? begin : s + 1);
    };
    if constexpr (OWN > 0) {  // the steps are counted out, so that the bytes stay in registers
#pragma unroll
      for (int s = 0; s < OWN; ++s)
        if (s < end) step(s, &own[s]);
    } else {
      for (int s = begin; s < end; ++s) step(s, nullptr);
    }

    if constexpr (SPLIT) {
      __shared__ i32x4 lds[kWaves - 1][ITEMS * USERS][64];
      __syncthreads();  // the last tile's sums have been read
      if (wave) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int u = 0; u < USERS; ++u) lds[wave - 1][i * USERS + u][lane] = acc[i][u];
      }
      __syncthreads();
      if (wave) continue;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int u = 0; u < USERS; ++u)
#pragma unroll
          for (int w = 0; w < kWaves - 1; ++w) acc[i][u] += lds[w][i * USERS + u][lane];
    }
    // lane l holds the sums of items 4 (l / 16) .. + 3 and user l % 16
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int64_t j = first_of(tile) + i * 16 + part * 4;
      float bs[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) bs[e] = __shfl(b[i], part * 4 + e);
      const int left = ITEMS > 1 || P.items - j > 3 ? 4 : (int)(P.items - j);
      if (left <= 0) continue;
#pragma unroll
      for (int u = 0; u < USERS; ++u) {
        const int64_t r = u * 16 + l16;
        if (r >= P.rows) continue;
        O v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = score_of<O>(acc[i][u][e], a_scale[u], bs[e]);
        O *to = static_cast<O *>(P.out) + r * P.out_stride + j;
        if (left == 4) __builtin_memcpy(to, v, 4 * sizeof(O));
        else
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (e < left) to[e] = v[e];
      }
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
  // a step's bytes, and afterwards the scores on their way out
  constexpr int kStage = 2 * kTile * kStep, kScores = kWaves * 32 * (64 * (int)sizeof(O) + 16);
  __shared__ i32x4 lds[(kStage > kScores ? kStage : kScores) / 16];
  i32x4 *lds_items = lds, *lds_users = lds + kTile * kStep / 16;
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
  // Register g of a lane is the sum of item 8 (g / 4) + 4 (l / 32) + g % 4 and
  // user l % 32.  The scores of 32 users at a time pass through LDS, so that a
  // user's 64 scores are stored in a row.
  constexpr int kPitch = 64 + 16 / (int)sizeof(O);  // elements
  __syncthreads();
  O *mine = reinterpret_cast<O *>(lds) + wave * (32 * kPitch);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float a = s_user[wu * 64 + u * 32 + l32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ji = i * 32 + g * 8 + half * 4;
        O v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = score_of<O>(acc[i][u][g * 4 + e], a, s_item[wi * 64 + ji + e]);
        __builtin_memcpy(__builtin_assume_aligned(mine + l32 * kPitch + ji, 4 * sizeof(O)), v,
                         4 * sizeof(O));
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int N = Vec<O>::N, kLanes = 64 / N;  // lanes of a user's row
#pragma unroll
    for (int q = 0; q < 32 * kLanes / 64; ++q) {
      const int ru = q * (64 / kLanes) + lane / kLanes, ji = lane % kLanes * N;
      const Vec<O> v = *reinterpret_cast<const Vec<O> *>(mine + ru * kPitch + ji);
      const int64_t r = r0 + wu * 64 + u * 32 + ru, j = j0 + wi * 64 + ji;
      O *to = static_cast<O *>(P.out) + r * P.out_stride + j;
      if (r < P.rows) {
        if (j + N <= P.items) store_vec(to, v);
        else
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (j + e < P.items) to[e] = v.v[e];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Workgroups that fill the GPU: eight of four waves on each of 256 CUs.
constexpr int64_t kFullGpu = 2048;

constexpr int64_t kCached = 192 << 20;  // items that stay in the 256 MB Infinity Cache

template <class O, class X, int OWN, int USERS, int ITEMS, bool SPLIT>
void launch_few(const Product &p, hipStream_t stream) {
  const int64_t per = 16 * ITEMS * (SPLIT ? 1 : kWaves);
  const dim3 groups((unsigned)std::min((p.items + per - 1) / per, kFullGpu)), threads(kThreads);
  constexpr bool BIG = ITEMS > 1;  // enough items that the caches may not keep them
  if (p.k % 16)
    hipLaunchKernelGGL((k_product_few<O, X, OWN, USERS, ITEMS, SPLIT, true, false>), groups,
                       threads, 0, stream, p);
  else if (BIG && p.b_end - p.b > kCached)
    hipLaunchKernelGGL((k_product_few<O, X, OWN, USERS, ITEMS, SPLIT, false, BIG>), groups,
                       threads, 0, stream, p);
  else
    hipLaunchKernelGGL((k_product_few<O, X, OWN, USERS, ITEMS, SPLIT, false, false>), groups,
                       threads, 0, stream, p);
}

constexpr int64_t kFewUsers = 64;
// Whether the product's waves turn the users' values into bytes themselves.
bool takes_values(int64_t rows, int64_t k, int64_t items_bytes) {
  return rows <= 16 && k <= 64 * kOwnMost && items_bytes >= 16;
}

template <class O, class X>
void launch_values(const Product &p, bool small, hipStream_t stream) {
  if (p.k <= 64) {
    if (small) launch_few<O, X, 1, 1, 1, false>(p, stream);
    else launch_few<O, X, 1, 1, 8, false>(p, stream);
  } else {
    if (small) launch_few<O, X, kOwnMost, 1, 1, false>(p, stream);
    else launch_few<O, X, kOwnMost, 1, 4, false>(p, stream);
  }
}

template <class O>
hipError_t product(const Product &p, int32_t type, hipStream_t stream) {
  const bool small = p.items < 64 * kFullGpu * kWaves;  // less than 64 items for each wave
  if (p.b_end - p.b < 16) {
    const int64_t groups = std::min((p.rows * p.items + kThreads - 1) / kThreads, kFullGpu);
    hipLaunchKernelGGL(k_product_tiny<O>, dim3((unsigned)groups), dim3(kThreads), 0, stream, p);
  } else if (p.x) {
    if (type == BGMF_TYPE_F32) launch_values<O, float>(p, small, stream);
    else if (type == BGMF_TYPE_BF16) launch_values<O, bf16_t>(p, small, stream);
    else launch_values<O, f16_t>(p, small, stream);
  } else if (p.rows <= kFewUsers) {
    // the waves of a workgroup share a tile where the tiles are few and k is long
    const bool split = p.items < 16 * 4096 && p.kp >= 512;
    if (p.rows <= 16) {
      if (split) launch_few<O, int8_t, 0, 1, 1, true>(p, stream);
      else if (small) launch_few<O, int8_t, 0, 1, 1, false>(p, stream);
      else launch_few<O, int8_t, 0, 1, 4, false>(p, stream);
    } else if (p.rows <= 32) {
      if (split) launch_few<O, int8_t, 0, 2, 1, true>(p, stream);
      else if (small) launch_few<O, int8_t, 0, 2, 1, false>(p, stream);
      else launch_few<O, int8_t, 0, 2, 4, false>(p, stream);
    } else {
      if (split) launch_few<O, int8_t, 0, 4, 1, true>(p, stream);
      else if (small) launch_few<O, int8_t, 0, 4, 1, false>(p, stream);
      else launch_few<O, int8_t, 0, 4, 2, false>(p, stream);
    }
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
  Product p{nullptr, 0, q, row_scale, rows, (int32_t)k, kp, items,
            items + (items_stride * (item_count - 1) + k), item_scale, item_count, items_stride,
            out, out_stride};
  hipError_t e = hipSuccess;
  if (type == BGMF_TYPE_I8) {
    const int64_t groups = std::min<int64_t>((rows * (kp / 16) + kThreads - 1) / kThreads, 4096);
    hipLaunchKernelGGL(k_pad_rows, dim3((unsigned)groups), dim3(kThreads), 0, stream,
                       static_cast<const int8_t *>(x), rows, (int32_t)k, row_stride, q, kp);
    e = hipGetLastError();
  } else if (takes_values(rows, k, p.b_end - p.b)) {
    p.x = x, p.x_stride = row_stride;
  } else {
    float *scale = reinterpret_cast<float *>(q + bytes_part(rows, k));
    e = quantize_by_type(type, x, rows, (int32_t)k, row_stride, q, kp, kp, scale, stream);
    p.a_scale = scale;
  }
  if (e == hipSuccess)
    e = out_type == BGMF_TYPE_F32    ? product<float>(p, type, stream)
        : out_type == BGMF_TYPE_BF16 ? product<bf16_t>(p, type, stream)
                                     : product<f16_t>(p, type, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
