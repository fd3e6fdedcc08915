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
// Bound: memory latency (a row's bytes are written after all of it has arrived):
// 4,096 rows of 4,096 bf16 take 17 us, 2.9 TB/s; catalogues of 5M rows of 64 fp32
// 419 us, 3.9 TB/s, of 128 558 us, 5.8 TB/s.
// ---------------------------------------------------------------------------

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
// A row's scale, and its values' bytes; NaN and 0 where the magnitude is
// infinite.  x / scale has to be rounded as by a division.  Where neither it
// nor its remainder can leave the normal range, the product with the rounded
// reciprocal, corrected once by its exact remainder (Markstein's division by
// fused multiply-adds), is that quotient (the error left, 2^-24 units, is less
// than a quotient of fp32 numbers keeps from a rounding boundary; equal to the
// division in 1.7e10 of them, half of these next to ties) in a third of the
// instructions.
struct Scale {
  float s, r;
  bool quick;
  __device__ __forceinline__ explicit Scale(float most) {
    s = most == INFINITY ? NAN : most / 127.0f;
    quick = s >= 0x1p-60f && s <= 0x1p60f;
    r = quick ? 1.0f / s : 0.0f;
  }
  __device__ __forceinline__ int8_t byte(float x) const {
    float y;
    if (quick) {
      y = x * r;
      y = fmaf(fmaf(-y, s, x), r, y);
    } else {
      y = s > 0.0f ? x / s : 0.0f;
    }
    return (int8_t)fminf(fmaxf(rintf(y), -127.0f), 127.0f);
  }
};

template <class T, int LANES>
__global__ void __launch_bounds__(kThreads) k_quantize(const T *x, int64_t rows, int32_t k,
                                                       int64_t stride, int8_t *q, int64_t q_stride,
                                                       int32_t fill, float *scale) {
  constexpr int N = Vec<T>::N, kHeld = LANES < 64 ? 2 : 8;
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
    const Scale s(most);
    if (lane == 0) scale[r] = s.s;
    int8_t *to = q + r * q_stride;
    const auto put = [&](int32_t v, const Vec<T> &a) {
      int8_t b[N];
#pragma unroll
      for (int i = 0; i < N; ++i) b[i] = s.byte(to_float(a.v[i]));
      __builtin_memcpy(to + v * N, b, N);
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (lane + h * LANES < vecs) put(lane + h * LANES, held[h]);
    for (int32_t v = lane + kHeld * LANES; v < vecs; v += LANES) put(v, load_vec(row + v * N));
    for (int32_t i = tail; i < fill; i += LANES) to[i] = i < k ? s.byte(to_float(row[i])) : 0;
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
  // few lanes to a row: short rows share a wave, and a wave that has a row needs
  // no barrier.  fp32 by 4, 16 and 64 lanes: 1M rows of 32 33, 82 and 596 us, 5M of
  // 64 340, 416 and 2868, 500,000 of 128 103, 60 and 306; by 16, 64 and 256:
  // 100,000 rows of 256 30, 65 and 234, of 1,024 145, 96 and 258, 20,000 of 4,096
  // 161, 86 and 78 (18,000 of 64 by 4 and 16: 3.9 and 3.6; 16 of 4,096 by 64 and
  // 256: 6.9 and 3.8)
  if (vecs <= 8) go(std::integral_constant<int, 4>{});
  else if (vecs <= 32) go(std::integral_constant<int, 16>{});
  else if (vecs <= 512) go(std::integral_constant<int, 64>{});
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

// Few users (16 USERS for each blockIdx.y): every item's bytes go from global
// memory into a matrix instruction once (v_mfma_i32_16x16x64_i8: 16 items x 16
// users, 64 columns of k; lane l holds 16 bytes of item l % 16 and of user l %
// 16).  A wave takes ITEMS tiles of 16 items at a time, and while it stores
// their scores the bytes and scales of its next step or tiles are on their way.
// With SPLIT, the waves of a workgroup share the tiles and take a quarter of k
// each.  ODD: k is no multiple of 16, so that a lane's bytes may end inside
// its 16.  Bound: HBM (the items' bytes): one user over 5M items (k = 64) takes
// 62 us, 5.8 TB/s of the 6.4 that loads alone reach.
//
// X: int8_t, users' bytes in P.a; or the type of their values in P.x, which
// every wave then turns into bytes itself (k <= 64: one launch less, 16
// quotients a lane; with four times as many the waves spend more on them than
// the launch costs: 16 x 100,003 x 200 23 us against 11 with a launch).
template <class X>
__device__ __forceinline__ float own_bytes(const Product &P, int64_t r, int part, i32x4 &y) {
  const X *x = static_cast<const X *>(P.x) + r * P.x_stride;
  float v[16];
  Largest a;
  const int32_t c = part * 16;
  if (c + 16 <= P.k) {
    constexpr int N = Vec<X>::N;
#pragma unroll
    for (int h = 0; h < 16 / N; ++h) {
      const Vec<X> w = load_vec(x + c + h * N);
#pragma unroll
      for (int i = 0; i < N; ++i) v[h * N + i] = to_float(w.v[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = c + i < P.k ? to_float(x[c + i]) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) a.look(v[i]);
  float most = a.get();
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const Scale s(most);
  int8_t b[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) b[i] = s.byte(v[i]);
  __builtin_memcpy(&y, b, 16);
  return s.s;
}

template <class O, class X, int USERS, int ITEMS, bool SPLIT, bool ODD, bool STREAM>
__global__ void __launch_bounds__(kThreads, 4) k_product_few(Product P) {
  constexpr bool OWN = !std::is_same<X, int8_t>::value;
  static_assert(!OWN || (USERS == 1 && !SPLIT), "own bytes: one tile of users");
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int l16 = lane % 16, part = lane / 16;
  const int64_t tiles = (P.items + 16 * ITEMS - 1) / (16 * ITEMS);
  int64_t tile = SPLIT ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;
  const int64_t stride = SPLIT ? gridDim.x : (int64_t)gridDim.x * kWaves;
  if (tile >= tiles) return;  // with SPLIT, all waves or none

  const int64_t r0 = (int64_t)blockIdx.y * (16 * USERS);
  const int64_t own_row = l16 < P.rows ? l16 : P.rows - 1;
  i32x4 own;
  float a_scale[USERS];
  const int8_t *user[USERS];
  if constexpr (OWN) {
    a_scale[0] = own_bytes<X>(P, own_row, part, own);
  } else {
#pragma unroll
    for (int u = 0; u < USERS; ++u) {
      const int64_t j = r0 + u * 16 + l16, r = j < P.rows ? j : P.rows - 1;
      a_scale[u] = P.a_scale[r];
      user[u] = P.a + r * P.kp + part * 16;
    }
  }
  const int steps = P.kp / 64, full = P.k / 64;
  const int begin = SPLIT ? steps * wave / kWaves : 0;
  const int end = SPLIT ? steps * (wave + 1) / kWaves : steps;

  // on its way: the bytes of the next AHEAD steps, and the scales of the next
  // tiles (lane l holds that of item l % 16)
  constexpr int AHEAD = ITEMS > 1 || OWN ? 1 : USERS > 2 ? 2 : 4;
  i32x4 x[AHEAD][ITEMS], y[AHEAD][USERS];
  float scale[ITEMS];
  // the last tiles of several go back so far that all of them are whole (the
  // scores that two waves then form are the same)
  const auto first_of = [&](int64_t t) {
    const int64_t j = t * (16 * ITEMS), most = P.items - 16 * ITEMS;
    return ITEMS > 1 && j > most ? most : j;
  };
  const auto load = [&](int64_t t, int s0) {
    const int64_t j0 = first_of(t);
    const int8_t *row[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      int64_t j = j0 + i * 16 + l16;
      if (ITEMS == 1 && j >= P.items) j = P.items - 1;
      row[i] = P.b + j * P.b_stride;
      if (s0 == begin) scale[i] = P.b_scale[j];
    }
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      const int s = s0 + p;
      const int32_t c = s * 64 + part * 16;
      if (s < full && s < end) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) x[p][i] = item_bytes<STREAM>(row[i], c);
      } else {  // the end of k, and steps past it
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          if constexpr (ODD) x[p][i] = item_bytes_tail(row[i], c, s < end ? P.k : 0, P.b_end);
          else x[p][i] = s < end && c < P.k ? item_bytes<STREAM>(row[i], c) : i32x4{0, 0, 0, 0};
        }
      }
      if constexpr (!OWN) {
#pragma unroll
        for (int u = 0; u < USERS; ++u)
          y[p][u] = *reinterpret_cast<const i32x4 *>(user[u] + (s < end ? s : s0) * 64);
      }
    }
  };
  load(tile, begin);
  for (; tile < tiles; tile += stride) {
    i32x4 acc[ITEMS][USERS] = {};
    float b[ITEMS];
    for (int s0 = begin; s0 < end; s0 += AHEAD) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int u = 0; u < USERS; ++u) {
            const i32x4 other = OWN ? own : y[p][u];
            acc[i][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[p][i], other, acc[i][u], 0, 0, 0);
          }
      const bool last = s0 + AHEAD >= end;
      const int64_t next = last ? tile + stride : tile;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) b[i] = scale[i];
      if (next < tiles) load(next, last ? begin : s0 + AHEAD);
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
        const int64_t r = r0 + u * 16 + l16;
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

// Many users: a workgroup of 2 x 2 waves takes tiles of 64 BI items x 64 BU
// users, each wave a quarter of it in BI x BU blocks of v_mfma_i32_32x32x32_i8
// (lane l holds 16 bytes of item or user l % 32).  STEP bytes of k at a time
// pass through LDS, in 16-byte chunks whose place in a row is swizzled so that
// 16 lanes that read 16 rows meet all 64 banks (places by eight rows, as for 32
// banks, cost a third of the LDS cycles in conflicts).  items >= 64 BI; the users'
// bytes are allocated up to a multiple of kUserPad rows.
constexpr int64_t kUserPad = 256;

template <class O, int BI, int BU, int STEP>
struct Many {
  static constexpr int kItems = 64 * BI, kUsers = 64 * BU, kChunks = STEP / 16;
  static constexpr int kPass = kThreads / kChunks;  // rows that the workgroup loads at a time
  static constexpr int kItemLoads = kItems / kPass, kUserLoads = kUsers / kPass;  // of a thread
  static constexpr int kBuffer = (kItems + kUsers) * kChunks;  // i32x4 of a step
  static constexpr int kPitch = 32 * BI + 16 / (int)sizeof(O);  // of the scores on their way out
  static constexpr int kScores = kWaves * 32 * kPitch * (int)sizeof(O) / 16;  // i32x4

  static __device__ __forceinline__ int at(int row, int c) {
    if constexpr (STEP == 64) return row * 4 + (c ^ ((row >> 2) & 3));
    else return row * 8 + (c ^ ((row >> 1) & 7));
  }

  // Tile t in the order in which workgroups take them: these go to the eight
  // XCDs in turn, and each XCD gets a part of the tiles of its own, four users'
  // tiles by one items' after another, so that its L2 serves many of them.  The
  // last items' tile goes back so far that it is whole.
  static __device__ __forceinline__ void place(const Product &P, int64_t t, int64_t &j0,
                                               int64_t &r0) {
    const int64_t item_tiles = (P.items + kItems - 1) / kItems;
    const int64_t user_tiles = (P.rows + kUsers - 1) / kUsers, tiles = item_tiles * user_tiles;
    const int64_t xcd = t % 8, per = tiles / 8, more = tiles % 8;
    const int64_t i = xcd * per + (xcd < more ? xcd : more) + t / 8;
    constexpr int64_t kGroup = 4;
    const int64_t group = i / (kGroup * item_tiles), in = i % (kGroup * item_tiles);
    const int64_t left = user_tiles - group * kGroup, size = left < kGroup ? left : kGroup;
    j0 = in / size * kItems;
    if (j0 > P.items - kItems) j0 = P.items - kItems;
    r0 = (group * kGroup + in % size) * kUsers;
  }

  // A thread's 16-byte chunks of step s of the items from j0 on.  FULL: the step
  // lies within k.
  template <bool ODD, bool FULL = false>
  static __device__ __forceinline__ void load_items(const Product &P, int64_t j0, int s,
                                                    i32x4 (&x)[kItemLoads]) {
    const int row = threadIdx.x / kChunks;
    const int32_t c = s * STEP + threadIdx.x % kChunks * 16;
    const int8_t *b = P.b + (j0 + row) * P.b_stride;
    if (FULL || (s + 1) * STEP <= P.k) {
#pragma unroll
      for (int h = 0; h < kItemLoads; ++h) x[h] = item_bytes(b + h * kPass * P.b_stride, c);
    } else {
#pragma unroll
      for (int h = 0; h < kItemLoads; ++h) {
        if constexpr (ODD) x[h] = item_bytes_tail(b + h * kPass * P.b_stride, c, P.k, P.b_end);
        else x[h] = c < P.k ? item_bytes(b + h * kPass * P.b_stride, c) : i32x4{0, 0, 0, 0};
      }
    }
  }
  // The same of the users from r0 on.
  template <bool FULL = false>
  static __device__ __forceinline__ void load_users(const Product &P, int64_t r0, int s,
                                                    i32x4 (&y)[kUserLoads]) {
    const int32_t c = s * STEP + threadIdx.x % kChunks * 16;
    const int8_t *a = P.a + (r0 + threadIdx.x / kChunks) * P.kp + c;
    if (FULL || STEP <= kUnit || c < P.kp) {
#pragma unroll
      for (int h = 0; h < kUserLoads; ++h)
        y[h] = *reinterpret_cast<const i32x4 *>(a + (int64_t)h * kPass * P.kp);
    }
  }
  // The users' values in place of bytes, for k <= STEP = 64: the four threads of
  // a row turn them into bytes, and the first writes the row's scale.
  template <class X>
  struct Values {
    Vec<X> v[16 / Vec<X>::N];
  };
  template <bool ODD, class X>
  static __device__ __forceinline__ void load_values(const Product &P, int64_t r0,
                                                     Values<X> (&y)[kUserLoads]) {
    constexpr int N = Vec<X>::N;
    const int32_t c = threadIdx.x % kChunks * 16;
#pragma unroll
    for (int h = 0; h < kUserLoads; ++h) {
      const int64_t j = r0 + threadIdx.x / kChunks + h * kPass, r = j < P.rows ? j : P.rows - 1;
      const X *x = static_cast<const X *>(P.x) + r * P.x_stride + c;
      if (c + 16 <= P.k) {
#pragma unroll
        for (int i = 0; i < 16 / N; ++i) y[h].v[i] = load_vec(x + i * N);
      } else {
#pragma unroll
        for (int i = 0; i < 16 / N; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e)
            y[h].v[i].v[e] = ODD && c + i * N + e < P.k ? x[i * N + e] : from_float<X>(0.0f);
      }
    }
  }
  template <class X>
  static __device__ __forceinline__ void to_bytes(const Values<X> (&values)[kUserLoads],
                                                  i32x4 (&y)[kUserLoads], float *s_user) {
    constexpr int N = Vec<X>::N;
#pragma unroll
    for (int h = 0; h < kUserLoads; ++h) {
      Largest a;
#pragma unroll
      for (int i = 0; i < 16; ++i) a.look(to_float(values[h].v[i / N].v[i % N]));
      float most = a.get();
      most = fmaxf(most, __shfl_xor(most, 1));
      most = fmaxf(most, __shfl_xor(most, 2));
      const Scale s(most);
      int8_t b[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) b[i] = s.byte(to_float(values[h].v[i / N].v[i % N]));
      __builtin_memcpy(&y[h], b, 16);
      if (threadIdx.x % kChunks == 0) s_user[threadIdx.x / kChunks + h * kPass] = s.s;
    }
  }
  static __device__ __forceinline__ void store(i32x4 *buffer, const i32x4 (&x)[kItemLoads],
                                               const i32x4 (&y)[kUserLoads]) {
    const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
#pragma unroll
    for (int h = 0; h < kItemLoads; ++h) buffer[at(row + kPass * h, chunk)] = x[h];
#pragma unroll
    for (int h = 0; h < kUserLoads; ++h)
      buffer[kItems * kChunks + at(row + kPass * h, chunk)] = y[h];
  }
  // A wave's bytes of 32 columns of k.
  static __device__ __forceinline__ void read(const i32x4 *buffer, int sub, i32x4 (&fi)[BI],
                                              i32x4 (&fu)[BU]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int c = sub * 2 + lane / 32;
#pragma unroll
    for (int h = 0; h < BI; ++h) fi[h] = buffer[at((wave % 2 * BI + h) * 32 + lane % 32, c)];
#pragma unroll
    for (int h = 0; h < BU; ++h)
      fu[h] = buffer[kItems * kChunks + at((wave / 2 * BU + h) * 32 + lane % 32, c)];
  }
  static __device__ __forceinline__ void multiply(i32x16 (&acc)[BI][BU], const i32x4 (&fi)[BI],
                                                  const i32x4 (&fu)[BU]) {
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int u = 0; u < BU; ++u)
        acc[i][u] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fi[i], fu[u], acc[i][u], 0, 0, 0);
  }
  // The scales of the tile's items, then of its users if they came as bytes
  // (those past the last user's are not used).
  static constexpr int kScaleLoads = (kItems + kUsers + kThreads - 1) / kThreads;
  static __device__ __forceinline__ void load_scales(const Product &P, int64_t j0, int64_t r0,
                                                     float (&scale)[kScaleLoads]) {
#pragma unroll
    for (int h = 0; h < kScaleLoads; ++h) {
      const int i = threadIdx.x + h * kThreads;
      const int64_t r = r0 + i - kItems;
      if (i < kItems) scale[h] = P.b_scale[j0 + i];
      else if (P.a_scale) scale[h] = P.a_scale[r < P.rows ? r : P.rows - 1];
    }
  }

  // Register g of a lane is the sum of item 8 (g / 4) + 4 (l / 32) + g % 4 and
  // user l % 32.  The scores of 32 users at a time pass through LDS (lds: the
  // whole workgroup's), so that a user's 32 BI scores are stored in a row.
  static __device__ __forceinline__ void store_scores(const Product &P, int64_t j0, int64_t r0,
                                                      const i32x16 (&acc)[BI][BU], i32x4 *lds,
                                                      const float *s_item) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wi = wave % 2, wu = wave / 2, l32 = lane % 32, half = lane / 32;
    const float *s_user = s_item + kItems;
    O *mine = reinterpret_cast<O *>(lds) + wave * (32 * kPitch);
    constexpr int N = Vec<O>::N, kLanes = 32 * BI / N;  // lanes of a user's row
#pragma unroll
    for (int u = 0; u < BU; ++u) {
      const float a = s_user[(wu * BU + u) * 32 + l32];
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int ji = i * 32 + g * 8 + half * 4;
          O v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = score_of<O>(acc[i][u][g * 4 + e], a, s_item[wi * BI * 32 + ji + e]);
          __builtin_memcpy(__builtin_assume_aligned(mine + l32 * kPitch + ji, 4 * sizeof(O)), v,
                           4 * sizeof(O));
        }
      __builtin_amdgcn_wave_barrier();
      const int64_t r1 = r0 + (wu * BU + u) * 32 + lane / kLanes;
      const int ji = lane % kLanes * N;
      O *to = static_cast<O *>(P.out) + r1 * P.out_stride + (j0 + wi * BI * 32 + ji);
#pragma unroll
      for (int q = 0; q < 32 * kLanes / 64; ++q) {
        const int ru = q * (64 / kLanes);
        const Vec<O> v =
            *reinterpret_cast<const Vec<O> *>(mine + (ru + lane / kLanes) * kPitch + ji);
        if (r1 + ru < P.rows) store_vec(to + ru * P.out_stride, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// Tiles of 128 or 64 items x 128 or 64 users, 64 bytes of k at a time: three or
// four workgroups on a CU overlap their loads, products and stores.  A
// workgroup's bytes of the next step, or of its next tile, are on their way into
// registers meanwhile.  Bound: HBM (the scores) up to k of some hundred: 2,048
// users x 18,000 items, k = 64, bf16 takes 17 us, 4.3 TB/s.
template <class O, class X, int BI, int BU, bool ODD>
__global__ void __launch_bounds__(kThreads, BI * BU == 4 ? 3 : 4) k_product_many(Product P, int64_t tiles) {
  using M = Many<O, BI, BU, 64>;
  constexpr bool OWN = !std::is_same<X, int8_t>::value;
  __shared__ i32x4 lds[M::kBuffer > M::kScores ? M::kBuffer : M::kScores];
  __shared__ float s_item[M::kScaleLoads * kThreads];
  const int steps = P.kp / 64;
  i32x4 x[M::kItemLoads], y[M::kUserLoads];
  typename M::template Values<typename std::conditional<OWN, X, float>::type>
      values[M::kUserLoads];
  float scale[M::kScaleLoads];
  const auto load = [&](int64_t j0, int64_t r0, int s) {
    M::template load_items<ODD>(P, j0, s, x);
    if constexpr (OWN) M::template load_values<ODD>(P, r0, values);
    else M::load_users(P, r0, s, y);
    if (s == 0) M::load_scales(P, j0, r0, scale);
  };
  i32x16 acc[BI][BU] = {};
  int64_t tile = blockIdx.x, j0, r0;
  M::place(P, tile, j0, r0);
  load(j0, r0, 0);
  for (int s = 0; tile < tiles;) {
    __syncthreads();
    if constexpr (OWN) M::to_bytes(values, y, s_item + M::kItems);
    M::store(lds, x, y);
    if (s == 0 && (!OWN || (int)threadIdx.x < M::kItems)) s_item[threadIdx.x] = scale[0];
    __syncthreads();
    const bool last = s + 1 == steps;
    int64_t jn = j0, rn = r0;
    const int64_t next = last ? tile + gridDim.x : tile;
    if (next < tiles) {
      if (last) M::place(P, next, jn, rn);
      load(jn, rn, last ? 0 : s + 1);
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      i32x4 fi[BI], fu[BU];
      M::read(lds, sub, fi, fu);
      M::multiply(acc, fi, fu);
    }
    ++s;
    if (last) {
      __syncthreads();
      M::store_scores(P, j0, r0, acc, lds, s_item);
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int u = 0; u < BU; ++u) acc[i][u] = i32x16{};
      tile = next, j0 = jn, r0 = rn, s = 0;
    }
  }
}

// Long k: tiles of 256 x 256, 128 bytes of k at a time, which halves the LDS
// traffic per product (LDS would bound the smaller tile before the matrix units
// do).  One workgroup fills a CU, so a wave itself reads its next 32 columns
// from LDS while the matrix unit works, and a step's bytes are loaded a whole
// step before they go to the other LDS buffer.  Bound: the matrix units, which
// work 56% of the cycles; the clock falls to about 1.75 GHz meanwhile.  4,096 x
// 8,192 x 4,096 to bf16 takes 137 us, 2.0e15 operations a second (the library's
// int8 product of these sizes: 141 us).  To fp32, where the stores need more
// registers (8 bytes a lane in scratch), it takes 12 us more.
// Kinds of instructions that the scheduler is told to place.
constexpr int kMfma = 0x8, kVmemRead = 0x20, kDsRead = 0x100, kDsWrite = 0x200;

template <class O, bool ODD>
__global__ void __launch_bounds__(kThreads, 1) k_product_large(Product P) {
  using M = Many<O, 4, 4, 128>;
  __shared__ i32x4 lds[2 * M::kBuffer > M::kScores ? 2 * M::kBuffer : M::kScores];
  __shared__ float s_item[M::kScaleLoads * kThreads];
  const int steps = (P.k + 127) / 128;
  int64_t j0, r0;
  M::place(P, blockIdx.x, j0, r0);
  i32x4 x[M::kItemLoads], y[M::kUserLoads];
  M::template load_items<ODD>(P, j0, 0, x);
  M::load_users(P, r0, 0, y);
  {
    float scale[M::kScaleLoads];
    M::load_scales(P, j0, r0, scale);
#pragma unroll
    for (int h = 0; h < M::kScaleLoads; ++h) s_item[threadIdx.x + h * kThreads] = scale[h];
  }
  M::store(lds, x, y);
  if (steps > 1) {
    M::template load_items<ODD>(P, j0, 1, x);
    M::load_users(P, r0, 1, y);
  }
  __syncthreads();
  i32x16 acc[4][4] = {};
  i32x4 fi[2][4], fu[2][4];
  M::read(lds, 0, fi[0], fu[0]);
  // Between two barriers: 48 products with the reads of the next columns, the
  // writes of the next step and the loads of the one after it spread over them.
  const int full = P.k / 128;
  int s = 0;
  for (; s + 2 < full; ++s) {
    i32x4 *now = lds + s % 2 * M::kBuffer, *other = lds + (s + 1) % 2 * M::kBuffer;
    M::read(now, 1, fi[1], fu[1]);
    M::multiply(acc, fi[0], fu[0]);
    M::read(now, 2, fi[0], fu[0]);
    M::multiply(acc, fi[1], fu[1]);
    M::read(now, 3, fi[1], fu[1]);
    M::multiply(acc, fi[0], fu[0]);
    M::store(other, x, y);
    M::template load_items<ODD, true>(P, j0, s + 2, x);
    M::template load_users<true>(P, r0, s + 2, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i % 2 == 0) __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
      __builtin_amdgcn_sched_group_barrier(kDsWrite, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kVmemRead, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    }
    __syncthreads();
    M::read(other, 0, fi[0], fu[0]);
    M::multiply(acc, fi[1], fu[1]);
  }
  for (; s < steps; ++s) {  // the last steps, where nothing or less follows
    i32x4 *now = lds + s % 2 * M::kBuffer, *other = lds + (s + 1) % 2 * M::kBuffer;
    M::read(now, 1, fi[1], fu[1]);
    M::multiply(acc, fi[0], fu[0]);
    M::read(now, 2, fi[0], fu[0]);
    M::multiply(acc, fi[1], fu[1]);
    M::read(now, 3, fi[1], fu[1]);
    M::multiply(acc, fi[0], fu[0]);
    if (s + 1 < steps) {
      M::store(other, x, y);
      if (s + 2 < steps) {
        M::template load_items<ODD>(P, j0, s + 2, x);
        M::load_users(P, r0, s + 2, y);
      }
    }
    __syncthreads();
    if (s + 1 < steps) M::read(other, 0, fi[0], fu[0]);
    M::multiply(acc, fi[1], fu[1]);
  }
  __syncthreads();
  M::store_scores(P, j0, r0, acc, lds, s_item);
}

// Workgroups that fill the GPU: eight of four waves on each of 256 CUs.
constexpr int64_t kFullGpu = 2048;

constexpr int64_t kCached = 192 << 20;  // items that stay in the 256 MB Infinity Cache

template <class O, class X, int USERS, int ITEMS, bool SPLIT>
void launch_few(Product p, hipStream_t stream) {
  const int64_t per = 16 * ITEMS * (SPLIT ? 1 : kWaves), all = (p.items + per - 1) / per;
  // equally many tiles for each
  const int64_t rounds = (all + kFullGpu - 1) / kFullGpu, groups = (all + rounds - 1) / rounds;
  constexpr bool BIG = ITEMS > 1;  // enough items that the caches may not keep them
  constexpr int64_t kMost = 65535ll * 16 * USERS;  // users of a launch
  for (int64_t left = p.rows; left > 0; left -= kMost) {
    p.rows = std::min(left, kMost);
    const dim3 grid((unsigned)groups, (unsigned)((p.rows + 16 * USERS - 1) / (16 * USERS)));
    if (p.k % 16)
      hipLaunchKernelGGL((k_product_few<O, X, USERS, ITEMS, SPLIT, true, false>), grid,
                         dim3(kThreads), 0, stream, p);
    else if (BIG && p.b_end - p.b > kCached)
      hipLaunchKernelGGL((k_product_few<O, X, USERS, ITEMS, SPLIT, false, BIG>), grid,
                         dim3(kThreads), 0, stream, p);
    else
      hipLaunchKernelGGL((k_product_few<O, X, USERS, ITEMS, SPLIT, false, false>), grid,
                         dim3(kThreads), 0, stream, p);
    if (left > kMost) {
      p.a += kMost * p.kp, p.a_scale += kMost;
      p.out = static_cast<O *>(p.out) + kMost * p.out_stride;
    }
  }
}

constexpr int64_t kFewUsers = 16, kFewItems = 128;
// Whether the product itself turns the users' values into bytes: one launch less
// (64 x 18,000 x 64, 282 tiles, 4.6 us against 5.8; 512 users 9.5 against 10.3;
// 4,000 x 3,000, 1,512 tiles, 10.8 against 12.0).  Each tile quantises its users
// again, so with many of them the launch is cheaper (100 x 125,000, 1,954 tiles,
// 14.1 us against 12.3; 2,048 x 18,000 24.7 against 20.3).
bool takes_values(int64_t rows, int64_t items, int64_t k, int64_t items_bytes) {
  if (k > 64 || items_bytes < 16) return false;  // (fewer bytes: k_product_tiny)
  return rows <= kFewUsers ||
         (items >= kFewItems && (items + 127) / 128 * ((rows + 63) / 64) <= 1536);
}

template <class O, class X, int BI, int BU>
void launch_many(const Product &p, hipStream_t stream) {
  const int64_t all =
      (p.items + 64 * BI - 1) / (64 * BI) * ((p.rows + 64 * BU - 1) / (64 * BU));
  constexpr int64_t kAtOnce = 256 * (BI * BU == 4 ? 3 : 4);
  const dim3 groups((unsigned)std::min(all, kAtOnce)), threads(kThreads);
  if (p.k % 16)
    hipLaunchKernelGGL((k_product_many<O, X, BI, BU, true>), groups, threads, 0, stream, p, all);
  else
    hipLaunchKernelGGL((k_product_many<O, X, BI, BU, false>), groups, threads, 0, stream, p, all);
}

// X: int8_t, or the type of the users' values that the product itself quantises.
template <class O, class X>
void launch_product(const Product &p, hipStream_t stream) {
  constexpr bool OWN = !std::is_same<X, int8_t>::value;
  // Less than 64 items for each wave: one tile at a time.  Several make their
  // loads overlap: one user, k = 64, 100,000 items 5.4 us one at a time and 4.2
  // eight at a time, 524,288 10.1 and 9.2, 5M 80 and 64; k = 100 from bytes, one
  // and four at a time, 100,000 6.5 and 6.3, 400,000 13.2 and 11.9, 5M 137 and 132.
  const bool small = p.items < 64 * kFullGpu * kWaves;
  // Few tiles and a long k: the waves of a workgroup share a tile.  One user,
  // shared and not: k = 512 2,048 items 5.3 and 6.3 us, 16,384 6.4 and 6.3, 32,768
  // 9.0 and 8.3; k = 1,024 5.7 and 8.1, 8.6 and 9.3, 10.9 and 10.9; k = 256 5.1 and
  // 5.4, 5.9 and 5.3.  64 users, shared and in tiles of 64 x 64: k = 512 4,096
  // items 8.0 and 9.1, 8,192 10.4 and 9.3; k = 1,024 8.7 and 12.7, 12.2 and 13.2,
  // 16,384 18.3 and 14.6; k = 4,096 17.9 and 34.5, 28.6 and 35.1, 50.5 and 35.9.
  const bool split = !OWN && p.items < (p.rows <= 16 ? 32768 : 8193) && p.kp >= 512;
  const auto tiles = [&](int64_t items, int64_t users) {
    return (p.items + items - 1) / items * ((p.rows + users - 1) / users);
  };
  if (p.rows <= kFewUsers) {
    if constexpr (OWN) {
      if (small) launch_few<O, X, 1, 1, false>(p, stream);
      else launch_few<O, X, 1, 8, false>(p, stream);
    } else {
      if (split) launch_few<O, X, 1, 1, true>(p, stream);
      else if (small) launch_few<O, X, 1, 1, false>(p, stream);
      else launch_few<O, X, 1, 4, false>(p, stream);
    }
    return;
  }
  if constexpr (!OWN) {
    // (fewer than 128 items: 100 x 100 x 256 6.5 us against 7.1 in tiles of 64 x 64)
    if (p.items < kFewItems || (p.rows <= 64 && split)) {
      if (split) launch_few<O, X, 2, 1, true>(p, stream);
      else launch_few<O, X, 2, 1, false>(p, stream);
      return;
    }
    // 256 x 256 and 128 x 128, to bf16: 4,096 x 8,192 (512 tiles), k = 256 32 and 27
    // us, 512 40 and 40, 768 49 and 53, 1,024 57 and 65, 4,096 154 and 215 (to fp32:
    // 512 60 and 55, 1,024 75 and 79); 2,048 x 4,096 (128 tiles), k = 1,024 27 and
    // 22, 4,096 62 and 60
    if (p.k >= 512 && p.items >= 256 && tiles(256, 256) >= 256) {
      const dim3 groups((unsigned)tiles(256, 256)), threads(kThreads);
      if (p.k % 16)
        hipLaunchKernelGGL((k_product_large<O, true>), groups, threads, 0, stream, p);
      else hipLaunchKernelGGL((k_product_large<O, false>), groups, threads, 0, stream, p);
      return;
    }
    // the largest tiles of which every CU gets one: 128 x 128, 128 x 64 and 64 x 64
    // take 20, 20 and 25 us for 2,048 x 18,000 x 64 to bf16, 9.1, 8.0 and 7.8 for
    // 128 x 16,384 x 72 to fp32
    if (p.rows > 64 && tiles(128, 128) >= 256) {
      launch_many<O, X, 2, 2>(p, stream);
      return;
    }
  }
  // (values take the registers that a second 64 users would need)
  if (tiles(128, 64) >= 256) launch_many<O, X, 2, 1>(p, stream);
  else launch_many<O, X, 1, 1>(p, stream);
}

template <class O>
hipError_t product(const Product &p, int32_t type, hipStream_t stream) {
  if (p.b_end - p.b < 16) {
    const int64_t groups = std::min((p.rows * p.items + kThreads - 1) / kThreads, kFullGpu);
    hipLaunchKernelGGL(k_product_tiny<O>, dim3((unsigned)groups), dim3(kThreads), 0, stream, p);
  } else if (!p.x) {
    launch_product<O, int8_t>(p, stream);
  } else if (type == BGMF_TYPE_F32) {
    launch_product<O, float>(p, stream);
  } else if (type == BGMF_TYPE_BF16) {
    launch_product<O, bf16_t>(p, stream);
  } else {
    launch_product<O, f16_t>(p, stream);
  }
  return hipGetLastError();
}

// Workspace: the users' bytes in the product's layout, then their scales.
int64_t bytes_part(int64_t rows, int64_t k) {
  if (rows > kFewUsers) rows = round_up(rows, kUserPad);
  return round_up(rows * round_up(k, kUnit), 256);
}

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
  if (share(q, BGMF_TYPE_I8, rows, k, q_stride, x, type, rows, k, row_stride) ||
      share(scale, BGMF_TYPE_F32, 1, rows, rows, x, type, rows, k, row_stride) ||
      share(scale, BGMF_TYPE_F32, 1, rows, rows, q, BGMF_TYPE_I8, rows, k, q_stride))
    return fail_call(BGMF_E_ARG, "%s: q or scale shares memory with another argument", call);
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
  const auto shares = [&](const void *y, int32_t y_type, int64_t y_rows, int64_t y_cols,
                          int64_t y_stride) {
    return share(out, out_type, rows, item_count, out_stride, y, y_type, y_rows, y_cols, y_stride);
  };
  if (shares(x, type, rows, k, row_stride) ||
      shares(items, BGMF_TYPE_I8, item_count, k, items_stride) ||
      shares(row_scale, BGMF_TYPE_F32, 1, rows, rows) ||
      shares(item_scale, BGMF_TYPE_F32, 1, item_count, item_count))
    return fail_call(BGMF_E_ARG, "%s: out shares memory with an input", call);
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
  } else if (takes_values(rows, item_count, k, p.b_end - p.b)) {
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
