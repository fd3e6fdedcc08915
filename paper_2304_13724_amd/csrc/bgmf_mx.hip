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
// threads to a row.  Bound: HBM: 625,000 rows of 128 fp32 take 74 us, 4.9 TB/s, and
// 33 us back to bf16 (6.1 TB/s); latency where there is little: 4,096 rows of 4,096
// bf16 8.8 us, 1,999 of 200 2.9.  (Long rows four chunks of a thread at a time:
// 10.0 us; a workgroup to each 256 chunks: 9.4.)
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
  const void *x;  // users' values, rows of k, where the product itself quantises them
  int64_t x_stride;
  int32_t k;
  const uint8_t *a, *a_scale;  // users: rows of `blocks` blocks
  int64_t rows, a_stride, as_stride;
  const uint8_t *b, *b_scale;  // items
  int64_t items, b_stride, bs_stride;
  int32_t blocks;
  void *out;
  int64_t out_stride;
};

// v_mfma_scale_f32_32x32x64_f8f6f4 on 4-bit values: lane l holds block l / 32
// (of two) of row l % 32 of either side, and in byte SEL of a word its scale.
// Register g of a lane is the sum of row 8 (g / 4) + 4 (l / 32) + g % 4 of a and
// row l % 32 of b.
template <int SEL>
__device__ __forceinline__ f32x16 multiply(i32x4 a, int a_scale, i32x4 b, int b_scale, f32x16 c) {
  const i32x8 x = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, y = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, SEL, a_scale, SEL,
                                                         b_scale);
}

// 16 bytes at any address.  STREAM: items that the caches cannot keep until the
// next call are read past them.
template <bool STREAM = false>
__device__ __forceinline__ i32x4 block_bytes(const uint8_t *p) {
  typedef int32_t quad __attribute__((ext_vector_type(4), aligned(1)));
  const quad *q = reinterpret_cast<const quad *>(p);
  if constexpr (STREAM) return __builtin_nontemporal_load(q);
  else return *q;
}

// Few users (32 for each blockIdx.y): every item's bytes go from global memory
// into a matrix instruction once.  A wave takes a tile of 32 items and STEPS pairs
// of blocks at a time; while it stores their scores, the bytes and scales of its
// next ones are on their way.  LONG: rows of more than STEPS pairs.
//
// X: uint8_t, users' bytes in P.a; or the type of their values in P.x (rows of at
// most kOwnBlocks blocks), which every workgroup then quantises into LDS, a block
// to a thread, while its first items are on their way: a launch less.
//
// Bound: HBM (the items' bytes): one user over 5M items (k = 64, 170 MB and 20 MB of
// scores) takes 36 us when the items come from HBM, 27.5 from the Infinity Cache (read
// around the caches 34 and 33).  A tile at a time, eight waves on a SIMD: several
// tiles' loads in one wave, with fewer waves, were slower or alike (5M items: one tile
// 27.5 us, four 29.9, eight 28.9; 1M of k = 128 12.1 and 14.5 with four).
constexpr int kOwnBlocks = 16;
template <class O, class X, int STEPS, bool LONG, bool STREAM>
__global__ void __launch_bounds__(kThreads, 4) k_mx_few(Product P) {
  constexpr bool OWN = !std::is_same<X, uint8_t>::value;
  __shared__ i32x4 own_bytes[OWN ? 32 * kOwnBlocks : 1];
  __shared__ uint8_t own_scales[OWN ? 32 * kOwnBlocks : 1];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int l32 = lane % 32, half = lane / 32;
  const int64_t r0 = (int64_t)blockIdx.y * 32, tiles = (P.items + 31) / 32;
  const int rows = P.rows - r0 < 32 ? (int)(P.rows - r0) : 32;
  const int row = l32 < rows ? l32 : rows - 1;
  const uint8_t *a = P.a + (r0 + row) * P.a_stride, *as = P.a_scale + (r0 + row) * P.as_stride;
  int64_t tile = (int64_t)blockIdx.x * kWaves + wave;
  const int64_t stride = (int64_t)gridDim.x * kWaves;
  i32x4 x[STEPS], y[STEPS];
  int xs[STEPS], ys[STEPS];
  const auto users = [&](int32_t s0) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int32_t at = (s0 + s) * 2 + half;
      y[s] = i32x4{}, ys[s] = 0;
      if (at < P.blocks) {
        if constexpr (OWN) {
          y[s] = own_bytes[row * P.blocks + at], ys[s] = own_scales[row * P.blocks + at];
        } else {
          y[s] = block_bytes(a + (int64_t)at * 16), ys[s] = as[at];
        }
      }
    }
  };
  const auto items = [&](int64_t t, int32_t s0) {
    int64_t j = t * 32 + l32;
    if (j >= P.items) j = P.items - 1;
    const uint8_t *b = P.b + j * P.b_stride, *bs = P.b_scale + j * P.bs_stride;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int32_t at = (s0 + s) * 2 + half;
      x[s] = i32x4{}, xs[s] = 0;
      if (at < P.blocks) x[s] = block_bytes<STREAM>(b + (int64_t)at * 16), xs[s] = bs[at];
    }
  };
  if (tile < tiles) items(tile, 0);
  if constexpr (OWN) {
    for (int i = threadIdx.x; i < rows * P.blocks; i += kThreads) {
      const X *v = static_cast<const X *>(P.x) + (r0 + i / P.blocks) * P.x_stride;
      float eight[4][8];
      uint32_t most = 0, bits[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        load_eight(v, i % P.blocks * kBlock + q * 8, P.k, eight[q]);
        most = max(most, largest_bits(eight[q]));
      }
      const int code = scale_byte(most);
#pragma unroll
      for (int q = 0; q < 4; ++q) bits[q] = eight_to_bits(eight[q], code);
      own_bytes[i] = i32x4{(int)bits[0], (int)bits[1], (int)bits[2], (int)bits[3]};
      own_scales[i] = (uint8_t)code;
    }
    __syncthreads();
  }
  if constexpr (!LONG) users(0);
  for (; tile < tiles; tile += stride) {
    f32x16 acc = {};
    for (int32_t s0 = 0;;) {
      if constexpr (LONG) users(s0);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) acc = multiply<0>(y[s], ys[s], x[s], xs[s], acc);
      if constexpr (LONG) {
        s0 += STEPS;
        if (s0 * 2 < P.blocks) {
          items(tile, s0);
          continue;
        }
      }
      break;
    }
    if (tile + stride < tiles) items(tile + stride, 0);
    const int64_t j = tile * 32 + l32;
    if (j >= P.items) continue;
    O *to = static_cast<O *>(P.out) + ((r0 + 4 * half) * P.out_stride + j);
#pragma unroll
    for (int g = 0; g < 16; ++g) {
      const int u = 8 * (g / 4) + g % 4;
      if (u >= rows) break;  // of the whole wave
      if (u + 4 * half < rows) *to = from_float<O>(acc[g]);
      to += g % 4 == 3 ? 5 * P.out_stride : P.out_stride;
      asm volatile("" : "+v"(to));  // (16 addresses would be kept)
    }
  }
}

// Many users: a workgroup of 2 x 2 waves takes tiles of 64 BI items x 64 BU
// users, each wave a quarter of it in BI x BU blocks of 32 x 32.  STEP bytes of
// a row (STEP / 16 blocks) at a time pass through LDS, in chunks of a block
// whose place in a row is swizzled so that 16 lanes that read 16 rows meet all
// 64 banks, and the row's scales as two words: those of its even blocks, then
// those of its odd ones.
constexpr int64_t kUserPad = 256;
constexpr int64_t kMostStride = 1 << 23;  // bytes from an item to the next (128 rows: 2^30)

template <class O, int BI, int BU, int STEP>
struct Many {
  static constexpr int kItems = 64 * BI, kUsers = 64 * BU, kChunks = STEP / 16;
  static constexpr int kSubs = kChunks / 2;  // pairs of blocks of a step
  static constexpr int kPass = kThreads / kChunks;  // rows that the workgroup loads at a time
  // of a thread (where a pass has more rows than there are, some threads' none)
  static constexpr int kItemLoads = (kItems + kPass - 1) / kPass;
  static constexpr int kUserLoads = (kUsers + kPass - 1) / kPass;
  static constexpr int kBuffer = (kItems + kUsers) * kChunks;  // i32x4 of a step
  static constexpr int kScaleLoads = (kItems + kUsers + kThreads - 1) / kThreads;
  static constexpr int kScaleWords = kScaleLoads * kThreads * 2;  // of a step
  static constexpr int kPitch = 32 * BI + 16 / (int)sizeof(O);  // of the scores on their way out
  static constexpr int kScores = kWaves * 32 * kPitch * (int)sizeof(O) / 16;  // i32x4

  static __device__ __forceinline__ int at(int row, int c) {
    if constexpr (kChunks == 2) return row * 2 + c;
    else if constexpr (kChunks == 4) return row * 4 + (c ^ ((row >> 2) & 3));
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

  // PAD (rows of at least kChunks blocks): without branches; the users' rows have
  // blocks of zeros up to a multiple of kChunks, and in place of an item's blocks
  // past its row come its last one with scales of 0, so that their products are 0.
  // Block q of a thread's blocks of a step (the items', then the users'), with PAD:
  static __device__ __forceinline__ i32x4 load_one(const Product &P, int64_t j0, int64_t r0, int s,
                                                   int q) {
    const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
    if (q < kItemLoads) {
      const int32_t c = min(s * kChunks + chunk, P.blocks - 1);
      const uint32_t at = (uint32_t)row * (uint32_t)P.b_stride + (uint32_t)c * 16;
      return block_bytes(P.b + (j0 + q * kPass) * P.b_stride + at);
    }
    const uint32_t at = (uint32_t)row * (uint32_t)P.a_stride + chunk * 16;
    const uint8_t *a = P.a + (r0 + (q - kItemLoads) * kPass) * P.a_stride + (int64_t)s * STEP;
    return block_bytes(a + at);
  }
  static __device__ __forceinline__ void store_one(i32x4 *buffer, int q, i32x4 x) {
    const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
    if (q < kItemLoads) buffer[at(row + kPass * q, chunk)] = x;
    else buffer[kItems * kChunks + at(row + kPass * (q - kItemLoads), chunk)] = x;
  }

  // A thread's blocks of step s of the items from j0 on (kItems of them are
  // there) and of the users from r0 on (kUsers rows are, as they are laid out up to
  // a multiple of kUserPad; none behind them need be).  A thread's offset within its
  // first row is 32 bits wide (see kMostStride).
  static __device__ __forceinline__ void load(const Product &P, int64_t j0, int64_t r0, int s,
                                              i32x4 (&x)[kItemLoads], i32x4 (&y)[kUserLoads]) {
    const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
    const bool some = s * kChunks + chunk < P.blocks;
    const uint32_t at_item = (uint32_t)row * (uint32_t)P.b_stride + chunk * 16;
    const uint32_t at_user = (uint32_t)row * (uint32_t)P.a_stride + chunk * 16;
    const uint8_t *b = P.b + (j0 * P.b_stride + (int64_t)s * STEP);
    const uint8_t *a = P.a + (r0 * P.a_stride + (int64_t)s * STEP);
#pragma unroll
    for (int h = 0; h < kItemLoads; ++h) {
      x[h] = i32x4{};
      if (some && (kPass <= kItems || row < kItems))
        x[h] = block_bytes(b + h * kPass * P.b_stride + at_item);
    }
#pragma unroll
    for (int h = 0; h < kUserLoads; ++h) {
      y[h] = i32x4{};
      if (some && (kPass <= kUsers || row < kUsers))
        y[h] = block_bytes(a + h * kPass * P.a_stride + at_user);
    }
  }
  static __device__ __forceinline__ void store(i32x4 *buffer, const i32x4 (&x)[kItemLoads],
                                               const i32x4 (&y)[kUserLoads]) {
    const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
#pragma unroll
    for (int h = 0; h < kItemLoads; ++h)
      if (kPass <= kItems || row < kItems) buffer[at(row + kPass * h, chunk)] = x[h];
#pragma unroll
    for (int h = 0; h < kUserLoads; ++h)
      if (kPass <= kUsers || row < kUsers)
        buffer[kItems * kChunks + at(row + kPass * h, chunk)] = y[h];
  }
  // The scales of a thread's rows (items, then users) in step s, as they are.
  struct Scales {
    uint32_t w[kScaleLoads][2];
  };
  template <bool PAD = false>
  static __device__ __forceinline__ void load_scales(const Product &P, int64_t j0, int64_t r0,
                                                     int s, Scales &scale) {
    const int32_t c = s * kChunks;
#pragma unroll
    for (int h = 0; h < kScaleLoads; ++h) {
      const int i = threadIdx.x + h * kThreads;
      scale.w[h][0] = scale.w[h][1] = 0;
      if (kScaleLoads * kThreads > kItems + kUsers && i >= kItems + kUsers) continue;
      const bool item = kItems % kThreads == 0 ? h * kThreads < kItems : i < kItems;
      const uint8_t *p = item ? P.b_scale + (j0 + i) * P.bs_stride
                              : P.a_scale + (r0 + i - kItems) * P.as_stride;
      if constexpr (PAD) {
        const int32_t from = min(c, P.blocks - kChunks), past = c - from;  // below 8
        uint64_t w;
        __builtin_memcpy(&w, p + from, 8);
        w >>= past * 8;
        scale.w[h][0] = (uint32_t)w, scale.w[h][1] = (uint32_t)(w >> 32);
        continue;
      }
      p += c;
      if (c + kChunks <= P.blocks) {
        __builtin_memcpy(scale.w[h], p, kChunks);
      } else {
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
          if (c + k < P.blocks) scale.w[h][k / 4] |= (uint32_t)p[k] << (k % 4 * 8);
      }
    }
  }
  static __device__ __forceinline__ void store_scales(uint32_t *words, const Scales &scale) {
#pragma unroll
    for (int h = 0; h < kScaleLoads; ++h) {
      const uint2 w = {__builtin_amdgcn_perm(scale.w[h][1], scale.w[h][0], 0x06040200u),
                       __builtin_amdgcn_perm(scale.w[h][1], scale.w[h][0], 0x07050301u)};
      *reinterpret_cast<uint2 *>(words + (threadIdx.x + h * kThreads) * 2) = w;
    }
  }
  // A wave's bytes of a pair of blocks, and its scales of a step.
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
  static __device__ __forceinline__ void read_scales(const uint32_t *words, int (&si)[BI],
                                                     int (&su)[BU]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
    for (int h = 0; h < BI; ++h)
      si[h] = (int)words[((wave % 2 * BI + h) * 32 + lane % 32) * 2 + lane / 32];
#pragma unroll
    for (int h = 0; h < BU; ++h)
      su[h] = (int)words[(kItems + (wave / 2 * BU + h) * 32 + lane % 32) * 2 + lane / 32];
  }
  template <int SUB>
  static __device__ __forceinline__ void products(f32x16 (&acc)[BI][BU], const i32x4 (&fi)[BI],
                                                  const i32x4 (&fu)[BU], const int (&si)[BI],
                                                  const int (&su)[BU]) {
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int u = 0; u < BU; ++u)
        acc[i][u] = multiply<SUB>(fi[i], si[i], fu[u], su[u], acc[i][u]);
  }

  // Register g of a lane is the sum of item 8 (g / 4) + 4 (l / 32) + g % 4 and
  // user l % 32.  The scores of 32 users at a time pass through LDS (lds: the
  // whole workgroup's), so that a user's 32 BI scores are stored in a row.
  static __device__ __forceinline__ void store_scores(const Product &P, int64_t j0, int64_t r0,
                                                      const f32x16 (&acc)[BI][BU], i32x4 *lds) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wi = wave % 2, wu = wave / 2, l32 = lane % 32, half = lane / 32;
    O *mine = reinterpret_cast<O *>(lds) + wave * (32 * kPitch);
    constexpr int N = Vec<O>::N, kLanes = 32 * BI / N;  // lanes of a user's row
#pragma unroll
    for (int u = 0; u < BU; ++u) {
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int ji = i * 32 + g * 8 + half * 4;
          O v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = from_float<O>(acc[i][u][g * 4 + e]);
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

// Tiles of 128 or 64 items x 128 or 64 users: three or four workgroups on a CU
// overlap their loads, products and stores.  A workgroup's bytes of the next
// step, or of its next tile, are on their way into registers meanwhile.  Bound:
// HBM (the scores) up to k of some hundred: 2,048 users x 18,000 items, k = 64, to bf16
// takes 15.7 us, 4.7 TB/s.
template <class O, int BI, int BU, int STEP>
__global__ void __launch_bounds__(kThreads, BI * BU == 4 ? 3 : 4)
    k_mx_many(Product P, int64_t tiles) {
  using M = Many<O, BI, BU, STEP>;
  __shared__ i32x4 lds[M::kBuffer > M::kScores ? M::kBuffer : M::kScores];
  __shared__ uint32_t s_scale[M::kScaleWords];
  const int steps = (P.blocks + M::kChunks - 1) / M::kChunks;
  i32x4 x[M::kItemLoads], y[M::kUserLoads];
  typename M::Scales scale;
  const auto load = [&](int64_t j0, int64_t r0, int s) {
    M::load(P, j0, r0, s, x, y);
    M::load_scales(P, j0, r0, s, scale);
  };
  f32x16 acc[BI][BU] = {};
  int64_t tile = blockIdx.x, j0, r0;
  M::place(P, tile, j0, r0);
  load(j0, r0, 0);
  for (int s = 0; tile < tiles;) {
    __syncthreads();
    M::store(lds, x, y);
    M::store_scales(s_scale, scale);
    __syncthreads();
    const bool last = s + 1 == steps;
    int64_t jn = j0, rn = r0;
    const int64_t next = last ? tile + gridDim.x : tile;
    if (next < tiles) {
      if (last) M::place(P, next, jn, rn);
      load(jn, rn, last ? 0 : s + 1);
    }
    int si[BI], su[BU];
    M::read_scales(s_scale, si, su);
    i32x4 fi[BI], fu[BU];
    M::read(lds, 0, fi, fu);
    M::template products<0>(acc, fi, fu, si, su);
    if constexpr (M::kSubs > 1) {
      M::read(lds, 1, fi, fu);
      M::template products<1>(acc, fi, fu, si, su);
    }
    ++s;
    if (last) {
      __syncthreads();
      M::store_scores(P, j0, r0, acc, lds);
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int u = 0; u < BU; ++u) acc[i][u] = f32x16{};
      tile = next, j0 = jn, r0 = rn, s = 0;
    }
  }
}

// Kinds of instructions that the scheduler is told to place.
constexpr int kMfma = 0x8, kVmemRead = 0x20, kDsRead = 0x100, kDsWrite = 0x200;

// Long rows: tiles of 256 x 256, eight blocks at a time, which halves the LDS
// traffic per product.  One workgroup fills a CU, so a wave itself reads its
// next pair of blocks from LDS while the matrix unit works, and a step's bytes
// are loaded a whole step before they go to the other LDS buffer.  Bound: the
// instructions' issue and the clock: 4,096 x 8,192 x 4,096 to bf16 takes 81 to 85 us,
// 3.3e15 operations a second (matrix instructions alone reach 5.2e15 to 6.2e15 on this
// card, on values that are not all alike); the matrix units work 45% of the cycles, and
// some 15 us go into the first loads and the stores of the two tiles that each CU has.
template <class O>
__global__ void __launch_bounds__(kThreads, 1) k_mx_large(Product P) {
  using M = Many<O, 4, 4, 128>;
  constexpr int kLoads = M::kItemLoads + M::kUserLoads;
  __shared__ i32x4 lds[2 * M::kBuffer > M::kScores ? 2 * M::kBuffer : M::kScores];
  __shared__ uint32_t s_scale[2][M::kScaleWords];
  const int steps = (P.blocks + 7) / 8;
  int64_t j0, r0;
  M::place(P, blockIdx.x, j0, r0);
  i32x4 x[kLoads];
  typename M::Scales scale;
#pragma unroll
  for (int q = 0; q < kLoads; ++q) x[q] = M::load_one(P, j0, r0, 0, q);
  M::template load_scales<true>(P, j0, r0, 0, scale);
#pragma unroll
  for (int q = 0; q < kLoads; ++q) M::store_one(lds, q, x[q]);
  M::store_scales(s_scale[0], scale);
  // past the last step: it once more, for nothing
#pragma unroll
  for (int q = 0; q < kLoads; ++q) x[q] = M::load_one(P, j0, r0, min(1, steps - 1), q);
  M::template load_scales<true>(P, j0, r0, min(1, steps - 1), scale);
  __syncthreads();
  f32x16 acc[4][4] = {};
  i32x4 fi[2][4], fu[2][4];
  int si[4], su[4], si_next[4], su_next[4];
  M::read_scales(s_scale[0], si, su);
  M::read(lds, 0, fi[0], fu[0]);
  // A step has four pairs of blocks, 16 products each.  During the products of the
  // first three the next pair is read, a third of the next step is written to the
  // other buffer, and the same third of the step after it is fetched; the last
  // one's cover the next step's first reads.
  // keeps products among the reads and writes that they are to cover (they have no
  // order of their own)
  const auto hold = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) asm volatile("" : "+a"(acc[i][u]));
  };
  for (int s = 0; s < steps; ++s) {
    i32x4 *now = lds + s % 2 * M::kBuffer, *other = lds + (s + 1) % 2 * M::kBuffer;
    const int ahead = min(s + 2, steps - 1);
    const auto third = [&](auto part) {
      constexpr int R = decltype(part)::value, kFrom = (kLoads * R + 2) / 3,
                    kTo = (kLoads * (R + 1) + 2) / 3;
      __builtin_amdgcn_sched_barrier(0);
      M::read(now, R + 1, fi[(R + 1) % 2], fu[(R + 1) % 2]);
#pragma unroll
      for (int q = kFrom; q < kTo; ++q) {
        M::store_one(other, q, x[q]);
        x[q] = M::load_one(P, j0, r0, ahead, q);
      }
      if constexpr (R == 2) {
        M::store_scales(s_scale[(s + 1) % 2], scale);
        M::template load_scales<true>(P, j0, r0, ahead, scale);
      }
      M::template products<R>(acc, fi[R % 2], fu[R % 2], si, su);
      hold();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        if (i < kTo - kFrom) __builtin_amdgcn_sched_group_barrier(kDsWrite, 1, 0);
        if (i < kTo - kFrom) __builtin_amdgcn_sched_group_barrier(kVmemRead, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      }
    };
    third(std::integral_constant<int, 0>{});
    third(std::integral_constant<int, 1>{});
    third(std::integral_constant<int, 2>{});
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    M::read_scales(s_scale[(s + 1) % 2], si_next, su_next);
    M::read(other, 0, fi[0], fu[0]);
    M::template products<3>(acc, fi[1], fu[1], si, su);
    hold();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < 4; ++h) si[h] = si_next[h], su[h] = su_next[h];
  }
  __syncthreads();
  M::store_scores(P, j0, r0, acc, lds);
}

// Workgroups that fill the GPU: eight of four waves on each of 256 CUs.
constexpr int64_t kFullGpu = 2048;
// Bytes of items that stay in the Infinity Cache between calls; more are read past the
// caches.  One user, k = 64, through and past them: 7M items (213 MB) 41.7 and 46.6 us,
// 8M 49.3 and 52.6, 10M 72.4 and 64.0, 20M 146 and 127.
constexpr int64_t kCached = 256 << 20;

template <class O, class X, int STEPS, bool LONG>
void launch_few(Product p, hipStream_t stream) {
  const int64_t all = (p.items + 32 * kWaves - 1) / (32 * kWaves);
  // equally many tiles for each
  const int64_t rounds = (all + kFullGpu - 1) / kFullGpu, groups = (all + rounds - 1) / rounds;
  const bool stream_items = p.rows <= 32 && p.items * (int64_t)p.blocks * 16 > kCached;
  constexpr int64_t kMost = 65535ll * 32;  // users of a launch
  for (int64_t left = p.rows; left > 0; left -= kMost) {
    p.rows = std::min(left, kMost);
    const dim3 grid((unsigned)groups, (unsigned)((p.rows + 31) / 32));
    if (stream_items)
      hipLaunchKernelGGL((k_mx_few<O, X, STEPS, LONG, true>), grid, dim3(kThreads), 0,
                         stream, p);
    else
      hipLaunchKernelGGL((k_mx_few<O, X, STEPS, LONG, false>), grid, dim3(kThreads), 0,
                         stream, p);
    if (p.x) p.x = static_cast<const X *>(p.x) + kMost * p.x_stride;
    p.a += kMost * p.a_stride, p.a_scale += kMost * p.as_stride;
    p.out = static_cast<O *>(p.out) + kMost * p.out_stride;
  }
}

template <class O, class X>
void product_few(const Product &p, hipStream_t stream) {
  if (p.blocks <= 2) launch_few<O, X, 1, false>(p, stream);
  else if (p.blocks <= 4) launch_few<O, X, 2, false>(p, stream);
  else if (p.blocks <= 8) launch_few<O, X, 4, false>(p, stream);
  else launch_few<O, X, 4, true>(p, stream);
}

template <class O, int BI, int BU, int STEP>
void launch_many(const Product &p, hipStream_t stream) {
  const int64_t all =
      (p.items + 64 * BI - 1) / (64 * BI) * ((p.rows + 64 * BU - 1) / (64 * BU));
  constexpr int64_t kAtOnce = 256 * (BI * BU == 4 ? 3 : 4);
  hipLaunchKernelGGL((k_mx_many<O, BI, BU, STEP>), dim3((unsigned)std::min(all, kAtOnce)),
                     dim3(kThreads), 0, stream, p, all);
}

// Whether the product itself quantises the users' values (few users, or so few
// scores that the other kernels' launch for it costs more): fp32, k = 64, own and
// in the faster of the other kernels, 18,000 items 48 users 4.4 and 5.7 us, 64 5.0
// and 5.7, 128 6.3 and 6.1, 100,003 items 48 users 8.8 and 8.7, 64 10.3 and 9.3; k =
// 200, 18,000 items 48 users 5.8 and 6.7, 128 8.7 and 8.2, 100,003 items 48 users
// 14.3 and 10.7.  Up to 32 users own and with a launch: k = 64 18,000 items 4.1 and
// 5.5 us, 1M 30.3 and 31.6; k = 512 18,000 items 8.4 and 8.3, 100,003 19.9 and 18.1,
// 1M 135 and 140.
inline bool takes_values(int64_t rows, int64_t items, int64_t blocks) {
  return rows <= 32 ? blocks <= kOwnBlocks : blocks <= 8 && rows * items <= (1 << 22) / blocks;
}
inline bool uses_few(int64_t rows, int64_t items, int64_t items_stride) {
  return rows <= 32 || items < 128 || items_stride > kMostStride;
}
// Tiles of 256 x 256 for rows of at least this many blocks and at least 128 tiles.
// Against 128 x 128, to bf16: 4,096 x 8,192 (512 tiles), k = 512 24 and 19 us, 1,024
// 29 and 30, 2,048 42 and 56, 4,096 71 and 129; 2,048 x 18,000 (568), k = 1,024 39
// and 34, 2,048 58 and 63; 512 x 18,000 (142), k = 1,024 14.7 and 13.8, 2,048 20.8 and
// 22.2; 2,048 x 4,096 (128), k = 2,048 19.9 and 18.1, 4,096 35.2 and 36.6 (all with
// bytes of one value, which the GPU multiplies at a higher clock).
constexpr int64_t kLargeBlocks = 64;

template <class O>
hipError_t product(const Product &p, int32_t type, hipStream_t stream) {
  const auto tiles = [&](int64_t items, int64_t users) {
    return (p.items + items - 1) / items * ((p.rows + users - 1) / users);
  };
  if (p.x || uses_few(p.rows, p.items, p.b_stride)) {
    if (!p.x) product_few<O, uint8_t>(p, stream);
    else if (type == BGMF_TYPE_F32) product_few<O, float>(p, stream);
    else if (type == BGMF_TYPE_BF16) product_few<O, bf16_t>(p, stream);
    else product_few<O, f16_t>(p, stream);
  } else if (p.blocks >= kLargeBlocks && p.items >= 256 && tiles(256, 256) >= 128) {
    hipLaunchKernelGGL(k_mx_large<O>, dim3((unsigned)tiles(256, 256)), dim3(kThreads), 0, stream,
                       p);
    // otherwise the largest tiles of which every CU gets one.  To bf16 by 64 x 64, 128 x
    // 64 and 128 x 128: 2,048 x 18,000, k = 64 19.0, 14.3 and 13.4 us, k = 512 39.8, 26.8
    // and 22.0; 128 x 18,000, k = 64 3.7, 3.8 and 3.9, k = 512 5.7, 5.6 and 5.8; 256 x 4,096,
    // k = 512 4.3, 4.7 and 5.5; 64 x 100,003, k = 64 6.5, 5.6 and 6.6
  } else if (p.rows > 64 && tiles(128, 128) >= 256) {
    if (p.blocks <= 2) launch_many<O, 2, 2, 32>(p, stream);
    else launch_many<O, 2, 2, 64>(p, stream);
  } else if (tiles(128, 64) >= 256) {
    if (p.blocks <= 2) launch_many<O, 2, 1, 32>(p, stream);
    else launch_many<O, 2, 1, 64>(p, stream);
  } else {
    if (p.blocks <= 2) launch_many<O, 1, 1, 32>(p, stream);
    else launch_many<O, 1, 1, 64>(p, stream);
  }
  return hipGetLastError();
}

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline int64_t blocks_of(int64_t k) { return (k + kBlock - 1) / kBlock; }
constexpr int64_t kMostK = (1 << 20) - 1;  // of a product

// Workspace: the users' bytes up to a multiple of kUserPad rows (and of eight
// blocks, the last ones 0, where k_mx_large may read them), then their scales.
int64_t padded_rows(int64_t rows) { return rows > 32 ? round_up(rows, kUserPad) : rows; }
int64_t padded_blocks(int64_t rows, int64_t k) {
  const int64_t blocks = blocks_of(k);
  return rows > 32 && blocks >= kLargeBlocks ? round_up(blocks, 8) : blocks;
}
int64_t bytes_part(int64_t rows, int64_t k) {
  return round_up(padded_rows(rows) * padded_blocks(rows, k) * 16, 256);
}

// Rows given in 4 bits, into the workspace's layout.
__global__ void __launch_bounds__(kThreads) k_copy_mx(Product P, uint8_t *q, uint8_t *scale,
                                                      int32_t padded) {
  const int64_t all = P.rows * padded;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all;
       i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / padded, c = i % padded;
    i32x4 x = {};
    uint8_t s = 0;
    if (c < P.blocks)
      x = block_bytes(P.a + r * P.a_stride + c * 16), s = P.a_scale[r * P.as_stride + c];
    *reinterpret_cast<i32x4 *>(q + i * 16) = x;
    scale[i] = s;
  }
}

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
      (type == BGMF_TYPE_MX4 && (rows <= 32 || item_count < 128)))
    return 0;
  return bytes_part(rows, k) + round_up(padded_rows(rows) * padded_blocks(rows, k), 256);
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
  Product p{nullptr, row_stride, (int32_t)k, static_cast<const uint8_t *>(x), row_scale, rows,
            row_stride, row_scale_stride, items, item_scale, item_count, items_stride,
            item_scale_stride, (int32_t)blocks, out, out_stride};
  hipError_t e = hipSuccess;
  if (own && takes_values(rows, item_count, blocks)) {
    p.x = x, p.a = nullptr;
  } else if (own || !uses_few(rows, item_count, items_stride)) {
    uint8_t *q = static_cast<uint8_t *>(ws), *scale = q + bytes_part(rows, k);
    const int64_t laid = padded_blocks(rows, k);
    if (own) {
      e = quantize_mx(type, Rows{x, rows, row_stride, (int32_t)k, (int32_t)(laid * 4), q, scale,
                                 laid * 16, laid}, stream);
    } else {
      const int64_t groups = std::min<int64_t>((rows * laid + kThreads - 1) / kThreads, 4096);
      hipLaunchKernelGGL(k_copy_mx, dim3((unsigned)groups), dim3(kThreads), 0, stream, p, q, scale,
                         (int32_t)laid);
      e = hipGetLastError();
    }
    p.a = q, p.a_scale = scale, p.a_stride = laid * 16, p.as_stride = laid;
  }
  if (e == hipSuccess)
    e = out_type == BGMF_TYPE_F32    ? product<float>(p, type, stream)
        : out_type == BGMF_TYPE_BF16 ? product<bf16_t>(p, type, stream)
                                     : product<f16_t>(p, type, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
