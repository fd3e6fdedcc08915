// Log probabilities of given items with entropy and top alternatives
// (bgmf_log_probs), and their gradient (bgmf_log_probs_grad).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

// Threads of a workgroup: 256, or one wave for short rows (TH below).
constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f;
constexpr double kLn2 = 0.69314718055994530942;

// Reductions over a wave in registers (DPP): four steps within rows of 16
// lanes, two between rows, the total in lane 63.  A lane without a source adds
// `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t dpp(int32_t none, int32_t x) {
  return __builtin_amdgcn_update_dpp(none, x, CTRL, ROWS, 0xF, false);
}
template <class F>
__device__ __forceinline__ int32_t wave_reduce(int32_t v, int32_t none, const F &f) {
  v = f(v, dpp<0x111, 0xF>(none, v));
  v = f(v, dpp<0x112, 0xF>(none, v));
  v = f(v, dpp<0x114, 0xF>(none, v));
  v = f(v, dpp<0x118, 0xF>(none, v));
  v = f(v, dpp<0x142, 0xA>(none, v));
  v = f(v, dpp<0x143, 0xC>(none, v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float wave_max(float v) {
  return __int_as_float(wave_reduce(__float_as_int(v), __float_as_int(-INFINITY),
                                    [](int32_t a, int32_t b) {
                                      return __float_as_int(
                                          fmaxf(__int_as_float(a), __int_as_float(b)));
                                    }));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double v) {
  const int32_t lo = dpp<CTRL, ROWS>(0, __double2loint(v)), hi = dpp<CTRL, ROWS>(0, __double2hiint(v));
  return v + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_sum(double v) {
  v = dpp_add<0x111, 0xF>(v);
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);
  v = dpp_add<0x143, 0xC>(v);
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63),
                          __builtin_amdgcn_readlane(__double2loint(v), 63));
}

// A row, or a part of one, in 16-byte vectors and up to N - 1 single elements
// at its end.
template <class T, bool EX>
struct Row {
  static constexpr int N = Vec<T>::N;
  const T *x;
  const uint8_t *ex;  // with EX
  int32_t len;
  __device__ __forceinline__ int32_t vecs() const { return len / N; }
  __device__ __forceinline__ float one(int32_t i) const {  // -inf where excluded
    if constexpr (EX)
      if (ex[i]) return -INFINITY;
    return to_float(x[i]);
  }
  // A vector as it is in memory, and its scores: several are fetched before the
  // first is looked at.
  struct Raw {
    Vec<T> a;
    uint32_t b[EX ? N / 4 : 1];
  };
  __device__ __forceinline__ Raw fetch(int32_t v) const {
    Raw r;
    r.a = load_vec(x + (int64_t)v * N);
    if constexpr (EX) __builtin_memcpy(r.b, ex + (int64_t)v * N, N);
    return r;
  }
  static __device__ __forceinline__ Raw nothing() {  // scores of -inf
    Raw r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.a.v[i] = from_float<T>(-INFINITY);
    if constexpr (EX)
      for (int i = 0; i < N / 4; ++i) r.b[i] = 0;
    return r;
  }
  static __device__ __forceinline__ void scores(const Raw &r, float (&out)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      out[i] = to_float(r.a.v[i]);
      if constexpr (EX) out[i] = r.b[i / 4] >> (i % 4 * 8) & 0xFF ? -INFINITY : out[i];
    }
  }
};

// Running maximum m, s = sum exp2(d) and w = sum exp2(d) d, d = (x - m) c, of
// the scores seen so far.  A group's terms are summed in fp32 and added to
// running sums in fp64 (rows of many equal scores lose a unit per addition in
// fp32).  A score of -inf adds nothing; a NaN or +inf makes s NaN.
struct Soft {
  float m = -INFINITY;
  double s = 0.0, w = 0.0;
  // to the maximum M >= m
  __device__ __forceinline__ void rescale(float M, float c) {
    if (m == -INFINITY) return;  // s and w are 0, or NaN from a NaN
    const float d = fmaxf((m - M) * c, -1e30f), f = __builtin_amdgcn_exp2f((m - M) * c);
    w = (w + s * d) * f;
    s *= f;
  }
  template <int COUNT>
  __device__ __forceinline__ void add(const float (&x)[COUNT], float gm, float c) {  // gm: max x
    if (gm > m) {
      rescale(gm, c);
      m = gm;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float gs = 0.0f, gw = 0.0f;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const float d = (x[i] - base) * c, e = __builtin_amdgcn_exp2f(d);
      gs += e;
      gw = fmaf(e, fmaxf(d, -200.0f), gw);  // 0 where d is -inf
    }
    s += gs;
    w += gw;
  }
};

// Sums over the workgroup in a fixed order; every thread has the result.
template <int TH>
struct SoftLds {
  float m[TH / 64];
  double s[TH / 64], w[TH / 64];
};
template <int TH>
__device__ __forceinline__ Soft block_soft(Soft a, float c, SoftLds<TH> &lds) {
  constexpr int W = TH / 64;
  const int wave = threadIdx.x / 64;
  Soft r;
  r.m = wave_max(a.m);
  if constexpr (W > 1) {
    if (threadIdx.x % 64 == 0) lds.m[wave] = r.m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) r.m = fmaxf(r.m, lds.m[i]);
  }
  a.rescale(r.m, c);
  a.s = wave_sum(a.s), a.w = wave_sum(a.w);
  if constexpr (W == 1) {
    r.s = a.s, r.w = a.w;
  } else {
    if (threadIdx.x % 64 == 0) lds.s[wave] = a.s, lds.w[wave] = a.w;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) r.s += lds.s[i], r.w += lds.w[i];
  }
  return r;
}

// ---------------------------------------------------------------------------
// The n best of the scores that a workgroup has just gone through, larger
// first, ties to the lower item.  A thread has kCols columns of the scores and
// kept the largest score of each.  The n-th largest of 256 maxima (of threads,
// or of columns where a workgroup is one wave) is a score that the n best are
// not below, and only columns with their maximum at or above it ("hot", a few
// more than n) can hold any of them: these are read once more, about n / 1024
// of the row and from the cache, and the scores at or above the bound, few more
// than n, are put in order by counting how many precede each.  If more
// than CAND qualify (equal scores, or the best ones all in few columns), the
// scores are gone through in order of items instead, merging each tile's
// candidates into a list.
//
// SRC: either SHARED, per_column() and piece(q, i, f): f(score, item) for
// each score of piece i of column q (the workgroup shares the hot columns'
// pieces), or not SHARED and column(q, bound, f): the same for scores of column
// q, all that are at or above the bound among them (by the column's thread);
// size() and at(p, item): all scores in the order of items.
// emit(rank, score, item), for every rank below n (item -1: none).
// ---------------------------------------------------------------------------
constexpr int kCols = 4;
constexpr int64_t kMostParts = kCols * kThreads;  // of a row, see split_of
template <int TH>
struct TopLds {
  static constexpr int CAND = TH == 64 ? 256 : 1024;
  float tm[TH == 64 ? 1 : TH];
  uint64_t k[CAND];
  uint64_t list[2][BGMF_TOP_MAX];
  uint16_t hot[kCols * TH];
  float bound;
  int hots, count;
};

// An order of floats as integers (no NaN).
__device__ __forceinline__ int32_t key_of(float x) {
  const int32_t b = __float_as_int(x + 0.0f);  // -0 becomes +0
  return b < 0 ? b ^ 0x7FFFFFFF : b;
}
__device__ __forceinline__ float of_key(int32_t k) {
  return __int_as_float(k < 0 ? k ^ 0x7FFFFFFF : k);
}
// A score and its item as one number, larger for what comes first.
__device__ __forceinline__ uint64_t rank_key(float v, int32_t j) {
  return (uint64_t)((uint32_t)key_of(v) ^ 0x80000000u) << 32 | (uint32_t)~j;
}
__device__ __forceinline__ float key_score(uint64_t k) {
  return of_key((int32_t)((uint32_t)(k >> 32) ^ 0x80000000u));
}
__device__ __forceinline__ int32_t key_item(uint64_t k) { return (int32_t)~(uint32_t)k; }

// By one wave: a score that at least n of 256 maxima (four in each lane) are
// not below, and few more than n; -inf if fewer than n are above -inf.
__device__ __forceinline__ float top_bound(const float (&tm)[4], int n) {
  const int32_t none = key_of(-INFINITY);
  int32_t k[4], lo = 0x7FFFFFFF, hi = none;
  int some = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    k[i] = key_of(tm[i]);
    if (k[i] > none) lo = min(lo, k[i]);
    hi = max(hi, k[i]);
    some += __popcll(__ballot(k[i] > none));
  }
  if (some < n) return -INFINITY;
  lo = wave_reduce(lo, 0x7FFFFFFF, [](int32_t a, int32_t b) { return min(a, b); });
  hi = wave_reduce(hi, none, [](int32_t a, int32_t b) { return max(a, b); });
  while (lo < hi) {  // at least n are at or above lo, fewer than n above hi
    const int32_t mid = (int32_t)((uint32_t)lo + ((uint32_t)hi - (uint32_t)lo + 1) / 2);
    int c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c += __popcll(__ballot(k[i] >= mid));
    if (c >= n) {
      lo = mid;
      if (c <= n + 2 + n / 8) break;
    } else {
      hi = mid - 1;
    }
  }
  return of_key(lo);
}

// How many of k[0..c) are larger, c at most CAND, zeros from c on; by G lanes
// for one number (all of them get the count).
template <int G>
__device__ __forceinline__ int count_larger(const uint64_t *k, int c, uint64_t mine) {
  int r = 0;
  for (int o = (int)(threadIdx.x % G) * 8; o < c; o += G * 8) {
    uint64_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = k[o + i];
#pragma unroll
    for (int i = 0; i < 8; ++i) r += x[i] > mine;
  }
#pragma unroll
  for (int o = 1; o < G; o *= 2) r += __shfl_xor(r, o);
  return r;
}

template <int TH, class SRC, class EMIT>
__device__ void top_in_order(const SRC &src, int n, TopLds<TH> &lds, float bound,
                             const EMIT &emit) {
  constexpr int CAND = TopLds<TH>::CAND;
  const int tid = threadIdx.x;
  int have = 0, now = 0;
  for (int64_t p0 = 0; p0 < src.size(); p0 += CAND) {
    if (tid == 0) lds.count = 0;
    __syncthreads();
    const uint64_t worst = have == n ? lds.list[now][n - 1] : 0;
#pragma unroll
    for (int q = 0; q < CAND / TH; ++q) {
      const int64_t p = p0 + q * TH + tid;
      if (p < src.size()) {
        int32_t j;
        const float v = src.at(p, j);
        if (v > -INFINITY && v >= bound) {
          const uint64_t k = rank_key(v, j);
          if (k > worst) lds.k[atomicAdd(&lds.count, 1)] = k;
        }
      }
    }
    __syncthreads();
    const int c = lds.count;
    if (c) {
      for (int i = tid; i < c + have; i += TH) {
        const uint64_t k = i >= c ? lds.list[now][i - c] : lds.k[i];
        int rank = 0;
        for (int o = 0; o < c; ++o) rank += lds.k[o] > k;
        for (int o = 0; o < have; ++o) rank += lds.list[now][o] > k;
        if (rank < n) lds.list[now ^ 1][rank] = k;
      }
      have = min(n, have + c);
      now ^= 1;
      __syncthreads();
    }
  }
  for (int i = tid; i < n; i += TH) {
    const uint64_t k = lds.list[now][i];
    if (i < have) emit(i, key_score(k), key_item(k));
    else emit(i, -INFINITY, -1);
  }
}

// Called by the whole workgroup; lds is free for other use after the next
// barrier.  tm: the maxima of the thread's columns.
template <int TH, class SRC, class EMIT>
__device__ __forceinline__ void top_select(const SRC &src, const float (&tm)[kCols], int n,
                                           TopLds<TH> &lds, const EMIT &emit) {
  constexpr int CAND = TopLds<TH>::CAND;
  const int tid = threadIdx.x;
  float most = tm[0];
#pragma unroll
  for (int q = 1; q < kCols; ++q) most = fmaxf(most, tm[q]);
#pragma unroll
  for (int q = 0; q < CAND / TH; ++q) lds.k[tid + q * TH] = 0;
  if (tid == 0) lds.hots = lds.count = 0;
  float bound;
  if constexpr (TH == 64) {
    bound = top_bound(tm, n);
    __syncthreads();
  } else {
    lds.tm[tid] = most;
    __syncthreads();
    if (tid < 64) {
      float four[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) four[i] = lds.tm[tid + 64 * i];
      bound = top_bound(four, n);
      if (tid == 0) lds.bound = bound;
    }
    __syncthreads();
    bound = lds.bound;
  }
  const auto candidate = [&](float v, int32_t j) {
    if (v > -INFINITY && v >= bound) {
      const int to = atomicAdd(&lds.count, 1);
      if (to < CAND) lds.k[to] = rank_key(v, j);
    }
  };
  if (most > -INFINITY && most >= bound) {
#pragma unroll
    for (int q = 0; q < kCols; ++q)
      if (tm[q] > -INFINITY && tm[q] >= bound) {
        if constexpr (SRC::SHARED) lds.hot[atomicAdd(&lds.hots, 1)] = (uint16_t)(tid + q * TH);
        else src.column(tid + q * TH, bound, candidate);
      }
  }
  __syncthreads();
  if constexpr (SRC::SHARED) {
    const uint32_t per = (uint32_t)src.per_column(), pieces = (uint32_t)lds.hots * per;
    for (uint32_t i = tid; i < pieces; i += TH) src.piece(lds.hot[i / per], i % per, candidate);
    __syncthreads();
  }
  const int c = lds.count;
  if (c > CAND) {
    __syncthreads();
    top_in_order<TH>(src, n, lds, bound, emit);
    return;
  }
  const auto order = [&](auto lanes) {
    constexpr int G = decltype(lanes)::value;
    for (int i = tid / G; i < c; i += TH / G) {
      const uint64_t k = lds.k[i];
      const int rank = count_larger<G>(lds.k, c, k);
      if (rank < n && tid % G == 0) emit(rank, key_score(k), key_item(k));
    }
  };
  if (c <= TH / 4) order(std::integral_constant<int, 4>{});
  else order(std::integral_constant<int, 1>{});
  for (int i = c + tid; i < n; i += TH) emit(i, -INFINITY, -1);
}

template <class T, bool EX, int TH>
struct RowSource {  // column q has vectors q, q + 4 TH, ..., and column q < TH tail element q
  static constexpr int N = Row<T, EX>::N;
  static constexpr bool SHARED = true;
  Row<T, EX> row;
  int32_t first;  // item of the row's first element
  __device__ __forceinline__ int32_t per_column() const {
    return (row.vecs() + kCols * TH - 1) / (kCols * TH) + 1;
  }
  template <class F>
  __device__ __forceinline__ void piece(int q, int32_t i, const F &f) const {
    const int32_t vecs = row.vecs();
    if (i == 0) {
      if (q < row.len - vecs * N) f(row.one(vecs * N + q), first + vecs * N + q);
      return;
    }
    const int32_t v = q + (i - 1) * (kCols * TH);
    if (v >= vecs) return;
    float x[N];
    row.scores(row.fetch(v), x);
#pragma unroll
    for (int e = 0; e < N; ++e) f(x[e], first + v * N + e);
  }
  __device__ __forceinline__ int64_t size() const { return row.len; }
  __device__ __forceinline__ float at(int64_t p, int32_t &j) const {
    j = first + (int32_t)p;
    return row.one((int32_t)p);
  }
};

struct LogProbs {
  const void *x;
  const uint8_t *ex;
  const int32_t *given;
  int64_t rows, cols, stride, ex_stride;
  float temperature;
  int32_t top;
  float *log_prob, *entropy, *row_max, *row_sum;
  int32_t *top_item;
  float *top_log_prob;
  // rows split in `parts` of part_len scores: where the parts' sums and tops go
  int64_t parts, part_len;
  struct PartSum *part_sum;  // [rows][parts]
  float *part_v;             // [rows][parts][top]
  int32_t *part_j;
};
struct PartSum {
  double s, w;
  float m;
};

template <class T>
__device__ __forceinline__ float given_score(const LogProbs &P, int64_t r, int64_t g) {
  if (P.ex && P.ex[r * P.ex_stride + g]) return -INFINITY;
  return to_float(static_cast<const T *>(P.x)[r * P.stride + g]);
}

// The row's results but for its tops, by one thread.
template <class T>
__device__ __forceinline__ void write_row(const LogProbs &P, int64_t r, const Soft &a, float log_s) {
  const float s = (float)a.s;
  if (P.row_max) P.row_max[r] = a.m;
  if (P.row_sum) P.row_sum[r] = s;
  if (P.entropy) P.entropy[r] = s == 0.0f ? 0.0f : log_s - (float)(a.w * kLn2 / a.s);
  if (P.log_prob) {
    const int64_t g = P.given[r];
    float lp = 0.0f;
    if (g < -1 || g >= P.cols) lp = NAN;
    else if (g >= 0)
      lp = s == 0.0f ? -INFINITY : (given_score<T>(P, r, g) - a.m) / P.temperature - log_s;
    P.log_prob[r] = lp;
  }
}

// One workgroup per row, or per part of a row.  Bound: HBM; the scores are
// read once.  A thread takes kGroup vectors at a time (64 bytes in flight),
// their maximum first, so that the running sums are rescaled once per group.
// 4,001 x 10,007 fp32 without alternatives takes 29 us, 5.5 TB/s.  A 16-bit type
// with exclusions is bound by the vector units: 1,999 x 18,000 bf16 takes 27 us
// without alternatives (they work 86% of the CUs' cycles, 19 instructions a
// score) and 31 with ten (80%, 22).  A group's vectors that a row does not have
// are computed all the same (18,000 scores are 2,250 vectors in three groups of
// 1,024).  Alternatives are chosen after a row's last score, and their registers
// (92 against 60) leave room for 1,280 workgroups at once in place of 2,048.
constexpr int kGroup = kCols;
template <class T, bool EX, bool TOP, int TH>
__global__ void __launch_bounds__(TH) k_log_probs(LogProbs P) {
  __shared__ SoftLds<TH> soft_lds;
  __shared__ typename std::conditional<TOP, TopLds<TH>, int>::type top_lds;
  constexpr int N = Vec<T>::N;
  const int tid = threadIdx.x;
  const float c = kLog2e / P.temperature;
  const int64_t units = P.rows * P.parts;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t r = P.parts == 1 ? u : u / P.parts, part = P.parts == 1 ? 0 : u % P.parts;
    const int64_t first = part * P.part_len;
    const int64_t left = P.cols - first;
    const Row<T, EX> row{static_cast<const T *>(P.x) + (r * P.stride + first),
                         EX ? P.ex + (r * P.ex_stride + first) : nullptr,
                         (int32_t)(left < P.part_len ? left : P.part_len)};
    Soft a;
    float tm[kCols];  // the largest score of the g-th vectors of all groups
#pragma unroll
    for (int g = 0; g < kCols; ++g) tm[g] = -INFINITY;
    const int32_t vecs = row.vecs();
    for (int32_t v0 = 0; v0 < vecs; v0 += TH * kGroup) {
      typename Row<T, EX>::Raw raw[kGroup];
      if (v0 + TH * kGroup <= vecs) {
#pragma unroll
        for (int g = 0; g < kGroup; ++g) raw[g] = row.fetch(v0 + g * TH + tid);
      } else {
#pragma unroll
        for (int g = 0; g < kGroup; ++g) {
          raw[g] = Row<T, EX>::nothing();
          if (v0 + g * TH + tid < vecs) raw[g] = row.fetch(v0 + g * TH + tid);
        }
      }
      constexpr int kOnce = 16 / N;  // vectors whose scores are in registers at a time
#pragma unroll
      for (int g0 = 0; g0 < kGroup; g0 += kOnce) {
        float x[kOnce][N], gm = -INFINITY;
#pragma unroll
        for (int g = 0; g < kOnce; ++g) {
          Row<T, EX>::scores(raw[g0 + g], x[g]);
          float vm = x[g][0];
#pragma unroll
          for (int i = 1; i < N; ++i) vm = fmaxf(vm, x[g][i]);
          if constexpr (TOP) tm[g0 + g] = fmaxf(tm[g0 + g], vm);
          gm = fmaxf(gm, vm);
        }
        a.add(reinterpret_cast<float(&)[kOnce * N]>(x), gm, c);
      }
    }
    if (tid < row.len - vecs * N) {
      const float x[1] = {row.one(vecs * N + tid)};
      tm[0] = fmaxf(tm[0], x[0]);
      a.add(x, x[0], c);
    }
    const Soft all = block_soft<TH>(a, c, soft_lds);
    const float log_s = logf((float)all.s);
    if (tid == 0) {
      if (P.parts == 1) write_row<T>(P, r, all, log_s);
      else P.part_sum[u] = PartSum{all.s, all.w, all.m};
    }
    if constexpr (TOP) {
      const int n = P.top;
      const RowSource<T, EX, TH> src{row, (int32_t)first};
      if (P.parts == 1)
        top_select<TH>(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
          P.top_item[r * n + rank] = j;
          P.top_log_prob[r * n + rank] = j < 0 ? v : (v - all.m) / P.temperature - log_s;
        });
      else
        top_select<TH>(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
          P.part_v[u * n + rank] = v;
          P.part_j[u * n + rank] = j;
        });
    }
    __syncthreads();  // before the next row uses LDS
  }
}

struct PartSource {  // column q has the list of part q, larger scores first
  static constexpr bool SHARED = false;
  const float *v;
  const int32_t *j;
  int64_t parts;
  int n;
  template <class F>
  __device__ __forceinline__ void column(int q, float bound, const F &f) const {
    const float *x = v + (int64_t)q * n;
    const int32_t *item = j + (int64_t)q * n;
    for (int i = 0; i < n; i += 4) {  // few lists have more at or above the bound
      float y[4];
      int32_t k[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        y[p] = i + p < n ? x[i + p] : -INFINITY;
        k[p] = i + p < n ? item[i + p] : -1;
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) f(y[p], k[p]);
      if (!(y[3] >= bound)) break;
    }
  }
  __device__ __forceinline__ int64_t size() const { return parts * n; }
  __device__ __forceinline__ float at(int64_t p, int32_t &item) const {
    item = j[p];
    return v[p];
  }
};

// Joins the parts of a row: one workgroup per row.  Bound: latency (eight rows
// of 153 parts with 50 alternatives each: 7 us).  A row with fewer parts than
// alternatives gets no bound from the parts' maxima, and all of its lists are
// put in order: one row of 625,001 (20 parts) takes 220 us with 100
// alternatives, one of 3.2M (98 parts) 319 us with 128, 15 and 18 with ten.
template <class T>
__global__ void __launch_bounds__(kThreads) k_log_probs_join(LogProbs P) {
  __shared__ SoftLds<kThreads> soft_lds;
  __shared__ TopLds<kThreads> top_lds;
  const int tid = threadIdx.x, n = P.top;
  const float c = kLog2e / P.temperature;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const PartSum *sums = P.part_sum + r * P.parts;
    Soft a;
    float tm[kCols];
    static_assert(kMostParts == kCols * kThreads, "a part is a column");
#pragma unroll
    for (int q = 0; q < kCols; ++q) {
      const int64_t i = tid + q * kThreads;
      Soft b;
      if (i < P.parts) b.m = sums[i].m, b.s = sums[i].s, b.w = sums[i].w;
      tm[q] = b.m;
      const float M = fmaxf(a.m, b.m);
      a.rescale(M, c);
      b.rescale(M, c);
      a.m = M, a.s += b.s, a.w += b.w;
    }
    const Soft all = block_soft<kThreads>(a, c, soft_lds);
    const float log_s = logf((float)all.s);
    if (tid == 0) write_row<T>(P, r, all, log_s);
    if (n) {
      const PartSource src{P.part_v + r * P.parts * n, P.part_j + r * P.parts * n, P.parts, n};
      top_select<kThreads>(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
        P.top_item[r * n + rank] = j;
        P.top_log_prob[r * n + rank] = j < 0 ? v : (v - all.m) / P.temperature - log_s;
      });
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient: every score is read and its gradient written once.  A workgroup
// takes a tile of one row at a time.  Bound: HBM: 4,096 x 18,000 fp32 take 104
// us, 5.7 TB/s.  16-bit types with exclusions take more registers: 8,192 x
// 18,000 bf16 150 us, 4.9 TB/s (127 of them, four waves a SIMD), f16 179 us (131,
// three waves; 154 and 127 with an entropy gradient).
// ---------------------------------------------------------------------------
struct LogProbsGrad {
  const void *x;
  const uint8_t *ex;
  const int32_t *given;
  int64_t rows, cols, stride, ex_stride, out_stride;
  float temperature;
  const float *row_max, *row_sum, *entropy, *g_log_prob, *g_entropy;
  void *out;
  int64_t tiles;  // of a row
};
constexpr int kGradGroup = 4;

template <class T, bool EX, bool ENT, int TH>
__global__ void __launch_bounds__(TH) k_log_probs_grad(LogProbsGrad P) {
  constexpr int N = Vec<T>::N;
  constexpr int64_t kGradTile = (int64_t)TH * kGradGroup * N;
  const int tid = threadIdx.x;
  const float c = kLog2e / P.temperature;
  for (int64_t u = blockIdx.x; u < P.rows * P.tiles; u += gridDim.x) {
    const int64_t r = u / P.tiles, first = u % P.tiles * kGradTile, left = P.cols - first;
    const int32_t len = (int32_t)(left < kGradTile ? left : kGradTile);
    const T *x = static_cast<const T *>(P.x) + (r * P.stride + first);
    const uint8_t *ex = EX ? P.ex + (r * P.ex_stride + first) : nullptr;
    T *out = static_cast<T *>(P.out) + (r * P.out_stride + first);
    const float m = P.row_max[r], s = P.row_sum[r];
    const int64_t g = P.given ? P.given[r] : -1;
    float gl = P.g_log_prob && g != -1 ? P.g_log_prob[r] / P.temperature : 0.0f;
    if (g < -1 || g >= P.cols) gl = NAN;
    const int64_t at_given = g - first;
    float gh = 0.0f, shift = 0.0f;
    if constexpr (ENT) {
      gh = P.g_entropy[r] / P.temperature;
      shift = P.entropy[r] - logf(s);
    }
    const bool none = s == 0.0f;
    const float inv = 1.0f / s;
    const auto grad = [&](float v, int32_t i, bool excluded) {
      const float d = (v - m) * c, p = __builtin_amdgcn_exp2f(d) * inv;
      float y = -gl * p;
      if constexpr (ENT) y -= gh * p * fmaf(fmaxf(d, -200.0f), (float)kLn2, shift);
      if (i == at_given) y += gl;
      return from_float<T>(excluded || none ? 0.0f : y);
    };
    Vec<T> a[kGradGroup];
    uint8_t b[kGradGroup][N];
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * TH) * N;
      if (i + N <= len) {
        a[q] = load_vec(x + i);
        if constexpr (EX) __builtin_memcpy(b[q], ex + i, N);
      }
    }
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * TH) * N;
      if (i + N <= len) {
        Vec<T> y;
#pragma unroll
        for (int e = 0; e < N; ++e) y.v[e] = grad(to_float(a[q].v[e]), i + e, EX && b[q][e]);
        store_vec(out + i, y);
      } else {
        for (int e = 0; e < N; ++e)
          if (i + e < len) out[i + e] = grad(to_float(x[i + e]), i + e, EX && ex[i + e]);
      }
    }
  }
}

constexpr int64_t kMostGroups = 1 << 20;

// How a row is split: in as few parts as hold at most 32,768 scores each, but
// no more than fill the GPU (eight workgroups for each of 256 CUs) or than 1024.
// Parts have to pay for the second launch.  One row, ten alternatives, in one,
// two and three parts: 18,000 scores 7.9, 12.7 and 12.2 us, 33,000 10.1, 13.7
// and 12.9, 65,000 13.6, 15.4 and 14.4, 80,000 16.0, 16.5 and 14.8; without
// alternatives 33,000 7.2, 8.1 and 7.2, 65,000 10.7, 9.8 and 8.6.  (Eight and 64
// rows are alike.)  So rows of up to 65,000 would be faster in one part with
// alternatives, and longer single rows in more than they get: 625,001 take 14.6
// us in 20 parts and 11.6 in 128, 5M 17.8 in 153 and 15.9 in 256.
constexpr int64_t kFullGpu = 2048, kPart = 32768;
struct Split {
  int64_t parts, len;
};
Split split_of(int64_t rows, int64_t cols) {
  int64_t parts = std::min({(cols + kPart - 1) / kPart,
                            std::max<int64_t>(kFullGpu / std::max<int64_t>(rows, 1), 1), kMostParts});
  if (parts <= 1) return {1, cols};
  const int64_t len = ((cols + parts - 1) / parts + 63) / 64 * 64;
  return {(cols + len - 1) / len, len};
}
int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

// Rows of at most this many scores go to workgroups of one wave.  Ten
// alternatives, a wave and 256 threads: 4,096 rows of 500 9.5 and 20.3 us, of
// 2,048 13.1 and 22.0, of 4,096 17.9 and 22.0, of 8,192 30.8 and 32.4; 100 rows
// of 500 6.2 and 6.5, of 2,048 6.7 and 6.7, of 3,000 7.1 and 6.7, of 8,192 9.5 and
// 6.8.  Their gradient: 4,096 rows of 500 5.6 and 9.2, of 2,048 12.3 and 12.8.
constexpr int64_t kShortRow = 2048;

template <bool V>
using Flag = std::integral_constant<bool, V>;
template <class F>
void with_flags(bool a, bool b, const F &f) {
  if (a && b) f(Flag<true>{}, Flag<true>{});
  else if (a) f(Flag<true>{}, Flag<false>{});
  else if (b) f(Flag<false>{}, Flag<true>{});
  else f(Flag<false>{}, Flag<false>{});
}

template <class T>
hipError_t log_probs(const LogProbs &p, hipStream_t stream) {
  const dim3 groups((unsigned)std::min(p.rows * p.parts, kMostGroups));
  with_flags(p.ex, p.top, [&](auto ex, auto top) {
    constexpr bool EX = decltype(ex)::value, TOP = decltype(top)::value;
    if (p.cols <= kShortRow)
      hipLaunchKernelGGL((k_log_probs<T, EX, TOP, 64>), groups, dim3(64), 0, stream, p);
    else
      hipLaunchKernelGGL((k_log_probs<T, EX, TOP, kThreads>), groups, dim3(kThreads), 0, stream,
                         p);
  });
  if (p.parts > 1)
    hipLaunchKernelGGL(k_log_probs_join<T>, dim3((unsigned)std::min(p.rows, kMostGroups)),
                       dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <class T>
hipError_t log_probs_grad(LogProbsGrad p, hipStream_t stream) {
  with_flags(p.ex, p.g_entropy, [&](auto ex, auto ent) {
    constexpr bool EX = decltype(ex)::value, ENT = decltype(ent)::value;
    const auto go = [&](auto threads) {
      constexpr int TH = decltype(threads)::value;
      constexpr int64_t kTile = (int64_t)TH * kGradGroup * Vec<T>::N;
      p.tiles = (p.cols + kTile - 1) / kTile;
      hipLaunchKernelGGL((k_log_probs_grad<T, EX, ENT, TH>),
                         dim3((unsigned)std::min(p.rows * p.tiles, kMostGroups)), dim3(TH), 0,
                         stream, p);
    };
    if (p.cols <= kShortRow) go(std::integral_constant<int, 64>{});
    else go(std::integral_constant<int, kThreads>{});
  });
  return hipGetLastError();
}

// The checks both calls share; 0 if the arguments are valid.
int check_scores(const char *call, const void *scores, int32_t type, int64_t rows, int64_t cols,
                 int64_t stride, const uint8_t *excluded, int64_t excluded_stride, float t) {
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: rows and cols must be in [0, 2^31): %lld x %lld", call,
                     (long long)rows, (long long)cols);
  if (!(t > 0.0f) || !std::isfinite(t) || !std::isfinite(kLog2e / t))
    return fail_call(BGMF_E_ARG, "%s: the temperature must be positive and finite: %g", call, t);
  if (bad_matrix(scores, rows, cols, stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad scores (pointer, alignment or row stride %lld)", call,
                     (long long)stride);
  if (excluded && bad_matrix(excluded, rows, cols, excluded_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad excluded (row stride %lld)", call,
                     (long long)excluded_stride);
  return 0;
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

int64_t bgmf_log_probs_workspace(int64_t rows, int64_t cols, int32_t top) {
  if (rows <= 0 || cols <= 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || top < 0 ||
      top > BGMF_TOP_MAX)
    return 0;
  const int64_t parts = split_of(rows, cols).parts;
  if (parts == 1) return 0;
  return padded(rows * parts * (int64_t)sizeof(PartSum)) + 2 * padded(rows * parts * top * 4);
}

int bgmf_log_probs(const void *scores, int32_t type, int64_t rows, int64_t cols,
                   int64_t row_stride, const uint8_t *excluded, int64_t excluded_stride,
                   const int32_t *given, float temperature, int32_t top, float *log_prob,
                   float *entropy, float *row_max, float *row_sum, int32_t *top_item,
                   float *top_log_prob, void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_log_probs";
  if (const int rc = check_scores(call, scores, type, rows, cols, row_stride, excluded,
                                  excluded_stride, temperature))
    return rc;
  if (top < 0 || top > BGMF_TOP_MAX)
    return fail_call(BGMF_E_ARG, "%s: top must be in [0, %d]: %d", call, BGMF_TOP_MAX, top);
  if (rows == 0) return BGMF_OK;
  if (log_prob && !given) return fail_call(BGMF_E_ARG, "%s: log_prob needs given", call);
  if (top && (!top_item || !top_log_prob))
    return fail_call(BGMF_E_ARG, "%s: top needs top_item and top_log_prob", call);
  const int64_t need = bgmf_log_probs_workspace(rows, cols, top);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 256))
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  const Split split = split_of(rows, cols);
  char *sums = static_cast<char *>(ws);
  char *vs = need ? sums + padded(rows * split.parts * (int64_t)sizeof(PartSum)) : nullptr;
  char *js = need ? vs + padded(rows * split.parts * top * 4) : nullptr;
  const LogProbs p{scores, excluded, given, rows, cols, row_stride, excluded_stride, temperature,
                   top, log_prob, entropy, row_max, row_sum, top_item, top_log_prob, split.parts,
                   split.len, reinterpret_cast<PartSum *>(sums), reinterpret_cast<float *>(vs),
                   reinterpret_cast<int32_t *>(js)};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = type == BGMF_TYPE_F32    ? log_probs<float>(p, stream)
                       : type == BGMF_TYPE_BF16 ? log_probs<bf16_t>(p, stream)
                                                : log_probs<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int bgmf_log_probs_grad(const void *scores, int32_t type, int64_t rows, int64_t cols,
                        int64_t row_stride, const uint8_t *excluded, int64_t excluded_stride,
                        const int32_t *given, float temperature, const float *row_max,
                        const float *row_sum, const float *entropy, const float *grad_log_prob,
                        const float *grad_entropy, void *grad_scores, int64_t grad_stride,
                        void *hip_stream) {
  const char *call = "bgmf_log_probs_grad";
  if (const int rc = check_scores(call, scores, type, rows, cols, row_stride, excluded,
                                  excluded_stride, temperature))
    return rc;
  if (bad_matrix(grad_scores, rows, cols, grad_stride, cols, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad grad_scores (pointer, alignment or row stride %lld)",
                     call, (long long)grad_stride);
  if (rows == 0 || cols == 0) return BGMF_OK;
  if (!row_max || !row_sum) return fail_call(BGMF_E_ARG, "%s: null row_max or row_sum", call);
  if (grad_log_prob && !given) return fail_call(BGMF_E_ARG, "%s: grad_log_prob needs given", call);
  if (grad_entropy && !entropy)
    return fail_call(BGMF_E_ARG, "%s: grad_entropy needs entropy", call);
  if (grad_scores == scores && grad_stride != row_stride && rows > 1)
    return fail_call(BGMF_E_ARG, "%s: in place, the row strides must be equal", call);
  const auto shares = [&](const void *q, int32_t q_type, int64_t q_rows, int64_t q_cols,
                          int64_t q_stride) {
    return share(grad_scores, type, rows, cols, grad_stride, q, q_type, q_rows, q_cols, q_stride);
  };
  if ((grad_scores != scores && shares(scores, type, rows, cols, row_stride)) ||
      shares(excluded, BGMF_TYPE_I8, rows, cols, excluded_stride) ||
      shares(given, BGMF_TYPE_F32, 1, rows, rows) || shares(row_max, BGMF_TYPE_F32, 1, rows, rows) ||
      shares(row_sum, BGMF_TYPE_F32, 1, rows, rows) ||
      shares(entropy, BGMF_TYPE_F32, 1, rows, rows) ||
      shares(grad_log_prob, BGMF_TYPE_F32, 1, rows, rows) ||
      shares(grad_entropy, BGMF_TYPE_F32, 1, rows, rows))
    return fail_call(BGMF_E_ARG, "%s: grad_scores shares memory with an input", call);
  const LogProbsGrad p{scores, excluded, given, rows, cols, row_stride, excluded_stride,
                       grad_stride, temperature, row_max, row_sum, entropy, grad_log_prob,
                       grad_entropy, grad_scores, 0};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = type == BGMF_TYPE_F32    ? log_probs_grad<float>(p, stream)
                       : type == BGMF_TYPE_BF16 ? log_probs_grad<bf16_t>(p, stream)
                                                : log_probs_grad<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
