// Log probabilities of given items with entropy and top alternatives
// (bgmf_log_probs), and their gradient (bgmf_log_probs_grad).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.44269504088896341f;
constexpr double kLn2 = 0.69314718055994530942;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
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
  __device__ __forceinline__ void load(int32_t v, float (&out)[N]) const {
    const Vec<T> a = load_vec(x + (int64_t)v * N);
    uint8_t b[N];
    if constexpr (EX) __builtin_memcpy(b, ex + (int64_t)v * N, N);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      out[i] = to_float(a.v[i]);
      if constexpr (EX) out[i] = b[i] ? -INFINITY : out[i];
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
  __device__ __forceinline__ void add(const float (&x)[COUNT], float c) {
    float gm = x[0];
#pragma unroll
    for (int i = 1; i < COUNT; ++i) gm = fmaxf(gm, x[i]);
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
struct SoftLds {
  float m[kWaves];
  double s[kWaves], w[kWaves];
};
__device__ __forceinline__ Soft block_soft(Soft a, float c, SoftLds &lds) {
  const int wave = threadIdx.x / 64;
  const float wm = wave_max(a.m);
  if (threadIdx.x % 64 == 0) lds.m[wave] = wm;
  __syncthreads();
  float M = lds.m[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) M = fmaxf(M, lds.m[i]);
  a.rescale(M, c);
  const double s = wave_sum(a.s), w = wave_sum(a.w);
  if (threadIdx.x % 64 == 0) lds.s[wave] = s, lds.w[wave] = w;
  __syncthreads();
  Soft r;
  r.m = M;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) r.s += lds.s[i], r.w += lds.w[i];
  return r;
}

// ---------------------------------------------------------------------------
// The n best of the scores that a workgroup has just gone through, larger
// first, ties to the lower item.  A thread kept the largest of its scores, tm.
// The n-th largest of the 256 tm is a score that the n best are not below, and
// only the threads with tm at or above it ("hot", about n) can hold any of
// them: their scores, n / 256 of the row, are read once more (from the cache),
// and those at or above the bound, few more than n, are put in order by
// counting how many precede each.  If more than kCandidates qualify (equal
// scores, or the best ones all with few threads), the scores are gone through
// in order of items instead, merging each tile's candidates into a list.
//
// SRC: per_thread() items of a thread; visit(thread, i, f): f(score, item) for
// each score of its i-th; size() and at(p, item): all scores in the order of
// items.  emit(rank, score, item), for every rank below n (item -1: none).
// ---------------------------------------------------------------------------
constexpr int kCandidates = 1024;
struct TopLds {
  float tm[kThreads];
  uint8_t hot[kThreads];
  float v[kCandidates];
  int32_t j[kCandidates];
  float lv[2][BGMF_TOP_MAX];
  int32_t lj[2][BGMF_TOP_MAX];
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

// By one wave: a score that at least n of the 256 tm are not below, and few
// more than n; -inf if fewer than n are above -inf.
__device__ __forceinline__ float top_bound(const float *tm, int n) {
  const int32_t none = key_of(-INFINITY);
  int32_t k[kWaves], lo = 0x7FFFFFFF, hi = none;
  int some = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    k[i] = key_of(tm[threadIdx.x % 64 + 64 * i]);
    if (k[i] > none) lo = min(lo, k[i]);
    hi = max(hi, k[i]);
    some += __popcll(__ballot(k[i] > none));
  }
  if (some < n) return -INFINITY;
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  while (lo < hi) {  // at least n are at or above lo, fewer than n above hi
    const int32_t mid = (int32_t)((uint32_t)lo + ((uint32_t)hi - (uint32_t)lo + 1) / 2);
    int c = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) c += __popcll(__ballot(k[i] >= mid));
    if (c >= n) {
      lo = mid;
      if (c <= n + 2 + n / 8) break;
    } else {
      hi = mid - 1;
    }
  }
  return of_key(lo);
}

__device__ __forceinline__ bool precedes(float v, int32_t j, float w, int32_t l) {
  return v > w || (v == w && j < l);
}

template <class SRC, class EMIT>
__device__ void top_in_order(const SRC &src, int n, TopLds &lds, float bound, const EMIT &emit) {
  const int tid = threadIdx.x;
  int have = 0, now = 0;
  constexpr int kPer = kCandidates / kThreads;
  for (int64_t p0 = 0; p0 < src.size(); p0 += kCandidates) {
    if (tid == 0) lds.count = 0;
    __syncthreads();
    const float worst = have == n ? lds.lv[now][n - 1] : -INFINITY;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int64_t p = p0 + q * kThreads + tid;
      if (p < src.size()) {
        int32_t j;
        const float v = src.at(p, j);
        if (v > worst && v >= bound) {  // a later item loses a tie
          const int at = atomicAdd(&lds.count, 1);
          lds.v[at] = v, lds.j[at] = j;
        }
      }
    }
    __syncthreads();
    const int c = lds.count;
    if (c) {
      for (int i = tid; i < c + have; i += kThreads) {
        const bool old = i >= c;
        const float v = old ? lds.lv[now][i - c] : lds.v[i];
        const int32_t j = old ? lds.lj[now][i - c] : lds.j[i];
        int rank = 0;
        for (int o = 0; o < c; ++o) rank += precedes(lds.v[o], lds.j[o], v, j);
        for (int o = 0; o < have; ++o) rank += precedes(lds.lv[now][o], lds.lj[now][o], v, j);
        if (rank < n) lds.lv[now ^ 1][rank] = v, lds.lj[now ^ 1][rank] = j;
      }
      have = min(n, have + c);
      now ^= 1;
      __syncthreads();
    }
  }
  for (int i = tid; i < n; i += kThreads)
    emit(i, i < have ? lds.lv[now][i] : -INFINITY, i < have ? lds.lj[now][i] : -1);
}

// Called by the whole workgroup; lds is free for other use after the next
// barrier.
template <class SRC, class EMIT>
__device__ __forceinline__ void top_select(const SRC &src, float tm, int n, TopLds &lds,
                                           const EMIT &emit) {
  const int tid = threadIdx.x;
  lds.tm[tid] = tm;
  if (tid == 0) lds.hots = lds.count = 0;
  __syncthreads();
  if (tid < 64) {
    const float b = top_bound(lds.tm, n);
    if (tid == 0) lds.bound = b;
  }
  __syncthreads();
  const float bound = lds.bound;
  if (tm > -INFINITY && tm >= bound) lds.hot[atomicAdd(&lds.hots, 1)] = (uint8_t)tid;
  __syncthreads();
  const uint32_t per = (uint32_t)src.per_thread(), items = (uint32_t)lds.hots * per;
  for (uint32_t i = tid; i < items; i += kThreads)
    src.visit(lds.hot[i / per], (int32_t)(i % per), [&](float v, int32_t j) {
      if (v > -INFINITY && v >= bound) {
        const int at = atomicAdd(&lds.count, 1);
        if (at < kCandidates) lds.v[at] = v, lds.j[at] = j;
      }
    });
  __syncthreads();
  const int c = lds.count;
  if (c > kCandidates) {
    __syncthreads();
    top_in_order(src, n, lds, bound, emit);
    return;
  }
  for (int i = tid; i < c; i += kThreads) {
    const float v = lds.v[i];
    const int32_t j = lds.j[i];
    int rank = 0;
    for (int o = 0; o < c; ++o) rank += precedes(lds.v[o], lds.j[o], v, j);
    if (rank < n) emit(rank, v, j);
  }
  for (int i = c + tid; i < n; i += kThreads) emit(i, -INFINITY, -1);
}

template <class T, bool EX>
struct RowSource {  // thread t has vectors t, t + 256, ... and element t of the tail
  Row<T, EX> row;
  int32_t first;  // item of the row's first element
  __device__ __forceinline__ int32_t per_thread() const {
    return (row.vecs() + kThreads - 1) / kThreads + 1;
  }
  template <class F>
  __device__ __forceinline__ void visit(int t, int32_t i, const F &f) const {
    constexpr int N = Row<T, EX>::N;
    const int32_t vecs = row.vecs();
    if (i == 0) {
      if (t < row.len - vecs * N) f(row.one(vecs * N + t), first + vecs * N + t);
      return;
    }
    const int32_t v = t + (i - 1) * kThreads;
    if (v >= vecs) return;
    float x[N];
    row.load(v, x);
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
constexpr int kGroup = 4;
template <class T, bool EX, bool TOP>
__global__ void __launch_bounds__(kThreads) k_log_probs(LogProbs P) {
  __shared__ SoftLds soft_lds;
  __shared__ typename std::conditional<TOP, TopLds, int>::type top_lds;
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
    const int32_t vecs = row.vecs();
    for (int32_t v = tid; v < vecs; v += kThreads * kGroup) {
      float x[kGroup][N];
#pragma unroll
      for (int g = 0; g < kGroup; ++g) {
        if (v + g * kThreads < vecs) row.load(v + g * kThreads, x[g]);
        else
#pragma unroll
          for (int i = 0; i < N; ++i) x[g][i] = -INFINITY;
      }
      a.add(reinterpret_cast<float(&)[kGroup * N]>(x), c);
    }
    if (tid < row.len - vecs * N) {
      const float x[1] = {row.one(vecs * N + tid)};
      a.add(x, c);
    }
    const float tm = a.m;
    const Soft all = block_soft(a, c, soft_lds);
    const float log_s = logf((float)all.s);
    if (tid == 0) {
      if (P.parts == 1) write_row<T>(P, r, all, log_s);
      else P.part_sum[u] = PartSum{all.s, all.w, all.m};
    }
    if constexpr (TOP) {
      const int n = P.top;
      const RowSource<T, EX> src{row, (int32_t)first};
      if (P.parts == 1)
        top_select(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
          P.top_item[r * n + rank] = j;
          P.top_log_prob[r * n + rank] = j < 0 ? v : (v - all.m) / P.temperature - log_s;
        });
      else
        top_select(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
          P.part_v[u * n + rank] = v;
          P.part_j[u * n + rank] = j;
        });
    }
    __syncthreads();  // before the next row uses LDS
  }
}

struct PartSource {  // thread t has the lists of parts t, t + 256, ...
  const float *v;
  const int32_t *j;
  int64_t parts;
  int n;
  __device__ __forceinline__ int32_t per_thread() const {
    return (int32_t)((parts + kThreads - 1) / kThreads) * n;
  }
  template <class F>
  __device__ __forceinline__ void visit(int t, int32_t i, const F &f) const {
    const int64_t part = t + (int64_t)(i / n) * kThreads;
    if (part < parts) f(v[part * n + i % n], j[part * n + i % n]);
  }
  __device__ __forceinline__ int64_t size() const { return parts * n; }
  __device__ __forceinline__ float at(int64_t p, int32_t &item) const {
    item = j[p];
    return v[p];
  }
};

// Joins the parts of a row: one workgroup per row.
template <class T>
__global__ void __launch_bounds__(kThreads) k_log_probs_join(LogProbs P) {
  __shared__ SoftLds soft_lds;
  __shared__ TopLds top_lds;
  const int tid = threadIdx.x, n = P.top;
  const float c = kLog2e / P.temperature;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const PartSum *sums = P.part_sum + r * P.parts;
    Soft a;
    for (int64_t i = tid; i < P.parts; i += kThreads) {
      Soft b;
      b.m = sums[i].m, b.s = sums[i].s, b.w = sums[i].w;
      const float M = fmaxf(a.m, b.m);
      a.rescale(M, c);
      b.rescale(M, c);
      a.m = M, a.s += b.s, a.w += b.w;
    }
    const float tm = a.m;
    const Soft all = block_soft(a, c, soft_lds);
    const float log_s = logf((float)all.s);
    if (tid == 0) write_row<T>(P, r, all, log_s);
    if (n) {
      const PartSource src{P.part_v + r * P.parts * n, P.part_j + r * P.parts * n, P.parts, n};
      top_select(src, tm, n, top_lds, [&](int rank, float v, int32_t j) {
        P.top_item[r * n + rank] = j;
        P.top_log_prob[r * n + rank] = j < 0 ? v : (v - all.m) / P.temperature - log_s;
      });
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient: every score is read and its gradient written once.  A workgroup
// takes a tile of one row at a time.  Bound: HBM.
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

template <class T, bool EX, bool ENT>
__global__ void __launch_bounds__(kThreads) k_log_probs_grad(LogProbsGrad P) {
  constexpr int N = Vec<T>::N;
  constexpr int64_t kGradTile = (int64_t)kThreads * kGradGroup * N;
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
      const int32_t i = (tid + q * kThreads) * N;
      if (i + N <= len) {
        a[q] = load_vec(x + i);
        if constexpr (EX) __builtin_memcpy(b[q], ex + i, N);
      }
    }
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * kThreads) * N;
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

// How a row is split: enough workgroups to fill the GPU (eight for each of
// 256 CUs) while a part keeps 64 KB or so of scores, and a row at most 1024
// parts.
constexpr int64_t kFullGpu = 2048, kLeastPart = 16384, kMostParts = 1024;
struct Split {
  int64_t parts, len;
};
Split split_of(int64_t rows, int64_t cols) {
  int64_t parts = std::min({(cols + kLeastPart - 1) / kLeastPart,
                            std::max<int64_t>(kFullGpu / std::max<int64_t>(rows, 1), 1), kMostParts});
  if (parts <= 1) return {1, cols};
  const int64_t len = ((cols + parts - 1) / parts + 63) / 64 * 64;
  return {(cols + len - 1) / len, len};
}
int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

template <class T>
hipError_t log_probs(const LogProbs &p, hipStream_t stream) {
  const dim3 groups((unsigned)std::min(p.rows * p.parts, kMostGroups)), threads(kThreads);
  if (p.ex) {
    if (p.top) hipLaunchKernelGGL((k_log_probs<T, true, true>), groups, threads, 0, stream, p);
    else hipLaunchKernelGGL((k_log_probs<T, true, false>), groups, threads, 0, stream, p);
  } else {
    if (p.top) hipLaunchKernelGGL((k_log_probs<T, false, true>), groups, threads, 0, stream, p);
    else hipLaunchKernelGGL((k_log_probs<T, false, false>), groups, threads, 0, stream, p);
  }
  if (p.parts > 1)
    hipLaunchKernelGGL(k_log_probs_join<T>, dim3((unsigned)std::min(p.rows, kMostGroups)), threads,
                       0, stream, p);
  return hipGetLastError();
}

template <class T>
hipError_t log_probs_grad(LogProbsGrad p, hipStream_t stream) {
  constexpr int64_t kTile = (int64_t)kThreads * kGradGroup * Vec<T>::N;
  p.tiles = (p.cols + kTile - 1) / kTile;
  const dim3 groups((unsigned)std::min(p.rows * p.tiles, kMostGroups)), threads(kThreads);
  if (p.ex) {
    if (p.g_entropy)
      hipLaunchKernelGGL((k_log_probs_grad<T, true, true>), groups, threads, 0, stream, p);
    else hipLaunchKernelGGL((k_log_probs_grad<T, true, false>), groups, threads, 0, stream, p);
  } else {
    if (p.g_entropy)
      hipLaunchKernelGGL((k_log_probs_grad<T, false, true>), groups, threads, 0, stream, p);
    else hipLaunchKernelGGL((k_log_probs_grad<T, false, false>), groups, threads, 0, stream, p);
  }
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
