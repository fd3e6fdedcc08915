// The clipped policy loss of shown items with a divergence from a reference
// (bgmf_policy_loss) and its gradient (bgmf_policy_loss_grad).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

// Threads of a workgroup: 256, or one wave for short rows (TH below).
constexpr int kThreads = 256;

struct Policy {
  const void *x, *y;  // scores, and the reference's or null
  const uint8_t *ex;
  const int32_t *given;
  const float *advantage, *old_log_prob, *ref_log_prob;
  int64_t rows, cols, stride, y_stride, ex_stride;
  float temperature, clip_low, clip_high, kl_weight;
  float *loss, *log_prob, *kl;
  float *state;  // [5][rows]: row_max, row_sum, the reference's row_max, slope, mean
  // rows split in `parts` of part_len scores: where the parts' sums go
  int64_t parts, part_len;
  struct PartSum *part_sum;  // [rows][parts]
  // the gradient
  const float *g_loss;
  void *out;
  int64_t out_stride, tiles;  // tiles of a row
};

// Running sums of a row's scores x and of the reference's y, m and my the
// largest of each so far, d = (x - m) c and dy = (y - my) c:
//   s = sum exp2(d)   sy = sum exp2(dy)   w = sum exp2(d) (d - dy)
// from which ln s, ln sy and the mean w / s of d - dy under p give
//   sum p ln(p / q) = (w / s) ln 2 - ln s + ln sy.
// Both differences are taken from their own maximum, so an offset between the
// two policies' scores costs nothing, and one item alone gives exactly 0.  A
// group's terms are summed in fp32 and added to running sums in fp64: the
// divergence is a small difference of large terms.  A score of -inf adds
// nothing; a NaN or +inf makes s (or sy) NaN.
template <bool REF>
struct Sums {
  float m = -INFINITY, my = -INFINITY;
  double s = 0.0, w = 0.0, sy = 0.0;
  static __device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
  // to the maxima M >= m and My >= my
  __device__ __forceinline__ void rescale(float M, float My, float c) {
    if (m != -INFINITY) {  // (otherwise s and w are 0, or NaN from a NaN)
      const float f = __builtin_amdgcn_exp2f((m - M) * c);
      // (in 64 bits, where maxima of the type's lowest value leave it finite)
      if constexpr (REF)
        w = (w + s * ((((double)m - M) + ((double)base_of(My) - base_of(my))) * c)) * f;
      s *= f;
    }
    if constexpr (REF)
      if (my != -INFINITY) sy *= __builtin_amdgcn_exp2f((my - My) * c);
    m = M, my = My;
  }
  template <int COUNT>
  __device__ __forceinline__ void add(const float (&x)[COUNT], const float (&y)[COUNT], float gm,
                                      float gmy, float c) {  // the largest of x and of y
    // d and dy are rounded alike, so that equal scores leave exactly 0
#pragma clang fp contract(off)
    if (gm > m || (REF && gmy > my)) rescale(fmaxf(m, gm), REF ? fmaxf(my, gmy) : my, c);
    const float bx = base_of(m), by = base_of(my);
    float gs = 0.0f, gw = 0.0f, gy = 0.0f;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const float d = (x[i] - bx) * c, e = __builtin_amdgcn_exp2f(d);
      gs += e;
      if constexpr (REF) {
        const float dy = (y[i] - by) * c, t = e * (d - dy);
        gy += __builtin_amdgcn_exp2f(dy);
        gw += e > 0.0f ? t : 0.0f;  // (e may be 0 where d - dy is not finite)
      }
    }
    s += gs;
    if constexpr (REF) w += gw, sy += gy;
  }
};

// Over the workgroup in a fixed order; every thread has the result.
template <int TH>
struct SumsLds {
  float m[TH / 64], my[TH / 64];
  double s[TH / 64], w[TH / 64], sy[TH / 64];
};
template <int TH, bool REF>
__device__ __forceinline__ Sums<REF> block_sums(Sums<REF> a, float c, SumsLds<TH> &lds) {
  constexpr int W = TH / 64;
  const int wave = threadIdx.x / 64;
  Sums<REF> r;
  r.m = wave_max(a.m);
  if constexpr (REF) r.my = wave_max(a.my);
  if constexpr (W > 1) {
    if (threadIdx.x % 64 == 0) lds.m[wave] = r.m, lds.my[wave] = r.my;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) {
      r.m = fmaxf(r.m, lds.m[i]);
      if constexpr (REF) r.my = fmaxf(r.my, lds.my[i]);
    }
  }
  a.rescale(r.m, r.my, c);
  a.s = wave_sum(a.s);
  if constexpr (REF) a.w = wave_sum(a.w), a.sy = wave_sum(a.sy);
  if constexpr (W == 1) {
    r.s = a.s, r.w = a.w, r.sy = a.sy;
  } else {
    if (threadIdx.x % 64 == 0) lds.s[wave] = a.s, lds.w[wave] = a.w, lds.sy[wave] = a.sy;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) {
      r.s += lds.s[i];
      if constexpr (REF) r.w += lds.w[i], r.sy += lds.sy[i];
    }
  }
  return r;
}

// What the gradient needs of a row: with d and dy as above,
//   dx_j = g / t (slope (1[j = given] - p_j) + kl_weight p_j ln 2 (d_j - dy_j - mean))
struct State {
  float m, s, my, slope, mean;  // s = 0: the row's gradient is 0
};

// The row's results, by one thread, in 64 bits.
template <class T, bool REF>
__device__ __forceinline__ State finish(const Policy &P, int64_t r, const Sums<REF> &a) {
  State st{a.m, (float)a.s, a.my, 0.0f, 0.0f};
  double loss = 0.0, lp = 0.0, kl = 0.0;
  const int64_t g = P.given[r];
  if (g == -1) {
    st.s = 0.0f;
  } else {
    const bool outside = g < 0 || g >= P.cols, none = a.s == 0.0;
    const double ln_s = none ? 0.0 : log(a.s);
    lp = -INFINITY;
    if (outside) lp = NAN;
    else if (!none && !(P.ex && P.ex[r * P.ex_stride + g]))
      lp = ((double)to_float(static_cast<const T *>(P.x)[r * P.stride + g]) - (double)a.m) /
               (double)P.temperature - ln_s;
    if (!none || outside) {
      const double A = P.advantage[r], rho = exp(lp - (double)P.old_log_prob[r]);
      const double lo = 1.0 - (double)P.clip_low, hi = 1.0 + (double)P.clip_high;
      const double unclipped = rho * A, clipped = (rho < lo ? lo : rho > hi ? hi : rho) * A;
      const bool passes = !(unclipped > clipped);
      loss = -(passes ? unclipped : clipped);
      double slope = passes ? -unclipped : 0.0;
      if (P.ref_log_prob) {
        const double z = (double)P.ref_log_prob[r] - lp, e = expm1(z);
        kl = z == INFINITY ? INFINITY : e - z;
        if (P.kl_weight != 0.0f) slope -= (double)P.kl_weight * e;
      }
      st.slope = (float)slope;
    }
    if constexpr (REF) {
      if (!none) {
        const double mean = a.w / a.s;
        st.mean = (float)mean;
        kl = a.sy == 0.0 ? INFINITY : mean * kLn2 - ln_s + log(a.sy);
      }
    }
    if (P.kl_weight != 0.0f) loss += (double)P.kl_weight * kl;
  }
  if (P.loss) P.loss[r] = (float)loss;
  if (P.log_prob) P.log_prob[r] = (float)lp;
  if (P.kl) P.kl[r] = (float)kl;
  if (P.state) {
    P.state[r] = st.m, P.state[P.rows + r] = st.s, P.state[2 * P.rows + r] = st.my;
    P.state[3 * P.rows + r] = st.slope, P.state[4 * P.rows + r] = st.mean;
  }
  return st;
}

struct PartSum {
  double s, w, sy;
  float m, my;
};

// Scores as a row's vectors hold them, those of excluded items -inf in both.
template <class T, bool EX, bool REF>
struct Pair {
  static constexpr int N = Vec<T>::N;
  Row<T, EX> row;
  const T *y;
  struct Raw {
    typename Row<T, EX>::Raw x;
    Vec<T> y;
  };
  __device__ __forceinline__ Raw fetch(int32_t v) const {
    Raw r;
    r.x = row.fetch(v);
    if constexpr (REF) r.y = load_vec(y + (int64_t)v * N);
    return r;
  }
  static __device__ __forceinline__ Raw nothing() {
    Raw r;
    r.x = Row<T, EX>::nothing();
    if constexpr (REF)
#pragma unroll
      for (int i = 0; i < N; ++i) r.y.v[i] = from_float<T>(-INFINITY);
    return r;
  }
  static __device__ __forceinline__ void scores(const Raw &r, float (&x)[N], float (&z)[N]) {
    Row<T, EX>::scores(r.x, x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] = -INFINITY;
      if constexpr (REF) {
        z[i] = to_float(r.y.v[i]);
        if constexpr (EX) z[i] = r.x.b[i / 4] >> (i % 4 * 8) & 0xFF ? -INFINITY : z[i];
      }
    }
  }
};

// One workgroup per row, or per part of a row; the scores and the reference are
// read once.
constexpr int kGroup = 2;
template <class T, bool EX, bool REF, int TH>
__global__ void __launch_bounds__(TH) k_policy(Policy P) {
  __shared__ SumsLds<TH> lds;
  using Two = Pair<T, EX, REF>;
  constexpr int N = Two::N;
  const int tid = threadIdx.x;
  const float c = kLog2e / P.temperature;
  const int64_t units = P.rows * P.parts;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t r = P.parts == 1 ? u : u / P.parts, part = P.parts == 1 ? 0 : u % P.parts;
    const int64_t first = part * P.part_len;
    const int64_t left = P.cols - first;
    const int32_t len = P.given[r] == -1 ? 0 : (int32_t)(left < P.part_len ? left : P.part_len);
    const Two two{{static_cast<const T *>(P.x) + (r * P.stride + first),
                   EX ? P.ex + (r * P.ex_stride + first) : nullptr, len},
                  REF ? static_cast<const T *>(P.y) + (r * P.y_stride + first) : nullptr};
    Sums<REF> a;
    const int32_t vecs = two.row.vecs();
    for (int32_t v0 = 0; v0 < vecs; v0 += TH * kGroup) {
      typename Two::Raw raw[kGroup];
#pragma unroll
      for (int g = 0; g < kGroup; ++g) {
        raw[g] = Two::nothing();
        if (v0 + g * TH + tid < vecs) raw[g] = two.fetch(v0 + g * TH + tid);
      }
#pragma unroll
      for (int g = 0; g < kGroup; ++g) {
        float x[N], y[N], gm = -INFINITY, gmy = -INFINITY;
        Two::scores(raw[g], x, y);
#pragma unroll
        for (int i = 0; i < N; ++i) gm = fmaxf(gm, x[i]), gmy = fmaxf(gmy, y[i]);
        a.add(x, y, gm, gmy, c);
      }
    }
    if (tid < len - vecs * N) {
      const int32_t i = vecs * N + tid;
      const float x[1] = {two.row.one(i)};
      float y[1] = {-INFINITY};
      if constexpr (REF)
        if (!EX || !two.row.ex[i]) y[0] = to_float(two.y[i]);
      a.add(x, y, x[0], y[0], c);
    }
    const Sums<REF> all = block_sums<TH>(a, c, lds);
    if (tid == 0) {
      if (P.parts == 1) finish<T>(P, r, all);
      else P.part_sum[u] = PartSum{all.s, all.w, all.sy, all.m, all.my};
    }
    __syncthreads();  // before the next row uses LDS
  }
}

// Joins the parts of a row: one workgroup per row.
constexpr int64_t kMostParts = 4 * kThreads;
template <class T, bool REF>
__global__ void __launch_bounds__(kThreads) k_policy_join(Policy P) {
  __shared__ SumsLds<kThreads> lds;
  const float c = kLog2e / P.temperature;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const PartSum *sums = P.part_sum + r * P.parts;
    Sums<REF> a;
    for (int64_t i = threadIdx.x; i < P.parts; i += kThreads) {
      Sums<REF> b;
      b.m = sums[i].m, b.s = sums[i].s;
      if constexpr (REF) b.my = sums[i].my, b.w = sums[i].w, b.sy = sums[i].sy;
      const float M = fmaxf(a.m, b.m), My = fmaxf(a.my, b.my);
      a.rescale(M, My, c);
      b.rescale(M, My, c);
      a.s += b.s, a.w += b.w, a.sy += b.sy;
    }
    const Sums<REF> all = block_sums<kThreads>(a, c, lds);
    if (threadIdx.x == 0) finish<T>(P, r, all);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient: the scores and the reference are read and the gradient is written
// once.  A workgroup takes a tile of one row at a time.
// ---------------------------------------------------------------------------

// A row's gradient from its scores.
template <class T, bool REF>
struct Slopes {
  float c, m, my, inv, gs, gk, mean;
  bool none;
  int64_t given;
  __device__ __forceinline__ Slopes(const Policy &P, int64_t r, const State &st) {
    c = kLog2e / P.temperature;
    const float g = (P.g_loss ? P.g_loss[r] : 1.0f) / P.temperature;
    given = P.given[r];
    m = st.m, my = Sums<REF>::base_of(st.my), mean = st.mean;
    none = st.s == 0.0f;
    inv = 1.0f / st.s;
    gs = g * st.slope;
    gk = REF && P.kl_weight != 0.0f ? g * P.kl_weight * (float)kLn2 : 0.0f;
  }
  __device__ __forceinline__ T operator()(float x, float y, int64_t j, bool excluded) const {
#pragma clang fp contract(off)
    const float d = (x - m) * c, p = __builtin_amdgcn_exp2f(d) * inv;
    float v = -gs * p;
    if constexpr (REF) {
      const float dy = (y - my) * c, t = p * (gk * ((d - dy) - mean));
      v += p == 0.0f || gk == 0.0f ? 0.0f : t;
    }
    if (j == given) v += gs;
    return from_float<T>(excluded || none ? 0.0f : v);
  }
};

constexpr int kGradGroup = 2;
template <class T, bool EX, bool REF, int TH>
__global__ void __launch_bounds__(TH) k_policy_grad(Policy P) {
  constexpr int N = Vec<T>::N;
  constexpr int64_t kTile = (int64_t)TH * kGradGroup * N;
  const int tid = threadIdx.x;
  for (int64_t u = blockIdx.x; u < P.rows * P.tiles; u += gridDim.x) {
    const int64_t r = u / P.tiles, first = u % P.tiles * kTile, left = P.cols - first;
    const int32_t len = (int32_t)(left < kTile ? left : kTile);
    const T *x = static_cast<const T *>(P.x) + (r * P.stride + first);
    const T *y = REF ? static_cast<const T *>(P.y) + (r * P.y_stride + first) : nullptr;
    const uint8_t *ex = EX ? P.ex + (r * P.ex_stride + first) : nullptr;
    T *out = static_cast<T *>(P.out) + (r * P.out_stride + first);
    const State st{P.state[r], P.state[P.rows + r], P.state[2 * P.rows + r],
                   P.state[3 * P.rows + r], P.state[4 * P.rows + r]};
    const Slopes<T, REF> grad(P, r, st);
    Vec<T> a[kGradGroup], b[kGradGroup];
    uint8_t e[kGradGroup][N];
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * TH) * N;
      if (i + N <= len) {
        a[q] = load_vec(x + i);
        if constexpr (REF) b[q] = load_vec(y + i);
        if constexpr (EX) __builtin_memcpy(e[q], ex + i, N);
      }
    }
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * TH) * N;
      if (i + N <= len) {
        Vec<T> v;
#pragma unroll
        for (int k = 0; k < N; ++k)
          v.v[k] = grad(to_float(a[q].v[k]), REF ? to_float(b[q].v[k]) : 0.0f, first + i + k,
                        EX && e[q][k]);
        store_vec(out + i, v);
      } else {
        for (int k = 0; k < N; ++k)
          if (i + k < len)
            out[i + k] = grad(to_float(x[i + k]), REF ? to_float(y[i + k]) : 0.0f, first + i + k,
                              EX && ex[i + k]);
      }
    }
  }
}

constexpr int64_t kMostGroups = 1 << 20;

// How a row is split: in as few parts as hold at most kPart scores each, but no
// more than fill the GPU or than kMostParts.
constexpr int64_t kFullGpu = 2048, kPart = 16384;
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

constexpr int64_t kShortRow = 2048;  // rows for workgroups of one wave

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
void policy_grad(Policy p, hipStream_t stream) {
  with_flags(p.ex, p.y, [&](auto ex, auto ref) {
    constexpr bool EX = decltype(ex)::value, REF = decltype(ref)::value;
    const auto go = [&](auto threads) {
      constexpr int TH = decltype(threads)::value;
      constexpr int64_t kTile = (int64_t)TH * kGradGroup * Vec<T>::N;
      p.tiles = (p.cols + kTile - 1) / kTile;
      hipLaunchKernelGGL((k_policy_grad<T, EX, REF, TH>),
                         dim3((unsigned)std::min(p.rows * p.tiles, kMostGroups)), dim3(TH), 0,
                         stream, p);
    };
    if (p.cols <= kShortRow) go(std::integral_constant<int, 64>{});
    else go(std::integral_constant<int, kThreads>{});
  });
}

template <class T>
hipError_t policy(const Policy &p, hipStream_t stream) {
  with_flags(p.ex, p.y, [&](auto ex, auto ref) {
    constexpr bool EX = decltype(ex)::value, REF = decltype(ref)::value;
    const dim3 groups((unsigned)std::min(p.rows * p.parts, kMostGroups));
    if (p.cols <= kShortRow)
      hipLaunchKernelGGL((k_policy<T, EX, REF, 64>), groups, dim3(64), 0, stream, p);
    else
      hipLaunchKernelGGL((k_policy<T, EX, REF, kThreads>), groups, dim3(kThreads), 0, stream, p);
    if (p.parts > 1)
      hipLaunchKernelGGL((k_policy_join<T, REF>), dim3((unsigned)std::min(p.rows, kMostGroups)),
                         dim3(kThreads), 0, stream, p);
  });
  if (p.out && p.cols) policy_grad<T>(p, stream);
  return hipGetLastError();
}

// The checks both calls share; 0 if the arguments are valid.
int check_policy(const char *call, const Policy &p, int32_t type, bool backward) {
  if (!is_float_type(type))
    return fail_call(BGMF_E_ARG, "%s: type must be F32, BF16 or F16: %d", call, type);
  if (p.rows < 0 || p.cols < 0 || p.rows >= (1ll << 31) || p.cols >= (1ll << 31))
    return fail_call(BGMF_E_ARG, "%s: rows and cols must be in [0, 2^31): %lld x %lld", call,
                     (long long)p.rows, (long long)p.cols);
  if (!(p.temperature > 0.0f) || !std::isfinite(p.temperature) ||
      !std::isfinite(kLog2e / p.temperature))
    return fail_call(BGMF_E_ARG, "%s: the temperature must be positive and finite: %g", call,
                     p.temperature);
  if (!std::isfinite(p.kl_weight))
    return fail_call(BGMF_E_ARG, "%s: kl_weight must be finite: %g", call, p.kl_weight);
  if (p.rows == 0) return 0;
  if (bad_matrix(p.x, p.rows, p.cols, p.stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad scores (pointer, alignment or row stride %lld)", call,
                     (long long)p.stride);
  if (p.y && bad_matrix(p.y, p.rows, p.cols, p.y_stride, 0, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad reference (alignment or row stride %lld)", call,
                     (long long)p.y_stride);
  if (p.ex && bad_matrix(p.ex, p.rows, p.cols, p.ex_stride, 0, 1))
    return fail_call(BGMF_E_ARG, "%s: bad excluded (row stride %lld)", call,
                     (long long)p.ex_stride);
  if (!p.given) return fail_call(BGMF_E_ARG, "%s: null given", call);
  if (!p.out) {
    if (backward && p.cols) return fail_call(BGMF_E_ARG, "%s: null grad_scores", call);
    return 0;
  }
  if (bad_matrix(p.out, p.rows, p.cols, p.out_stride, p.cols, type_bytes(type)))
    return fail_call(BGMF_E_ARG, "%s: bad grad_scores (alignment or row stride %lld)", call,
                     (long long)p.out_stride);
  if (p.rows > 1 && ((p.out == p.x && p.out_stride != p.stride) ||
                     (p.out == p.y && p.out_stride != p.y_stride)))
    return fail_call(BGMF_E_ARG, "%s: in place, the row strides must be equal", call);
  const auto shares = [&](const void *q, int32_t q_type, int64_t q_rows, int64_t q_cols,
                          int64_t q_stride) {
    return share(p.out, type, p.rows, p.cols, p.out_stride, q, q_type, q_rows, q_cols, q_stride);
  };
  const auto vector = [&](const void *q) { return shares(q, BGMF_TYPE_F32, 1, p.rows, p.rows); };
  if ((p.out != p.x && shares(p.x, type, p.rows, p.cols, p.stride)) ||
      (p.out != p.y && shares(p.y, type, p.rows, p.cols, p.y_stride)) ||
      shares(p.ex, BGMF_TYPE_I8, p.rows, p.cols, p.ex_stride) || vector(p.given) ||
      vector(p.advantage) || vector(p.old_log_prob) || vector(p.ref_log_prob) ||
      vector(p.g_loss) || vector(p.loss) || vector(p.log_prob) || vector(p.kl) ||
      shares(p.state, BGMF_TYPE_F32, 5, p.rows, p.rows))
    return fail_call(BGMF_E_ARG, "%s: grad_scores shares memory with another argument", call);
  return 0;
}

}  // namespace
}  // namespace bgmfk

using namespace bgmfk;

extern "C" {

// Workspace: the parts' sums, then row_state where the caller wants none.
int64_t bgmf_policy_loss_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows >= (1ll << 31) || cols >= (1ll << 31)) return 0;
  const int64_t parts = split_of(rows, cols).parts;
  return (parts == 1 ? 0 : padded(rows * parts * (int64_t)sizeof(PartSum))) +
         padded(5 * rows * (int64_t)sizeof(float));
}

int bgmf_policy_loss(const void *scores, int32_t type, int64_t rows, int64_t cols,
                     int64_t row_stride, const void *reference, int64_t reference_stride,
                     const uint8_t *excluded, int64_t excluded_stride, const int32_t *given,
                     const float *advantage, const float *old_log_prob,
                     const float *reference_log_prob, float temperature, float clip_low,
                     float clip_high, float kl_weight, float *loss, float *log_prob, float *kl,
                     float *row_state, const float *grad_loss, void *grad_scores,
                     int64_t grad_stride, void *ws, int64_t ws_bytes, void *hip_stream) {
  const char *call = "bgmf_policy_loss";
  Policy p{};
  p.x = scores, p.y = reference, p.ex = excluded, p.given = given;
  p.advantage = advantage, p.old_log_prob = old_log_prob, p.ref_log_prob = reference_log_prob;
  p.rows = rows, p.cols = cols, p.stride = row_stride, p.y_stride = reference_stride;
  p.ex_stride = excluded_stride;
  p.temperature = temperature, p.clip_low = clip_low, p.clip_high = clip_high;
  p.kl_weight = kl_weight, p.loss = loss, p.log_prob = log_prob, p.kl = kl, p.state = row_state;
  p.g_loss = grad_loss, p.out = grad_scores, p.out_stride = grad_stride;
  if (const int rc = check_policy(call, p, type, false)) return rc;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f))
    return fail_call(BGMF_E_ARG, "%s: clip_low must be in [0, 1] and clip_high at least 0: %g, %g",
                     call, clip_low, clip_high);
  if (reference && reference_log_prob)
    return fail_call(BGMF_E_ARG, "%s: reference or reference_log_prob, not both", call);
  if (rows == 0) return BGMF_OK;
  if (!advantage || !old_log_prob)
    return fail_call(BGMF_E_ARG, "%s: null advantage or old_log_prob", call);
  const int64_t need = bgmf_policy_loss_workspace(rows, cols);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 256))
    return fail_call(BGMF_E_ARG, "%s: the workspace must start on a 256-byte boundary", call);
  if (ws_bytes < need)
    return fail_call(BGMF_E_BUDGET, "%s: the workspace has %lld bytes, %lld are needed", call,
                     (long long)ws_bytes, (long long)need);
  const Split split = split_of(rows, cols);
  p.parts = split.parts, p.part_len = split.len;
  p.part_sum = static_cast<PartSum *>(ws);
  if (grad_scores && cols && !row_state)
    p.state = reinterpret_cast<float *>(
        static_cast<char *>(ws) +
        (split.parts == 1 ? 0 : padded(rows * split.parts * (int64_t)sizeof(PartSum))));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = type == BGMF_TYPE_F32    ? policy<float>(p, stream)
                       : type == BGMF_TYPE_BF16 ? policy<bf16_t>(p, stream)
                                                : policy<f16_t>(p, stream);
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

int bgmf_policy_loss_grad(const void *scores, int32_t type, int64_t rows, int64_t cols,
                          int64_t row_stride, const void *reference, int64_t reference_stride,
                          const uint8_t *excluded, int64_t excluded_stride, const int32_t *given,
                          float temperature, float kl_weight, const float *row_state,
                          const float *grad_loss, void *grad_scores, int64_t grad_stride,
                          void *hip_stream) {
  const char *call = "bgmf_policy_loss_grad";
  Policy p{};
  p.x = scores, p.y = reference, p.ex = excluded, p.given = given;
  p.rows = rows, p.cols = cols, p.stride = row_stride, p.y_stride = reference_stride;
  p.ex_stride = excluded_stride, p.temperature = temperature, p.kl_weight = kl_weight;
  p.state = const_cast<float *>(row_state), p.g_loss = grad_loss;
  p.out = grad_scores, p.out_stride = grad_stride;
  if (const int rc = check_policy(call, p, type, true)) return rc;
  if (rows == 0 || cols == 0) return BGMF_OK;
  if (!row_state) return fail_call(BGMF_E_ARG, "%s: null row_state", call);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (type == BGMF_TYPE_F32) policy_grad<float>(p, stream);
  else if (type == BGMF_TYPE_BF16) policy_grad<bf16_t>(p, stream);
  else policy_grad<f16_t>(p, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail_call(BGMF_E_HIP, "%s: %s", call, hipGetErrorString(e));
  return BGMF_OK;
}

}  // extern "C"
