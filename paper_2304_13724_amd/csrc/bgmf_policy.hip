// The clipped policy loss of shown items with a divergence from a reference
// (bgmf_policy_loss) and its gradient (bgmf_policy_loss_grad).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bgmf_rank.h"

namespace bgmfk {
namespace {

// Threads of a workgroup (where it is not TH).
constexpr int kThreads = 256;

struct Policy {
  const void *x, *y;  // scores, and the reference's or null
  const uint8_t *ex;
  const int32_t *given;
  const float *advantage, *old_log_prob, *ref_log_prob;
  int64_t rows, cols, stride, y_stride, ex_stride;
  float temperature, clip_low, clip_high, kl_weight;
  float *loss, *log_prob, *kl;
  int64_t first;  // a launch's first row (or part): workgroups have one each
  float *state;  // [5][rows]: row_max, row_sum, the reference's row_max, slope, mean
  // rows split in `parts` of part_len scores: where the parts' sums go
  int64_t parts, part_len;
  struct PartSum *part_sum;  // [rows][parts]
  // the gradient
  const float *g_loss;
  void *out;
  int64_t out_stride, tiles;  // tiles of a row
};

// a b, but 0 where either is 0, whatever the other is (v_mul_legacy_f32; the
// compiler has no builtin for it).
extern "C" __device__ float bgmf_mul_legacy(float a, float b) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float times_or_0(float a, float b) { return bgmf_mul_legacy(a, b); }

// exp(x) - 1 and exp(x) to 6e-10 of themselves, by the series of exp over [-ln 2 /
// 2, ln 2 / 2] to the eighth power and a power of two; ln S, to as much, from a
// 32-bit logarithm y and what S exp(-y) is off from 1 (below 1e-5, so that two
// terms of the series of ln(1 + d) do).  The library's functions would take twice
// the registers of everything else in these kernels.
struct Exp {
  double less1, value;
  __device__ __forceinline__ explicit Exp(double x) {
    const double most = x > 1000.0 ? 1000.0 : x < -1100.0 ? -1100.0 : x;  // NaN stays
    const double k = rint(most * 1.4426950408889634074);
    double r = fma(-k, 0x1.62e42fefa39efp-1, most);
    r = fma(-k, 0x1.abc9e3b39803fp-56, r);
    double p = 1.0 / 40320.0;
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p * r, r, r);
    const int e = (int)k;  // (0 for a NaN, whose r is NaN)
    value = ldexp(1.0 + p, e);
    less1 = e == 0 ? p : value - 1.0;
  }
};
__device__ __forceinline__ double ln(double s) {  // s > 0, in the range of 32 bits, or NaN
  const double y = (double)__builtin_amdgcn_logf((float)s) * kLn2;
  const double d = s * Exp(-y).value - 1.0;
  return y + fma(-0.5 * d, d, d);
}

// Running sums of a row's scores x and of the reference's y, m and my the
// largest of each so far, d = (x - m) c and dy = (y - my) c:
//   s = sum exp2(d)   sy = sum exp2(dy)   w = sum exp2(d) (d - dy)
// from which ln s, ln sy and the mean w / s of d - dy under p give
//   sum p ln(p / q) = (w / s) ln 2 - ln s + ln sy.
// Both differences are taken from their own maximum, so an offset between the
// two policies' scores costs nothing, and one item alone gives exactly 0.  The
// divergence is a small difference of large terms: a group's are summed in fp32 and
// added to running sums in fp64, and in place of sy goes the sum of exp2(dy) -
// exp2(d), beside which the rounding of s cancels (with sy itself the divergence
// was four times as far off as by its terms' own roundings, 2e-6 of itself over 16
// items).  A score of -inf adds nothing; a NaN or +inf makes s (or sy) NaN.
template <bool REF>
struct Sums {
  float m = -INFINITY, my = -INFINITY;
  double s = 0.0, w = 0.0, sy = 0.0;
  static __device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
  // To the maxima M >= m and My >= my, by factors in 64 bits: each part has its own, and
  // their roundings would not cancel in the divergence as those of a row's terms do
  // (with factors in fp32 it was 1.9e-8 off over 18,433 items, where it is 0.04, and 7e-9
  // over 625,001, now 3e-9 and 2e-10; 33 rows of 123 parts 4.8 us with either).
  __device__ __forceinline__ void rescale(float M, float My, float c) {
    if (m != -INFINITY) {  // (otherwise s and w are 0, or NaN from a NaN)
      const double down = (double)m - M, f = exp2(down * c);
      if constexpr (REF)  // (the differences first: equal scores leave exactly 0)
        w = (w + s * ((down + ((double)base_of(My) - base_of(my))) * c)) * f;
      s *= f;
    }
    if constexpr (REF)
      if (my != -INFINITY) sy *= exp2(((double)my - My) * c);
    m = M, my = My;
  }
  // A group's sums, with m and my not below its scores.
  struct Group {
    float s = 0.0f, w = 0.0f, sy = 0.0f;
    template <int COUNT>
    __device__ __forceinline__ void add(const float (&x)[COUNT], const float (&y)[COUNT], float bx,
                                        float by, float c) {
      // d and dy are rounded alike, so that equal scores leave exactly 0
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < COUNT; ++i) {
        const float d = (x[i] - bx) * c, e = __builtin_amdgcn_exp2f(d);
        s += e;
        if constexpr (REF) {
          const float dy = (y[i] - by) * c;
          sy += __builtin_amdgcn_exp2f(dy) - e;
          w += times_or_0(e, d - dy);  // (e may be 0 where d - dy is not finite)
        }
      }
    }
  };
  __device__ __forceinline__ void add(const Group &g) {
    s += g.s;
    if constexpr (REF) w += g.w, sy += g.sy;
  }
};

// What the gradient needs of a row: with d and dy as above,
//   dx_j = g / t (slope (1[j = given] - p_j) + kl_weight p_j ln 2 (d_j - dy_j - mean))
struct State {
  float m, s, my, slope, mean;  // s = 0: the row's gradient is 0
};

// What a row's results need of its given item, fetched before its sums are there.
// Every thread of the row has the same.
template <class T, bool REF>
struct Given {
  int64_t item;
  bool inside, excluded;
  float x = 0.0f, y = 0.0f, advantage, old_log_prob, ref_log_prob = 0.0f;
  __device__ __forceinline__ Given(const Policy &P, int64_t r) {
    item = P.given[r];
    inside = item >= 0 && item < P.cols;
    excluded = inside && P.ex && P.ex[r * P.ex_stride + item];
    if (inside) {
      x = to_float(static_cast<const T *>(P.x)[r * P.stride + item]);
      if constexpr (REF) y = to_float(static_cast<const T *>(P.y)[r * P.y_stride + item]);
    }
    advantage = P.advantage[r], old_log_prob = P.old_log_prob[r];
    if (P.ref_log_prob) ref_log_prob = P.ref_log_prob[r];
    x = scalar(x), y = scalar(y), advantage = scalar(advantage);
    old_log_prob = scalar(old_log_prob), ref_log_prob = scalar(ref_log_prob);
    excluded = __builtin_amdgcn_readfirstlane(excluded);
  }
  static __device__ __forceinline__ float scalar(float v) {  // out of the vector registers
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
  }
};

// The row's results, by one thread, in 64 bits.
template <class T, bool REF>
__device__ __forceinline__ State finish(const Policy &P, int64_t r, const Given<T, REF> &g,
                                        const Sums<REF> &a) {
  State st{a.m, (float)a.s, a.my, 0.0f, 0.0f};
  double loss = 0.0, lp = 0.0, kl = 0.0;
  if (g.item == -1) {
    st.s = 0.0f;
  } else {
    const bool none = a.s == 0.0;
    const double ln_s = none ? 0.0 : ln(a.s);
    lp = -INFINITY;
    if (!g.inside) lp = NAN;
    else if (!none && !g.excluded)
      lp = ((double)g.x - (double)a.m) / (double)P.temperature - ln_s;
    if (!none || !g.inside) {
      const double A = g.advantage, rho = Exp(lp - (double)g.old_log_prob).value;
      const double lo = 1.0 - (double)P.clip_low, hi = 1.0 + (double)P.clip_high;
      const double unclipped = rho * A, clipped = (rho < lo ? lo : rho > hi ? hi : rho) * A;
      const bool passes = !(unclipped > clipped);
      loss = -(passes ? unclipped : clipped);
      double slope = passes ? -unclipped : 0.0;
      if (P.ref_log_prob) {
        const double z = (double)g.ref_log_prob - lp, e = Exp(z).less1;
        kl = z == INFINITY ? INFINITY : e - z;
        if (P.kl_weight != 0.0f) slope -= (double)P.kl_weight * e;
      }
      st.slope = (float)slope;
    }
    if constexpr (REF) {
      if (!none) {
        const double mean = a.w / a.s;
        kl = a.sy == 0.0 ? INFINITY : mean * kLn2 - ln_s + ln(a.sy);
        // (a NaN or +inf in the reference shows in sy alone where p is 0)
        st.mean = isnan(kl) ? NAN : (float)mean;
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

// A part's sums.  w is that of the items whose reference is not 0, so that it can be
// rescaled; none: the largest score of the others (-inf: there are none), by which
// the row decides whether they count.
struct PartSum {
  double s, w, sy;
  float m, my, none;
};

// A row's gradient but for its given item's own term: with d, dy and e = exp2(d),
//   p (gk (d - dy - mean) - gs) = e (slope (d - dy) + level)
// and 0 for items of probability 0, excluded ones among them.  In an odd row every
// item that is not excluded has the same: 0 where the row takes no part, NaN where
// its level is.
template <bool REF>
struct Slopes {
  float c, m, my, slope, level, gs;  // slope 0: the reference plays no part
  bool odd;
  __device__ __forceinline__ Slopes(const Policy &P, int64_t r, const State &st) {
    c = kLog2e / P.temperature;
    const float w = P.g_loss ? P.g_loss[r] : 1.0f, g = w / P.temperature, inv = 1.0f / st.s;
    m = st.m, my = Sums<REF>::base_of(st.my);
    const bool none = st.s == 0.0f || w == 0.0f;
    gs = none ? 0.0f : g * st.slope;
    const bool flat = !REF || P.kl_weight == 0.0f;
    slope = flat ? 0.0f : g * P.kl_weight * (float)kLn2;
    level = none ? 0.0f : -(flat ? gs : fmaf(slope, st.mean, gs)) * inv;
    slope *= inv;
    odd = none || isnan(level);
  }
  __device__ __forceinline__ float operator()(float x, float y) const {
    // (contracted, d - dy would not be 0 for equal scores)
#pragma clang fp contract(off)
    const float d = (x - m) * c, e = __builtin_amdgcn_exp2f(d);
    float v = level;
    if constexpr (REF) {
      const float dy = (y - my) * c;
      v = times_or_0(slope, d - dy) + level;
    }
    return times_or_0(e, v);
  }
};

// Scores as a row's vectors hold them, those of excluded items -inf in both.
template <class T, bool EX, bool REF>
struct Pair {
  static constexpr int N = Vec<T>::N;
  Row<T, EX> row;
  const T *y;
  // Vectors as they are in memory, in 32-bit words (held as 16-bit values, each
  // would take a register of its own).
  struct Raw {
    uint32_t x[4], y[REF ? 4 : 1], ex[EX ? N / 4 : 1];
  };
  static constexpr uint32_t kLow = sizeof(T) == 4 ? 0xFF800000u
                                   : std::is_same<T, bf16_t>::value ? 0xFF80FF80u
                                                                    : 0xFC00FC00u;  // -inf
  __device__ __forceinline__ Raw fetch(int32_t v) const {
    Raw r;
    __builtin_memcpy(r.x, row.x + (int64_t)v * N, 16);
    if constexpr (REF) __builtin_memcpy(r.y, y + (int64_t)v * N, 16);
    if constexpr (EX) __builtin_memcpy(r.ex, row.ex + (int64_t)v * N, N);
    return r;
  }
  // Once fetched: -inf in place of excluded scores, by words.
  static __device__ __forceinline__ void exclude(Raw &r) {
    if constexpr (EX) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t b = r.ex[k * (N / 4) / 4];
        const uint32_t some = ((b & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | b;  // bit 7 of each byte
        uint32_t mask;
        if constexpr (N == 4)
          mask = (uint32_t)((int32_t)(some << (24 - 8 * k)) >> 31);
        else  // (8 to 11 repeat bits 15, 31, 47 and 63 of both words)
          mask = __builtin_amdgcn_perm(some << 8, some, k % 2 ? 0x09090B0Bu : 0x08080A0Au);
        r.x[k] = (mask & kLow) | (~mask & r.x[k]);
        if constexpr (REF) r.y[k] = (mask & kLow) | (~mask & r.y[k]);
      }
      renew(r);  // (the compiler would mask each element by itself)
    }
  }
  static __device__ __forceinline__ float element(const uint32_t *w, int i) {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(w[i]);
    } else if constexpr (std::is_same<T, bf16_t>::value) {
      return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    } else {
      return to_float(__builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (i % 2 * 16))));
    }
  }
  __device__ __forceinline__ float other(int32_t i) const {  // as row.one(i)
    if constexpr (!REF) return -INFINITY;
    if constexpr (EX)
      if (row.ex[i]) return -INFINITY;
    return to_float(y[i]);
  }
  // Between two passes over the same vectors: what the first made of them is not
  // kept (the scores take two or three times the registers of the vectors).
  static __device__ __forceinline__ void renew(Raw &r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      asm volatile("" : "+v"(r.x[i]));
      if constexpr (REF) asm volatile("" : "+v"(r.y[i]));
    }
  }
  static __device__ __forceinline__ void scores(const Raw &r, float (&x)[N], float (&z)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = element(r.x, i);
      z[i] = REF ? element(r.y, i) : -INFINITY;
    }
  }
  // The gradient of vector v, and of one element.
  __device__ __forceinline__ Vec<T> gradient(int32_t v, const Raw &r,
                                             const Slopes<REF> &grad) const {
    Vec<T> to;
    if (grad.odd) {
      for (int i = 0; i < N; ++i) to.v[i] = gradient(v * N + i, grad);
      return to;
    }
    float x[N], z[N];
    scores(r, x, z);
#pragma unroll
    for (int i = 0; i < N; ++i) to.v[i] = from_float<T>(grad(x[i], z[i]));
    return to;
  }
  __device__ __forceinline__ T gradient(int32_t i, const Slopes<REF> &grad) const {
    if (grad.odd) return from_float<T>(EX && row.ex[i] ? 0.0f : grad.level);
    return from_float<T>(grad(row.one(i), other(i)));
  }
};

// Joins the parts of a row, in a fixed order: one workgroup per row, a part to a
// thread: the maxima, then the sums brought to them.  Bound: latency (33 rows of 123
// parts: 4.8 us).
template <class T, bool REF>
__global__ void __launch_bounds__(kThreads) k_policy_join(Policy P) {
  constexpr int W = kThreads / 64;
  __shared__ float s_m[W], s_my[W], s_none[W];
  __shared__ double s_s[W], s_w[W], s_sy[W];
  const float c = kLog2e / P.temperature;
  const int tid = threadIdx.x, wave = tid / 64;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x) {
    const PartSum *sums = P.part_sum + r * P.parts;
    const Given<T, REF> given(P, r);
    const PartSum first = tid < P.parts ? sums[tid]
                                        : PartSum{0.0, 0.0, 0.0, -INFINITY, -INFINITY, -INFINITY};
    Sums<REF> a;
    a.m = first.m, a.my = first.my;
    float none = first.none;
    for (int64_t i = tid + kThreads; i < P.parts; i += kThreads) {
      a.m = fmaxf(a.m, sums[i].m);
      if constexpr (REF) a.my = fmaxf(a.my, sums[i].my), none = fmaxf(none, sums[i].none);
    }
    a.m = wave_max(a.m);
    if constexpr (REF) a.my = wave_max(a.my), none = wave_max(none);
    if (tid % 64 == 0) s_m[wave] = a.m, s_my[wave] = a.my, s_none[wave] = none;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a.m = fmaxf(a.m, s_m[i]);
      if constexpr (REF) a.my = fmaxf(a.my, s_my[i]), none = fmaxf(none, s_none[i]);
    }
    const auto add = [&](const PartSum &p) {
      Sums<REF> b;
      b.m = p.m, b.s = p.s;
      if constexpr (REF) b.my = p.my, b.w = p.w, b.sy = p.sy;
      b.rescale(a.m, a.my, c);
      a.s += b.s;
      if constexpr (REF) a.w += b.w, a.sy += b.sy;
    };
    add(first);
    for (int64_t i = tid + kThreads; i < P.parts; i += kThreads) add(sums[i]);
    a.s = wave_sum(a.s);
    if constexpr (REF) a.w = wave_sum(a.w), a.sy = wave_sum(a.sy);
    if (tid % 64 == 0) s_s[wave] = a.s, s_w[wave] = a.w, s_sy[wave] = a.sy;
    __syncthreads();
    a.s = a.w = a.sy = 0.0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a.s += s_s[i];
      if constexpr (REF) a.w += s_w[i], a.sy += s_sy[i];
    }
    if constexpr (REF)  // p > 0 = q, by the exponential that a row held in registers has
      if (__builtin_amdgcn_exp2f((none - Sums<REF>::base_of(a.m)) * c) > 0.0f) a.w = INFINITY;
    if (tid == 0) finish(P, r, given, a);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient: the scores and the reference are read and the gradient is written
// once.  A workgroup takes a tile of one row at a time.  Bound: HBM: 33 x 625,001 f32
// with a reference take 37 us, 6.6 TB/s (the Infinity Cache has some of what the
// forward pass read).
// ---------------------------------------------------------------------------

// The given item's gradient.
template <class T, bool REF>
__device__ __forceinline__ T given_gradient(float x, float y, bool excluded,
                                            const Slopes<REF> &grad) {
  const float v = grad.odd ? grad.level : grad(x, y) + grad.gs;
  return from_float<T>(excluded ? 0.0f : v);
}

constexpr int kGradGroup = 2;
template <class T, bool EX, bool REF, int TH>
__global__ void __launch_bounds__(TH) k_policy_grad(Policy P) {
  using Two = Pair<T, EX, REF>;
  constexpr int N = Vec<T>::N;
  constexpr int64_t kTile = (int64_t)TH * kGradGroup * N;
  const int tid = threadIdx.x;
  for (int64_t u = blockIdx.x; u < P.rows * P.tiles; u += gridDim.x) {
    const int64_t r = u / P.tiles, first = u % P.tiles * kTile, left = P.cols - first;
    const int32_t len = (int32_t)(left < kTile ? left : kTile);
    const Two two{{static_cast<const T *>(P.x) + (r * P.stride + first),
                   EX ? P.ex + (r * P.ex_stride + first) : nullptr, len},
                  REF ? static_cast<const T *>(P.y) + (r * P.y_stride + first) : nullptr};
    T *out = static_cast<T *>(P.out) + (r * P.out_stride + first);
    typename Two::Raw raw[kGradGroup];
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q)
      if ((tid + q * TH) * N + N <= len) raw[q] = two.fetch(tid + q * TH);
    const State st{P.state[r], P.state[P.rows + r], P.state[2 * P.rows + r],
                   P.state[3 * P.rows + r], P.state[4 * P.rows + r]};
    const Slopes<REF> grad(P, r, st);
    // the thread whose vector has the given item writes it once more
    const int64_t g = P.given[r] - first;
    const bool own = g >= 0 && g < len && g / N % TH == tid;
    T given;
    if (own)
      given = given_gradient<T>(to_float(two.row.x[g]), REF ? to_float(two.y[g]) : 0.0f,
                                EX && two.row.ex[g], grad);
#pragma unroll
    for (int q = 0; q < kGradGroup; ++q) {
      const int32_t i = (tid + q * TH) * N;
      if (i + N <= len) {
        Two::exclude(raw[q]);
        store_vec(out + i, two.gradient(tid + q * TH, raw[q], grad));
      } else {
        for (int k = 0; k < N; ++k)
          if (i + k < len) out[i + k] = two.gradient(i + k, grad);
      }
    }
    if (own) out[g] = given;
  }
}

// ---------------------------------------------------------------------------
// Rows that fit the registers of a workgroup (H vectors a thread), with their
// gradient or without, or (PART) parts of a row, whose sums are joined: the scores and
// the reference are read and the gradient is written once, all of a row on its way
// at the same time.  Three passes over the registers: the maxima, the sums with them, the
// gradient.  A workgroup has one row and no loop over rows (the compiler would keep the
// 64-bit functions' constants in registers through it).  Bound: 2,047 x 18,000 bf16
// with a reference, exclusions and the gradient take 55 us: HBM, 4.7 TB/s, and the vector
// units (87% of the CUs' cycles, 39 instructions a score, three exponentials among
// them); 4,001 x 10,007 f32 with a reference alone 55 us, 5.8 TB/s; 16 x 18,000 f32 6.0
// us: latency (a row's loads, three reductions, the 64-bit functions of one thread).
// ---------------------------------------------------------------------------
template <int TH>
struct StepLds {
  float m[TH / 64], my[TH / 64];
  double s[TH / 64], w[TH / 64], sy[TH / 64];
  State st;
};
template <class T, bool EX, bool REF, bool PART, int TH, int H>
__global__ void __launch_bounds__(TH, TH > 512 || H > 5 ? 4 : 5) k_policy_step(Policy P) {
  __shared__ StepLds<TH> lds;
  using Two = Pair<T, EX, REF>;
  constexpr int N = Two::N, W = TH / 64;
  const int tid = threadIdx.x, wave = tid / 64;
  const float c = kLog2e / P.temperature;
  const int64_t u = P.first + blockIdx.x, r = PART ? u / P.parts : u;
  const int64_t first = PART ? u % P.parts * P.part_len : 0, left = P.cols - first;
  const int32_t len = (int32_t)(PART && left > P.part_len ? P.part_len : left), vecs = len / N;
  T *out = static_cast<T *>(P.out) + r * P.out_stride;
  const Two two{{static_cast<const T *>(P.x) + (r * P.stride + first),
                 EX ? P.ex + (r * P.ex_stride + first) : nullptr, len},
                REF ? static_cast<const T *>(P.y) + (r * P.y_stride + first) : nullptr};
  const bool tail = tid < len - vecs * N;
  Sums<REF> a;
  typename Two::Raw raw[H];
  float x1 = -INFINITY, y1 = -INFINITY;
#pragma unroll
  for (int h = 0; h < H; ++h)
    if (h * TH + tid < vecs) raw[h] = two.fetch(h * TH + tid);
  if (tail) x1 = two.row.one(vecs * N + tid), y1 = two.other(vecs * N + tid);
  std::conditional_t<PART, int, Given<T, REF>> given = [&] {
    if constexpr (PART) return 0;
    else return Given<T, REF>(P, r);
  }();
  const int64_t g = P.given[r];
  if (g != -1) {  // of all threads
    // the largest
    a.m = x1, a.my = y1;
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (h * TH + tid < vecs) {
        float x[N], y[N];
        Two::exclude(raw[h]);
        Two::scores(raw[h], x, y);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          a.m = fmaxf(a.m, x[i]);
          if constexpr (REF) a.my = fmaxf(a.my, y[i]);
        }
      }
    a.m = wave_max(a.m);
    if constexpr (REF) a.my = wave_max(a.my);
    if constexpr (W > 1) {
      if (tid % 64 == 0) lds.m[wave] = a.m, lds.my[wave] = a.my;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) {
        a.m = fmaxf(a.m, lds.m[i]);
        if constexpr (REF) a.my = fmaxf(a.my, lds.my[i]);
      }
    }
    // the sums, of 16 scores in 32 bits
    const float bx = Sums<REF>::base_of(a.m), by = Sums<REF>::base_of(a.my);
    typename Sums<REF>::Group group;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if (h * TH + tid < vecs) {
        float x[N], y[N];
        Two::renew(raw[h]);
        Two::scores(raw[h], x, y);
        group.add(x, y, bx, by, c);
      }
      if ((h + 1) * N % 16 == 0 || h == H - 1) {
        a.add(group);
        group = {};
      }
    }
    if (tail) {
      const float x[1] = {x1}, y[1] = {y1};
      group.add(x, y, bx, by, c);
      a.add(group);
    }
    a.s = wave_sum(a.s);
    if constexpr (REF) a.w = wave_sum(a.w), a.sy = wave_sum(a.sy);
    if constexpr (W > 1) {
      if (tid % 64 == 0) lds.s[wave] = a.s, lds.w[wave] = a.w, lds.sy[wave] = a.sy;
      __syncthreads();
      a.s = a.w = a.sy = 0.0;
      for (int i = 0; i < W; ++i) {
        a.s += lds.s[i];
        if constexpr (REF) a.w += lds.w[i], a.sy += lds.sy[i];
      }
    }
    if constexpr (REF) {
      // sy from the sum of differences, whose rounding the divergence does not
      // magnify; where the two policies are so far apart that it would be lost
      // beside s, by itself
      if (fabs(a.sy) <= 0.5 * a.s) {
        a.sy += a.s;
      } else {  // of all threads
        a.sy = 0.0;
#pragma unroll
        for (int h = 0; h < H; ++h)
          if (h * TH + tid < vecs) {
            float x[N], y[N], sum = 0.0f;
            Two::renew(raw[h]);
            Two::scores(raw[h], x, y);
#pragma unroll
            for (int i = 0; i < N; ++i) sum += __builtin_amdgcn_exp2f((y[i] - by) * c);
            a.sy += sum;
          }
        if (tail) a.sy += __builtin_amdgcn_exp2f((y1 - by) * c);
        a.sy = wave_sum(a.sy);
        if constexpr (W > 1) {
          __syncthreads();
          if (tid % 64 == 0) lds.sy[wave] = a.sy;
          __syncthreads();
          a.sy = 0.0;
          for (int i = 0; i < W; ++i) a.sy += lds.sy[i];
        }
      }
    }
  }
  if constexpr (PART) {
    float none = -INFINITY;
    if constexpr (REF) {
      if (isinf(a.w)) {  // of all threads: some item's reference is 0
        const float bx = Sums<REF>::base_of(a.m), by = Sums<REF>::base_of(a.my);
        a.w = 0.0;
        const auto add = [&](float x, float y) {
#pragma clang fp contract(off)
          const float d = (x - bx) * c, e = __builtin_amdgcn_exp2f(d);
          const float moved = d - (y - by) * c;
          if (moved == INFINITY) none = fmaxf(none, e > 0.0f ? x : -INFINITY);
          else a.w += times_or_0(e, moved);
        };
#pragma unroll
        for (int h = 0; h < H; ++h)
          if (h * TH + tid < vecs) {
            float x[N], y[N];
            Two::renew(raw[h]);
            Two::scores(raw[h], x, y);
#pragma unroll
            for (int i = 0; i < N; ++i) add(x[i], y[i]);
          }
        if (tail) add(x1, y1);
        a.w = wave_sum(a.w), none = wave_max(none);
        __syncthreads();
        if (tid % 64 == 0) lds.w[wave] = a.w, lds.m[wave] = none;
        __syncthreads();
        a.w = 0.0;
        for (int i = 0; i < W; ++i) a.w += lds.w[i], none = fmaxf(none, lds.m[i]);
      }
    }
    if (tid == 0) P.part_sum[u] = PartSum{a.s, a.w, a.sy, a.m, a.my, none};
  } else {
    if (tid == 0) lds.st = finish(P, r, given, a);
    if (!P.out) return;  // of all threads
    __syncthreads();
    const Slopes<REF> grad(P, r, lds.st);
    // the thread whose vector has the given item writes it once more
    const bool own = given.inside &&
                     (g / N < vecs ? (int)(g / N % TH) : (int)(g - vecs * N)) == tid;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int32_t v = h * TH + tid;
      if (v < vecs) {
        Two::renew(raw[h]);
        store_vec(out + (int64_t)v * N, two.gradient(v, raw[h], grad));
      }
    }
    if (tail) out[vecs * N + tid] = two.gradient(vecs * N + tid, grad);
    if (own) out[g] = given_gradient<T>(given.x, given.y, given.excluded, grad);
  }
}

constexpr int64_t kMostGroups = 1 << 20;

// Rows that no workgroup holds go in as few parts as one of 256 threads holds (kPart
// vectors), all as long, and a join.  Parts of 256 x 5, 256 x 9 and 512 x 5, with
// exclusions and a reference: f32 33 x 625,001 34.0, 34.5 and 33.9 us, 1 x 200,000 7.7,
// 8.7 and 8.7, 4,096 x 24,000 158, 162 and 159; bf16 128 x 200,000 27.7, 29.2 and 31.6.
// (Going through a longer part with running sums, next vectors on their way: 35.7,
// 9.8, 157 and 33.0.)
constexpr int64_t kPart = 5 * 256;
struct Split {
  int64_t parts, len;
};
Split split_of(int64_t cols, int64_t per) {  // per: scores of a vector
  const int64_t parts = (cols + kPart * per - 1) / (kPart * per);
  const int64_t len = ((cols + parts - 1) / parts + 63) / 64 * 64;
  return {(cols + len - 1) / len, len};
}
int64_t padded(int64_t x) { return (x + 255) / 256 * 256; }

// Rows of at most this many scores go to workgroups of one wave (as in log_probs,
// whose figures are at its constant).
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
void policy_grad(Policy p, hipStream_t stream) {
  with_flags(p.ex, p.y && p.kl_weight != 0.0f, [&](auto ex, auto ref) {
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

// Whether a workgroup holds a row.  With exclusions and a reference, the results and the
// gradient in one pass and in two: f32 4,096 x 18,000 182 and 299 us, 4,096 x 36,000 392
// and 577, 16 x 18,000 8.7 and 12.5, 1 x 36,000 12.4 and 12.3 (one workgroup has all of
// it); bf16 4,096 x 18,000 101 and 173.  The results alone, held and in parts: f32
// 4,096 x 18,000 111 and 122, 8 rows 7.0 and 8.2, 8 x 36,000 10.1 and 8.2; bf16 8 x
// 36,000 10.4 and 9.1, 512 rows 23.7 and 23.7.
constexpr int64_t kMostHeld = 9 * 1024, kMostHeldValue = 9 * 512;  // vectors
template <class T>
bool in_registers(const Policy &p) {
  return p.cols <= (p.out ? kMostHeld : kMostHeldValue) * Vec<T>::N;
}

template <class T>
hipError_t policy_step(Policy p, hipStream_t stream) {
  const int64_t vecs = p.cols / Vec<T>::N;
  with_flags(p.ex, p.y, [&](auto ex, auto ref) {
    constexpr bool EX = decltype(ex)::value, REF = decltype(ref)::value;
    const auto go = [&](auto threads, auto held) {
      constexpr int TH = decltype(threads)::value, H = decltype(held)::value;
      for (p.first = 0; p.first < p.rows; p.first += kMostGroups)
        hipLaunchKernelGGL((k_policy_step<T, EX, REF, false, TH, H>),
                           dim3((unsigned)std::min(p.rows - p.first, kMostGroups)), dim3(TH), 0,
                           stream, p);
    };
    using std::integral_constant;
    using Few = integral_constant<int, 5>;
    using Most = integral_constant<int, 9>;
    // the fewest threads that hold a row, but for few rows no more than five vectors
    // each.  With exclusions and a reference: bf16 4,096 x 2,000 by 64 x 4 and 256 x 5
    // 18.3 and 21.3 us, 16 x 2,000 5.8 and 4.8; 4,096 x 18,000 by 256 x 9 and 512 x 5 101
    // and 108, 256 x 18,000 10.8 and 10.4; f32 4,096 x 18,000 by 512 x 9 and 1,024 x 5
    // 182 and 213, 512 rows 21.5 and 27.9, 256 rows 14.4 and 14.4
    const bool many = p.rows >= 512;
    if (vecs <= 4 * 64) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (vecs <= 5 * 256) go(integral_constant<int, 256>{}, Few{});
    else if (many && vecs <= 9 * 256) go(integral_constant<int, 256>{}, Most{});
    else if (vecs <= 5 * 512) go(integral_constant<int, 512>{}, Few{});
    else if (many && vecs <= 9 * 512) go(integral_constant<int, 512>{}, Most{});
    else if (vecs <= 5 * 1024) go(integral_constant<int, 1024>{}, Few{});
    else go(integral_constant<int, 1024>{}, Most{});
  });
  return hipGetLastError();
}

template <class T>
hipError_t policy(Policy p, hipStream_t stream) {
  if (in_registers<T>(p)) return policy_step<T>(p, stream);
  const Split split = split_of(p.cols, Vec<T>::N);
  p.parts = split.parts, p.part_len = split.len;
  with_flags(p.ex, p.y, [&](auto ex, auto ref) {
    constexpr bool EX = decltype(ex)::value, REF = decltype(ref)::value;
    const int64_t units = p.rows * p.parts;
    for (p.first = 0; p.first < units; p.first += kMostGroups)
      hipLaunchKernelGGL((k_policy_step<T, EX, REF, true, 256, 5>),
                         dim3((unsigned)std::min(units - p.first, kMostGroups)), dim3(256), 0,
                         stream, p);
    hipLaunchKernelGGL((k_policy_join<T, REF>), dim3((unsigned)std::min(p.rows, kMostGroups)),
                       dim3(kThreads), 0, stream, p);
  });
  if (p.out) policy_grad<T>(p, stream);
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

// Workspace: row_state where the caller wants none, then the parts' sums, of the
// type whose rows have most.
int64_t bgmf_policy_loss_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= kMostHeldValue * 4 || rows >= (1ll << 31) || cols >= (1ll << 31))
    return 0;
  return padded(5 * rows * (int64_t)sizeof(float)) +
         rows * split_of(cols, 4).parts * (int64_t)sizeof(PartSum);
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
  if (need) {
    if (grad_scores && !row_state) p.state = static_cast<float *>(ws);
    p.part_sum = reinterpret_cast<PartSum *>(static_cast<char *>(ws) +
                                             padded(5 * rows * (int64_t)sizeof(float)));
  }
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
