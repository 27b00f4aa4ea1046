// Log probability and rank of a given class, log normaliser, entropy and the
// best classes of every row of scores (sb_log_probs).
//
// With m = max_j a_j, c2 = log2(e) / T, y_j = (a_j - m) c2, e_j = 2^y_j,
// s = sum e_j, t = sum e_j y_j:
//   lse = m / T + log s,  log p_y = (a_y - m) / T - log s,
//   entropy = log s - ln 2 t / s
// (log s >= 0 >= t, so the entropy has no cancellation).
//
// k_cols_by_lane, k_rows_by_lane: one lane per row, the columns in order, 16 at a
//   time: a running maximum, the two sums rescaled when it grows, and the best classes
//   so far as a sorted list in registers; a score enters it if it is above the last one
//   (equal scores stay behind the earlier class).  Column-major scores are read as runs
//   of a column; where there are few rows the columns are split over waves, and k_join
//   joins the partial statistics and lists.  Row-major ones go through an LDS tile of
//   128 bytes of 64 rows, unsplit.
// k_row_in_block (row-major): a row in the registers of a wave or of a block.  The
//   k-th largest of the threads' maxima bounds the k-th largest score from below; the
//   scores not under it, seldom many more than k, are collected in LDS and ranked
//   there by counting.
//
// Every score is read from memory once.  Its exponential takes 4 issue slots and the
// rest 7 to 10, about what its bytes take; lists and joins come on top, so that vector
// instructions bound all of these.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <cfloat>
#include <cmath>
#include <type_traits>

#include "sb_common.h"

namespace sb {
namespace {

constexpr float LN2 = 0.693147180559945309f;

struct LogProbArgs {
  const void* F;
  int64_t n;
  int32_t d;
  int64_t ld;
  float c, c2;  // 1 / T, log2(e) / T
  const int32_t* labels;
  float* logp;
  int32_t* rank;
  float* lse;
  float* entropy;
  int32_t k;
  int32_t* top_id;
  float* top_logp;
  int64_t ld_top;
  int tiles;        // of 64 rows: k_cols_by_lane, k_rows_by_lane
  int splits, per;  // k_cols_by_lane: column splits, columns per split
  double* part;     // splits > 1: [split][2 + k][n]: (m, s), (t, before), the list
};

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(__half x) { return __half2float(x); }
__device__ inline float to_f32(__hip_bfloat16 x) { return __bfloat162float(x); }
// The scores in 16 bytes, and 16 bytes of excluded ones.  The compiler sees the bytes
// anew: it would otherwise widen once and keep both forms.  fp16 ones are compared as
// they are, and widened by the instruction that scales them.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T>
using Score = std::conditional_t<std::is_same_v<T, __half>, _Float16, float>;
template <typename T>
__device__ inline void decode(u32x4& raw, Score<T> (&x)[16 / sizeof(T)]) {
  asm volatile("" : "+v"(raw));
  if constexpr (std::is_same_v<T, __half>) {
    __builtin_memcpy(x, &raw, 16);
  } else {
    T e[16 / sizeof(T)];
    __builtin_memcpy(e, &raw, 16);
#pragma unroll
    for (int u = 0; u < (int)(16 / sizeof(T)); ++u) x[u] = to_f32(e[u]);
  }
}
// The maxima (of numbers) of their first and second halves.  As it stands: the compiler
// would round bf16 maxima to bf16 again.
__device__ inline void halves_max(const u32x4& raw, const _Float16 (&)[8], float (&m)[2]) {
  uint32_t p[2];
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(p[0]) : "v"(raw.x), "v"(raw.y));
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(p[1]) : "v"(raw.z), "v"(raw.w));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    _Float16 h[2];
    __builtin_memcpy(h, &p[i], 4);
    const float x = (float)h[0], y = (float)h[1];
    asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m[i]) : "v"(x), "v"(y));
  }
}
template <int N>
__device__ inline void halves_max(const u32x4&, const float (&x)[N], float (&m)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int u = i * N / 2; u < (i + 1) * N / 2; u += 2)
      asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m[i]) : "v"(x[u]), "v"(x[u + 1]));
}
__device__ inline float max_of(const u32x4& raw, const _Float16 (&)[8]) {
  uint32_t a, b;
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(a) : "v"(raw.x), "v"(raw.y));
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(b) : "v"(raw.z), "v"(raw.w));
  asm("v_pk_max_f16 %0, %0, %1" : "+v"(a) : "v"(b));
  _Float16 h[2];
  __builtin_memcpy(h, &a, 4);
  return fmaxf((float)h[0], (float)h[1]);
}
template <int N>
__device__ inline float max_of(const u32x4&, const float (&x)[N]) {
  float m = x[N - 1];
#pragma unroll
  for (int u = 0; u + 1 < N; u += 2) {
    if (u + 2 < N) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m) : "v"(x[u]), "v"(x[u + 1]));
    else asm("v_max_f32 %0, %0, %1" : "+v"(m) : "v"(x[u]));
  }
  return m;
}
__device__ inline uint32_t excluded(float) { return 0xff800000u; }
__device__ inline uint32_t excluded(__half) { return 0xfc00fc00u; }
__device__ inline uint32_t excluded(__hip_bfloat16) { return 0xff80ff80u; }

__device__ inline void wave_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// Reductions over the lanes of a wave, in registers; every lane gets the result.
// Within rows of 16 the partner differs in one lane bit (quad permutations, mirrors of
// half rows and rows), then rows and halves of the wave meet by permlane swaps.
template <int CTRL>
__device__ inline uint32_t dpp_u32(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
template <typename Op>
__device__ inline uint32_t wave_all(uint32_t x, Op op) {
  x = op(x, dpp_u32<0xb1>(x));   // quad_perm [1, 0, 3, 2]
  x = op(x, dpp_u32<0x4e>(x));   // quad_perm [2, 3, 0, 1]
  x = op(x, dpp_u32<0x141>(x));  // row_half_mirror
  x = op(x, dpp_u32<0x140>(x));  // row_mirror
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op(r[0], r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op(h[0], h[1]);
}
__device__ inline float wave_sum(float x) {
  return __uint_as_float(wave_all(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ inline float wave_max(float x) {
  return __uint_as_float(wave_all(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ inline int wave_sum(int x) {
  return (int)wave_all((uint32_t)x, [](uint32_t a, uint32_t b) { return a + b; });
}

// The row's real outputs from its statistics.  m starts at -FLT_MAX, so that a row of
// -inf has s = 0 and no differences of infinities.
struct RowStats {
  float m, s, t;
  float r;  // s and t are those of y_j + r (see rows_in_block); 0 elsewhere
  // in powers of 2 by the hardware's logarithm: s is near 1 or above, or 0
  __device__ float log2_s() const { return __builtin_amdgcn_logf(s); }
  __device__ float log_s(float l2) const { return LN2 * (l2 - r); }
  __device__ float entropy(float l2) const { return LN2 * (l2 - t * __builtin_amdgcn_rcpf(s)); }
};
// ls: log s; h: the entropy
__device__ inline void store_row(const LogProbArgs& a, int64_t row, const RowStats& r, float ls, float h, int y, float ay,
                                 int before) {
  const bool none = r.s == 0.0f;
  const bool has = y >= 0 && y < a.d;
  if (a.lse) a.lse[row] = none ? -INFINITY : fmaf(r.m, a.c, ls);
  if (a.entropy) a.entropy[row] = none || h < 0.0f ? 0.0f : h;
  if (a.logp) a.logp[row] = !has ? 0.0f : none ? -INFINITY : (ay - r.m) * a.c - ls;
  if (a.rank) a.rank[row] = has ? min(before, a.d - 1) : -1;  // a NaN compares with no score
}
__device__ inline void store_top(const LogProbArgs& a, int64_t row, int place, float v, int id, const RowStats& r,
                                 float ls) {
  a.top_id[place * a.ld_top + row] = id;
  a.top_logp[place * a.ld_top + row] = id < 0 ? -INFINITY : (v - r.m) * a.c - ls;
}

// ---------------------------------------------------------------- one lane per row
constexpr int CH = 16;         // columns per step
constexpr int TILE_B = 144;    // bytes of a row's 128 in the LDS tile: lanes' 16-byte reads fall on different banks

// A place of a lane's list as one double: the score, exact in the upper 23 bits of the
// mantissa, and in the lower ones the class, so that of two equal scores the smaller
// class is the larger double.  Minima and maxima of doubles then move score and class
// together, at the rate of 32-bit ones.  Both zeros are +0 here, whose doubles are
// subnormal; no double of a class rounds to another score.  (+inf, which has no room
// for a class, counts as the largest finite score.)
__device__ inline double place_of(float x, int j) {
  const double v = (double)(__builtin_amdgcn_fmed3f(x, -FLT_MAX, FLT_MAX) + 0.0f);
  const uint32_t low = __double2loint(v) | (x < 0.0f ? (uint32_t)j : 0xffffu - (uint32_t)j);
  return __hiloint2double(__double2hiint(v), (int)low);
}
__device__ inline float place_score(double p) { return (float)p; }
__device__ inline int place_class(double p) {
  const int low = __double2loint(p) & 0xffff;
  return p == -INFINITY ? -1 : p < 0.0 ? low : 0xffff - low;
}
// The larger of v and p stays in v, the smaller is returned.
__device__ inline double keep_larger(double& v, double p) {
  double r;
  // in one piece, so that v stays in its registers
  asm("v_min_f64 %1, %0, %2\n\tv_max_f64 %0, %0, %2" : "+v"(v), "=&v"(r) : "v"(p));
  return r;
}

// bits = 2 bits + (x > y), the comparison's carry in one addition (two wait states
// between a vector comparison and a vector instruction that reads its mask).
__device__ inline void push_bit_if_above(uint32_t& bits, float x, float y) {
  asm("v_cmp_gt_f32 vcc, %1, %2\n\ts_nop 1\n\tv_addc_co_u32 %0, vcc, %0, %0, vcc" : "+v"(bits) : "v"(x), "v"(y) : "vcc");
}

// Places in a lane's queue (long lists only).
constexpr int QUEUE = 16;

// v[LO .. LO + N) from a bitonic sequence to descending order.
template <int LO, int N, int KM>
__device__ __forceinline__ void bitonic_merge(double (&v)[KM]) {
  if constexpr (N > 1) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[LO + N / 2 + i] = keep_larger(v[LO + i], v[LO + N / 2 + i]);
    bitonic_merge<LO, N / 2>(v);
    bitonic_merge<LO + N / 2, N / 2>(v);
  }
}
// Descending order by merging sorted halves (Batcher's odd-even merges).
template <int LO, int N, int R>
__device__ __forceinline__ void odd_even_merge(double (&v)[QUEUE]) {
  if constexpr (2 * R < N) {
    odd_even_merge<LO, N, 2 * R>(v);
    odd_even_merge<LO + R, N, 2 * R>(v);
#pragma unroll
    for (int i = LO + R; i + R < LO + N; i += 2 * R) v[i + R] = keep_larger(v[i], v[i + R]);
  } else {
    v[LO + R] = keep_larger(v[LO], v[LO + R]);
  }
}
template <int LO, int N>
__device__ __forceinline__ void odd_even_sort(double (&v)[QUEUE]) {
  if constexpr (N > 1) {
    odd_even_sort<LO, N / 2>(v);
    odd_even_sort<LO + N / 2, N / 2>(v);
    odd_even_merge<LO, N, 1>(v);
  }
}

template <int KM>
struct LaneRow {
  static constexpr bool QUEUED = KM > 16;  // a list of 32 or 64 places
  float m = -FLT_MAX, s = 0.0f, t = 0.0f;
  int before = 0;
  float last = INFINITY;  // the list's last score
  int queued = 0;
  double v[KM ? KM : 1];

  // A queued list starts empty, its places past k at +inf in front, where nothing gets
  // before them, so that its last place is the k-th.
  __device__ void clear(int k) {
    if constexpr (QUEUED) {
#pragma unroll
      for (int i = 0; i < KM; ++i) v[i] = i < KM - k ? INFINITY : -INFINITY;
      last = -INFINITY;
    }
  }
  // Others start as the first 16 columns in order; their k-th place is looked up.
  __device__ void start(const float (&x)[CH], int j0, int k) {
    double q[QUEUE];
    static_assert(CH == QUEUE, "the first step fills a queue");
#pragma unroll
    for (int i = 0; i < CH; ++i) q[i] = x[i] > -INFINITY ? place_of(x[i], j0 + i) : -INFINITY;
    odd_even_sort<0, QUEUE>(q);
#pragma unroll
    for (int i = 0; i < KM; ++i) v[i] = q[i < QUEUE ? i : 0];
    find_last(k);
  }
  __device__ void find_last(int k) {
    double p = v[QUEUED ? KM - 1 : 0];
#pragma unroll
    for (int i = 1; i < KM && !QUEUED; ++i) {
      asm volatile("" : "+s"(k));  // else an index into a list in memory
      p = i < k ? v[i] : p;
    }
    last = place_score(p);
  }
  // v[i] of the list from its first place on (i is known where this is used).
  __device__ static int place_in(int i, int k) { return QUEUED ? i - (KM - k) : i; }
  // A place between those that it is below and those that it beats, which move on by
  // one (-inf: nothing changes).
  __device__ void insert(double p) {
#pragma unroll
    for (int q = 0; q < KM; ++q) p = keep_larger(v[q], p);
  }
  // The queue into the list: sorted, its m-th best meets the list's m-th last, the
  // larger stays, and what results falls and then rises.
  __device__ void take(const double* queue) {
    double q[QUEUE];
#pragma unroll
    for (int i = 0; i < QUEUE; ++i) {
      const double p = queue[i * 64];
      q[i] = i < queued ? p : -INFINITY;
    }
    odd_even_sort<0, QUEUE>(q);
#pragma unroll
    for (int i = 0; i < QUEUE; ++i) (void)keep_larger(v[KM - 1 - i], q[i]);
    bitonic_merge<0, KM>(v);
    queued = 0;
  }
  // Columns j0 .. j0 + CH - 1 (those past the last are -inf); again(i) is column
  // j0 + i once more, for i that differs from lane to lane.  Long lists take the scores
  // above their last place through a queue in LDS (a place every 64 doubles), 16 at a
  // time or with the row's end; short ones take them one at a time, all lanes until the
  // slowest is through.  (When this was chosen: 300,007 x 1000 with 32 alternatives 309 us
  // by queue and 399 one at a time, 2M x 100 with 10 alternatives 346 and 291.)
  template <typename Again>
  __device__ __forceinline__ void step(const LogProbArgs& a, const float (&x)[CH], int j0, int y, float ay, bool end,
                                       bool first, double* queue, Again again) {
    float mn = x[0];
#pragma unroll
    for (int i = 1; i < CH; ++i) mn = fmaxf(mn, x[i]);
    const bool news = KM > 0 && mn > last;
    mn = fmaxf(m, mn);
    const float dy = fmaxf((m - mn) * a.c2, -1500.0f), f = exp2_hw(dy);
    float as = 0.0f, at = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float yv = (x[i] - mn) * a.c2, e = exp2_hw(yv);
      as += e;
      at = fmaf(e, fmaxf(yv, -1500.0f), at);
      if (i % 4 == 3) asm volatile("" : "+v"(as), "+v"(at));  // here and now: put off, the terms take registers
    }
    t = fmaf(f, fmaf(s, dy, t), at);
    s = fmaf(f, s, as);
    m = mn;
    if (a.rank) {
#pragma unroll
      for (int i = 0; i < CH; ++i) before += (x[i] > ay) | ((x[i] == ay) & (j0 + i < y));
    }
    if (KM > 0 && !QUEUED && first) {
      start(x, j0, a.k);
    } else if (KM > 0 && (__any(news) || (QUEUED && end))) {
      // a bit per column above the list's last place, then the lanes' columns one after
      // the other, the first one first
      uint32_t bits = 0;
#pragma unroll
      for (int i = CH - 1; i >= 0; --i) push_bit_if_above(bits, x[i], last);
      do {
        if (bits) {
          const int i = __builtin_ctz(bits);
          const double p = place_of(again(i), j0 + i);
          if constexpr (QUEUED) queue[queued++ * 64] = p;
          else insert(p);
        }
        bits &= bits - 1;
        if constexpr (QUEUED)
          if (__any(queued == QUEUE) || (end && !__any(bits != 0))) take(queue);
      } while (__any(bits != 0));
      find_last(a.k);
    }
  }
};

template <int KM>
__device__ inline void finish_lane(const LogProbArgs& a, LaneRow<KM>& r, int64_t row, int split, int y, float ay) {
  if (a.splits == 1) {
    const RowStats st{r.m, r.s, r.t, 0.0f};
    const float l2 = st.log2_s(), ls = st.log_s(l2);
    store_row(a, row, st, ls, st.entropy(l2), y, ay, r.before);
#pragma unroll
    for (int q = 0; q < KM; ++q) {
      const int at = r.place_in(q, a.k);
      if (at >= 0 && at < a.k) store_top(a, row, at, place_score(r.v[q]), place_class(r.v[q]), st, ls);
    }
    return;
  }
  double* p = a.part + (int64_t)split * (2 + a.k) * a.n + row;
  reinterpret_cast<float2*>(p)[0] = make_float2(r.m, r.s);
  reinterpret_cast<float2*>(p)[a.n] = make_float2(r.t, __int_as_float(r.before));
#pragma unroll
  for (int q = 0; q < KM; ++q) {
    const int at = r.place_in(q, a.k);
    if (at >= 0 && at < a.k) p[(int64_t)(2 + at) * a.n] = r.v[q];
  }
}

constexpr int STEP_S = CH + 4;  // floats of a row's step in LDS

// LDS of a wave of k_cols_by_lane: the lanes' current scores, for the few that enter
// their lists, and the lists' queues.
template <int KM>
struct ColsShared {
  float step[KM ? 64 * STEP_S : 1];
  double queue[LaneRow<KM>::QUEUED ? 64 * QUEUE : 1];
};

// Column-major: lanes on consecutive rows, so that every load is a run of a column; the
// next step's 16 loads are on their way during a step.  No lane needs another one.
// Bound by vector instructions: they fill the issue slots at 2M x 100 with 10 alternatives (240 us, 4.2 TB/s of the needed bytes)
// and 0.72 of them at 300,007 x 1000 with 32 (300 us, 4.3 TB/s), where lists leave
// registers for three waves per SIMD.
template <int KM>
__global__ void __launch_bounds__(256) k_cols_by_lane(LogProbArgs a) {
  __shared__ __align__(16) ColsShared<KM> sh[4];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = (int64_t)blockIdx.x * 4 + w;
  if (unit >= (int64_t)a.tiles * a.splits) return;
  const int split = (int)(unit / a.tiles);
  const int64_t base = (unit - (int64_t)split * a.tiles) * 64;
  const int64_t left = a.n - 1 - base;  // rows past the end read row n - 1 and store nothing
  const int loc = lane < left ? lane : (int)left;
  const int64_t row = base + loc;
  const int j0 = split * a.per, j1 = j0 + a.per < a.d ? j0 + a.per : a.d;
  const float* F = static_cast<const float*>(a.F) + base;
  const int y = a.labels ? a.labels[row] : -1;
  const float ay = y >= 0 && y < a.d ? F[(int64_t)y * a.ld + loc] : 0.0f;
  LaneRow<KM> r;
  r.clear(a.k);
  float* mine = sh[w].step + (KM ? lane * STEP_S : 0);
  double* queue = sh[w].queue + (LaneRow<KM>::QUEUED ? lane : 0);
  auto load = [&](float (&to)[CH], int j) {
    const float* p = F + (int64_t)j * a.ld;
    if (j + CH <= j1) {
#pragma unroll
      for (int i = 0; i < CH; ++i, p += a.ld) to[i] = p[loc];
    } else {
#pragma unroll
      for (int i = 0; i < CH; ++i, p += a.ld) {
        to[i] = -INFINITY;
        if (j + i < j1) to[i] = p[loc];
      }
    }
  };
  auto step = [&](const float (&now)[CH], int j) {
    if (KM) {
#pragma unroll
      for (int i = 0; i < CH; i += 4)
        *reinterpret_cast<float4*>(mine + i) = make_float4(now[i], now[i + 1], now[i + 2], now[i + 3]);
    }
    r.step(a, now, j, y, ay, j + CH >= j1, j == j0, queue, [&](int i) { return mine[i]; });
  };
  if constexpr (LaneRow<KM>::QUEUED) {
    float x[CH], nx[CH];
    load(nx, j0);
    for (int j = j0; j < j1; j += CH) {
#pragma unroll
      for (int i = 0; i < CH; ++i) x[i] = nx[i];
      if (j + CH < j1) load(nx, j + CH);
      step(x, j);
    }
  } else {
    // two sets of registers in turn: one is read while the other is used
    float x[2][CH];
    load(x[0], j0);
    for (int j = j0; j < j1; j += 2 * CH) {
      wait_loads();
      if (j + CH < j1) load(x[1], j + CH);
      step(x[0], j);
      if (j + CH < j1) {
        wait_loads();
        if (j + 2 * CH < j1) load(x[0], j + 2 * CH);
        step(x[1], j + CH);
      }
    }
  }
  if (lane <= left) finish_lane<KM>(a, r, row, split, y, ay);
}

// Row-major: 128 bytes of each of 64 rows at a time, eight lanes a row, through LDS.
// (200,000 x 640 fp32 with 5 alternatives 134 us, 3.9 TB/s; 1M x 30 64 us.)
template <typename T, int KM>
__global__ void __launch_bounds__(256) k_rows_by_lane(LogProbArgs a) {
  constexpr int VEC = 16 / sizeof(T), COLS = 8 * VEC;
  __shared__ __align__(16) char lds[4][64 * TILE_B];
  __shared__ double queues[4][LaneRow<KM>::QUEUED ? 64 * QUEUE : 1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tile = (int64_t)blockIdx.x * 4 + w;
  if (tile >= a.tiles) return;
  const int64_t base = tile * 64;
  const int64_t left = a.n - 1 - base;
  const int loc = lane < left ? lane : (int)left;
  const int64_t row = base + loc;
  const T* F = static_cast<const T*>(a.F);
  const int y = a.labels ? a.labels[row] : -1;
  const float ay = y >= 0 && y < a.d ? to_f32(F[row * a.ld + y]) : 0.0f;
  LaneRow<KM> r;
  r.clear(a.k);
  // lane l brings vector l % 8 of rows l / 8, l / 8 + 8, ...
  const int vrow = lane >> 3, vcol = (lane & 7) * VEC;
  char* put = lds[w] + vrow * TILE_B + (lane & 7) * 16;
  const char* get = lds[w] + lane * TILE_B;
  double* queue = queues[w] + (LaneRow<KM>::QUEUED ? lane : 0);
  uint4 nx[8];
  auto load = [&](int j) {
    const int c = j + vcol;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int rr = vrow + q * 8;
      const T* p = F + (base + (rr < left ? rr : left)) * a.ld + c;
      if (c + VEC <= a.d) {
        __builtin_memcpy(&nx[q], p, 16);
      } else {  // the row's end: its elements one by one
        T e[VEC];
#pragma unroll
        for (int u = 0; u < VEC; ++u)
          if (c + u < a.d) e[u] = p[u];
        __builtin_memcpy(&nx[q], e, 16);
      }
    }
  };
  load(0);
  for (int j = 0; j < a.d; j += COLS) {
    wave_sync();
#pragma unroll
    for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(put + q * 8 * TILE_B) = nx[q];
    wave_sync();
    if (j + COLS < a.d) load(j + COLS);
#pragma unroll 1
    for (int h = 0; h < COLS / CH; ++h) {
      if (j + h * CH >= a.d) break;
      float x[CH];
#pragma unroll
      for (int q = 0; q < CH / VEC; ++q) {
        const uint4 raw = *reinterpret_cast<const uint4*>(get + (h * (CH / VEC) + q) * 16);
        T e[VEC];
        __builtin_memcpy(e, &raw, 16);
#pragma unroll
        for (int u = 0; u < VEC; ++u) x[q * VEC + u] = j + h * CH + q * VEC + u < a.d ? to_f32(e[u]) : -INFINITY;
      }
      r.step(a, x, j + h * CH, y, ay, j + h * CH + CH >= a.d, j + h == 0, queue,
             [&](int i) { return to_f32(reinterpret_cast<const T*>(get)[h * CH + i]); });
    }
  }
  if (lane <= left) finish_lane<KM>(a, r, row, 0, y, ay);
}

// The splits' statistics and lists of a row joined by G lanes, lane per split (20,000 x
// 1000 with 10 alternatives: 47 us with the splits' own pass, 93 with a wave per row).  Each
// lane has its list's next place and the one after it in hand; the best of the G next
// places is the row's next alternative.
template <int CTRL>
__device__ inline double dpp_place(double p) {
  return __hiloint2double((int)dpp_u32<CTRL>((uint32_t)__double2hiint(p)), (int)dpp_u32<CTRL>((uint32_t)__double2loint(p)));
}
template <int G, typename T, typename Op>
__device__ inline T group_all(T x, Op op, T (*dpp[4])(T)) {
#pragma unroll
  for (int q = 0; q < (G >= 16 ? 4 : 3); ++q) x = op(x, dpp[q](x));
  if (G == 64) {
    x = op(x, __shfl_xor(x, 16, 64));
    x = op(x, __shfl_xor(x, 32, 64));
  }
  return x;
}

template <int G>
__global__ void __launch_bounds__(256) k_join(LogProbArgs a) {
  const int lane = threadIdx.x & (G - 1);
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G;
  if (row >= a.n) return;  // whole groups, which exchange nothing with others
  float (*fdpp[4])(float) = {
      [](float x) { return __uint_as_float(dpp_u32<0xb1>(__float_as_uint(x))); },
      [](float x) { return __uint_as_float(dpp_u32<0x4e>(__float_as_uint(x))); },
      [](float x) { return __uint_as_float(dpp_u32<0x141>(__float_as_uint(x))); },
      [](float x) { return __uint_as_float(dpp_u32<0x140>(__float_as_uint(x))); }};
  int (*idpp[4])(int) = {[](int x) { return (int)dpp_u32<0xb1>((uint32_t)x); }, [](int x) { return (int)dpp_u32<0x4e>((uint32_t)x); },
                         [](int x) { return (int)dpp_u32<0x141>((uint32_t)x); },
                         [](int x) { return (int)dpp_u32<0x140>((uint32_t)x); }};
  double (*ddpp[4])(double) = {dpp_place<0xb1>, dpp_place<0x4e>, dpp_place<0x141>, dpp_place<0x140>};
  auto add = [](auto x, auto y) { return x + y; };
  const bool on = lane < a.splits;
  const double* list = a.part + (int64_t)(on ? lane : 0) * (2 + a.k) * a.n + row;
  const float2* head = reinterpret_cast<const float2*>(list);  // (m, s), then (t, before)
  const float2 ms = on ? head[0] : make_float2(-FLT_MAX, 0.0f);
  const float2 tb = on ? head[a.n] : make_float2(0.0f, 0.0f);
  const float mm = group_all<G>(ms.x, [](float x, float y) { return fmaxf(x, y); }, fdpp);
  const float dy = fmaxf((ms.x - mm) * a.c2, -1500.0f), f = exp2_hw(dy);
  const float s = group_all<G>(f * ms.y, add, fdpp);
  const float t = group_all<G>(f * fmaf(ms.y, dy, tb.x), add, fdpp);
  const int before = group_all<G>(__float_as_int(tb.y), add, idpp);
  const RowStats st{mm, s, t, 0.0f};
  const float l2 = st.log2_s(), ls = st.log_s(l2);
  const int y = a.labels ? a.labels[row] : -1;
  if (lane == 0) {
    const float ay = y >= 0 && y < a.d ? static_cast<const float*>(a.F)[(int64_t)y * a.ld + row] : 0.0f;
    store_row(a, row, st, ls, st.entropy(l2), y, ay, before);
  }
  if (a.k == 0) return;
  list += 2 * a.n;
  auto place = [&](int at) { return on && at < a.k ? list[(int64_t)at * a.n] : -INFINITY; };
  int at = 2;
  double p = place(0), after = place(1);
  for (int q = 0; q < a.k; ++q) {
    const double best = group_all<G>(p, [](double x, double y) { return x > y ? x : y; }, ddpp);
    if (lane == (q & (G - 1))) store_top(a, row, q, place_score(best), place_class(best), st, ls);
    if (p == best && best > -INFINITY) {  // one lane: places of different classes differ
      p = after;
      after = place(at++);
    }
  }
}

// ---------------------------------------------------------------- a row in a wave's or a block's registers
// NT threads per row, E elements each; ROWS rows per block.
// Places for collected scores, and half as many for 16-byte pieces of the row.
constexpr int CAND_WAVE = 256, CAND_BLOCK = 1024;
// Order-preserving bits of a score (both zeros alike), and back.
__device__ inline uint32_t score_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ (uint32_t)((int32_t)b >> 31 | 0x80000000);
}
__device__ inline float key_score(uint32_t k) { return __uint_as_float(k ^ (~(uint32_t)((int32_t)k >> 31) | 0x80000000)); }
constexpr uint32_t KEY_EXCLUDED = 0x007fffffu;  // of -inf

// What the threads of one row share.  Candidates are ordered by one 64-bit
// comparison: the score's key, then the smaller class.
template <int NT>
struct RowShared {
  static constexpr int W = NT / 64, CAP = NT == 64 ? CAND_WAVE : CAND_BLOCK;
  static_assert(CAP % 8 == 0, "places are read eight at a time");
  u32x4 piece[CAP / 2];
  uint64_t cand[CAP];
  uint64_t best[SB_MAX_TOP];
  int piece_at[CAP / 2];
  float lane_max[2][W][64];
  float sums[3][W];
  int pieces[2], count[2];  // of even and odd rows: one is cleared while the other counts
};
__device__ inline uint64_t cand_of(float v, int j) { return (uint64_t)score_key(v) << 32 | (uint32_t)~j; }
__device__ inline float cand_score(uint64_t c) { return key_score((uint32_t)(c >> 32)); }
__device__ inline int cand_class(uint64_t c) { return (int)~(uint32_t)c; }

// A key that at least k and not many more of the lanes' keys (one or two each) reach,
// by bisection over its bits; every lane gets it.
template <bool TWO>
__device__ inline uint32_t key_bound(uint32_t k0, uint32_t k1, int k) {
  uint32_t bound = 0;
  const int enough = k + (k >> 3);
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    const uint32_t t = bound | bit;
    int n = __popcll(__ballot(k0 >= t));
    if (TWO) n += __popcll(__ballot(k1 >= t));
    if (n >= k) {
      bound = t;
      if (n <= enough) break;
    }
  }
  return bound;
}

// The largest score below v, so that x >= v is x > below(v); NaN below -inf, which
// nothing is "not above".
__device__ inline float below(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return v == -INFINITY ? NAN : __uint_as_float(b == 0 ? 0x80000001u : v > 0.0f ? b - 1 : b + 1);
}
__device__ inline _Float16 below(_Float16 v) {
  const uint16_t b = __builtin_bit_cast(uint16_t, v);
  const uint16_t to = (b & 0x7fff) == 0 ? 0x8001 : (b & 0x8000) == 0 ? b - 1 : b + 1;
  return __builtin_bit_cast(_Float16, (uint16_t)(b == 0xfc00 ? 0x7e00 : to));
}

// put(place, candidate) for the k best of the first `found` candidates: a candidate's
// place is the number of better ones.
template <int NT, typename Put>
__device__ inline void ranked(const RowShared<NT>& sh, int found, int k, int tid, Put put) {
  for (int i = tid; i < found; i += NT) {
    const uint64_t mine = sh.cand[i];
    int place = 0, o = 0;
    for (; o + 8 <= found; o += 8) {
      uint64_t c[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) c[u] = sh.cand[o + u];
#pragma unroll
      for (int u = 0; u < 8; ++u) place += c[u] > mine;
    }
    if (o < found) {  // the rest, as many read at once
      uint64_t c[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) c[u] = sh.cand[o + u];
#pragma unroll
      for (int u = 0; u < 7; ++u) place += o + u < found && c[u] > mine;
    }
    if (place < k) put(place, mine);
  }
}

// Rows of NT threads, E scores each, one after the other.  As many rows as fit are in
// registers at once, so a row is read once, and its 16 bytes make way for those of the
// next row as soon as they are summed: loads and arithmetic overlap in every wave
// (4096 x 65,000 bf16 with 20 alternatives 177 us with the loads after the sums).
// Bound by vector instructions: 0.84 of the issue slots at that shape (138 us, 3.9 TB/s),
// 0.86 at 200,001 x 1000 fp16 with 16 alternatives (208 us), where a row's 500
// instructions are more for its list and its joins than for its scores.
template <typename T, int NT, int E>
__device__ __forceinline__ void rows_in_block(const LogProbArgs& a, RowShared<NT>& sh, int64_t row, int64_t stride) {
  constexpr int VEC = 16 / sizeof(T), NV = E / VEC, W = NT / 64, CAP = RowShared<NT>::CAP;
  int tid = threadIdx.x & (NT - 1);
  const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto sync = [&]() {
    if (NT == 64) wave_sync();
    else __syncthreads();
  };
  // what is left past the last whole 16 bytes is one score per thread
  const int whole = a.d & ~(VEC - 1);
  // The maxima that bound a list: 64, or one for every 16 bytes of a shorter row; both
  // halves' where the list is longer than half of them (the smallest of the maxima would
  // let too many scores through, and fewer than k would bound nothing).
  const int keys = whole / VEC < 64 ? whole / VEC : 64;
  auto row_at = [&](int64_t r) { return static_cast<const T*>(a.F) + r * a.ld; };
  auto load_vec = [&](const T* F, int q) {
    const uint32_t none = excluded(T());
    u32x4 v = u32x4{none, none, none, none};
    const int j = (q * NT + tid) * VEC;
    if (j < whole) __builtin_memcpy(&v, F + j, 16);
    return v;
  };
  // Scores stay as they are in memory until they are used: a conversion here would wait
  // for them.  The given class is known a row ahead, so its score is read with the row.
  u32x4 raw[NV];
  T tail_raw, ay_raw, mates_raw;  // mates: those before the given class in its 16 bytes, one per thread
  int y = -1, y_next = -1;
  int lane_0 = 0;
  asm("" : "+v"(lane_0));  // labels in vector registers: moved to scalar ones, they would be waited for
  auto load_scalars = [&](int64_t r) {
    const T* F = row_at(r < a.n ? r : a.n - 1);
    int tail_at = whole + tid < a.d ? whole + tid : 0, at = y >= 0 && y < a.d ? y : 0;
    int mate_at = at - min(at & (VEC - 1), tid + 1);
    asm("" : "+v"(tail_at), "+v"(at), "+v"(mate_at));  // indices, not branches
    tail_raw = F[tail_at];
    ay_raw = F[at];
    mates_raw = F[mate_at];
  };
  auto load_label = [&](int64_t r) {
    if (a.labels) y_next = (a.labels + (r < a.n ? r : a.n - 1))[lane_0];
  };
#pragma unroll
  for (int q = 0; q < NV; ++q)
    if (q * NT * VEC < whole) raw[q] = load_vec(row_at(row), q);
  load_label(row);
  y = y_next;
  load_scalars(row);
  load_label(row + stride);
  if (tid == 0) sh.pieces[0] = sh.count[0] = 0;
  for (int turn = 0; row < a.n; row += stride, turn ^= 1) {
    // the compiler sees the thread anew in every row: the places of its scores, a
    // register each, would otherwise be held across the rows
    asm volatile("" : "+v"(tid));
    // the maxima of the first halves of the 16 bytes and of the second ones
    const float tail = whole + tid < a.d ? to_f32(tail_raw) : -INFINITY;
    float lm[2] = {tail, -INFINITY};
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      if (q * NT * VEC >= whole) continue;
      Score<T> x[VEC];
      decode<T>(raw[q], x);
      halves_max(raw[q], x, lm);
      asm volatile("" : "+v"(lm[0]), "+v"(lm[1]));
    }
    // the row is here; told so, the compiler waits for nothing among the sums below, where
    // the next one's scores are on their way
    wait_loads();
    const int64_t next_row = row + stride;
    const int y_now = y;
    const float ay = y >= 0 && y < a.d ? to_f32(ay_raw) : 0.0f;
    const bool mate = y >= 0 && y < whole && tid < (y & (VEC - 1)) && to_f32(mates_raw) == ay;
    if (W > 1) {
      sh.lane_max[0][w][lane] = lm[0];
      sh.lane_max[1][w][lane] = lm[1];
    }
    sync();  // 1
    if (W > 1) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < W; ++u) lm[h] = fmaxf(lm[h], sh.lane_max[h][u][lane]);
    }
    if (tid == 0) sh.pieces[turn ^ 1] = sh.count[turn ^ 1] = 0;
    float m = fmaxf(fmaxf(lm[0], lm[1]), -FLT_MAX);
    m = wave_max(m);
    float b = INFINITY;  // candidates are the scores from here on
    if (a.k > 0) {
      const uint32_t kb = 2 * a.k > keys ? key_bound<true>(score_key(lm[0]), score_key(lm[1]), a.k)
                                          : key_bound<false>(score_key(fmaxf(lm[0], lm[1])), 0, a.k);
      // -inf is no candidate; the lowest score above it is -FLT_MAX
      b = kb > KEY_EXCLUDED ? key_score(kb) : -FLT_MAX;
    }
    // y_j + r in one rounding: a_j c2 - m2 for the rounded m2 = m c2, where its error r is small
    const float m2 = m * a.c2;
    const bool far = !(fabsf(m2) < 0x1p20f);
    const float r = far ? 0.0f : fmaf(m, a.c2, -m2);
    float s = 0.0f, t = 0.0f;
    int before = 0;
    auto term = [&](float yv) {
      const float e = exp2_hw(yv);
      s += e;
      t = fmaf(e, fmaxf(yv, -1500.0f), t);
    };
    // the next of a row's numbers for every thread that wants one: a wave alone counts by itself
    int own_pieces = 0, own_count = 0;
    auto number = [&](bool want, int& own, int* shared) {
      const uint64_t all = __ballot(want);
      int at = own;
      if constexpr (W > 1) {
        int first = 0;
        if (all && lane == 0) first = atomicAdd(shared, __popcll(all));
        at = __builtin_amdgcn_readfirstlane(first);
      } else {
        own += __popcll(all);
      }
      return at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
    };
    auto collect = [&](float xv, int j) {
      if (!__any(xv >= b)) return;
      const int at = number(xv >= b, own_count, &sh.count[turn]);
      if (xv >= b && at < CAP) sh.cand[at] = cand_of(xv, j);
    };
    term(fmaf(tail, a.c2, -m2));
    if (a.rank) before = (tail > ay || (tail == ay && whole + tid < y_now)) + mate;
    if (a.k > 0) collect(tail, whole + tid);
    const Score<T> ay_below = below((Score<T>)ay);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      if (q * NT * VEC >= whole) continue;
      Score<T> x[VEC];
      decode<T>(raw[q], x);
      const int j = (q * NT + tid) * VEC;
#pragma unroll
      for (int u = 0; u < VEC; ++u) term(fmaf((float)x[u], a.c2, -m2));
      asm volatile("" : "+v"(s), "+v"(t));  // here and now: put off, the terms take more registers than there are
      if (a.rank) {
        // classes before y come first at equal scores; those in its own 16 bytes are mates
        const Score<T> over = j + VEC <= y_now ? ay_below : (Score<T>)ay;
#pragma unroll
        for (int u = 0; u < VEC; ++u) before += !(x[u] <= over);
        asm volatile("" : "+v"(before));
      }
      if (a.k > 0) {
        const float xm = max_of(raw[q], x);
        if (__any(xm >= b)) {  // the 16 bytes that hold a candidate
          const int at = number(xm >= b, own_pieces, &sh.pieces[turn]);
          if (xm >= b && at < CAP / 2) {
            sh.piece[at] = raw[q];
            sh.piece_at[at] = j;
          }
        }
      }
      if (next_row < a.n) raw[q] = load_vec(row_at(next_row), q);
    }
    y = y_next;
    load_scalars(next_row);
    load_label(next_row + stride);
    if (far) {  // scores of such size: differences first, from memory once more
      s = t = 0.0f;
      for (int j = tid; j < a.d; j += NT) term((to_f32(row_at(row)[j]) - m) * a.c2);
    }
    s = wave_sum(s);
    t = wave_sum(t);
    if (a.rank) before = wave_sum(before);
    if (W > 1 && lane == 0) {
      sh.sums[0][w] = s;
      sh.sums[1][w] = t;
      sh.sums[2][w] = __int_as_float(before);
    }
    sync();  // 2
    if (W > 1) {
      s = t = 0.0f;
      before = 0;
#pragma unroll
      for (int u = 0; u < W; ++u) {
        s += sh.sums[0][u];
        t += sh.sums[1][u];
        before += __float_as_int(sh.sums[2][u]);
      }
    }
    const RowStats st{m, s, t, r};
    const float l2 = st.log2_s(), ls = st.log_s(l2);
    if (tid == 0) store_row(a, row, st, ls, st.entropy(l2), y_now, ay, before);
    if (a.k == 0) continue;
    const int pieces = W > 1 ? sh.pieces[turn] : own_pieces;
    const int parts = (pieces < CAP / 2 ? pieces : CAP / 2) * VEC;
    for (int i0 = 0; i0 < parts; i0 += NT) {
      const uint32_t i = i0 + tid, at = (int)i < parts ? i : 0;
      const float v = to_f32(reinterpret_cast<const T*>(sh.piece)[at]);
      collect((int)i < parts ? v : -INFINITY, sh.piece_at[at / VEC] + (int)(at % VEC));
    }
    sync();  // 3
    int found = W > 1 ? sh.count[turn] : own_count;
    if (pieces <= CAP / 2 && found <= CAP) {
      ranked<NT>(sh, found, a.k, tid,
                 [&](int place, uint64_t c) { store_top(a, row, place, cand_score(c), cand_class(c), st, ls); });
    } else {
      // Too many (equal scores, or lanes that hold most of the large ones): the row once
      // more, in order, and the k best so far whenever the places run out; from then on a
      // candidate is above the k-th.
      constexpr int PART = NT < CAP / 2 ? NT : CAP / 2;
      const T* F = row_at(row);
      uint32_t above = score_key(b) - 1;
      found = 0;
      for (int j0 = 0; j0 < a.d; j0 += PART) {
        sync();  // the places are free, and the count is read
        if (tid == 0) sh.count[turn] = found;
        sync();
        const int j = j0 + tid;
        if (tid < PART && j < a.d) {
          const float v = to_f32(F[j]);
          if (v > -INFINITY && score_key(v) > above) sh.cand[atomicAdd(&sh.count[turn], 1)] = cand_of(v, j);
        }
        sync();
        found = sh.count[turn];
        if (found + PART > CAP || j0 + PART >= a.d) {
          ranked<NT>(sh, found, a.k, tid, [&](int place, uint64_t c) { sh.best[place] = c; });
          sync();
          found = found < a.k ? found : a.k;
          for (int i = tid; i < found; i += NT) sh.cand[i] = sh.best[i];
          if (found == a.k) above = (uint32_t)(sh.best[a.k - 1] >> 32);
        }
      }
      sync();
      for (int i = tid; i < found; i += NT)
        store_top(a, row, i, cand_score(sh.cand[i]), cand_class(sh.cand[i]), st, ls);
    }
    for (int q = found + tid; q < a.k; q += NT) store_top(a, row, q, -INFINITY, -1, st, ls);
  }
}

// A block of 256 has four rows of a wave each, or one row.
template <typename T, int NT, int E>
__global__ void __launch_bounds__(NT == 64 ? 256 : NT, 4) k_row_in_block(LogProbArgs a) {
  constexpr int ROWS = NT == 64 ? 4 : 1;
  __shared__ RowShared<NT> sh[ROWS];
  const int rg = NT == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const int64_t row = (int64_t)blockIdx.x * ROWS + rg;
  if (row < a.n) rows_in_block<T, NT, E>(a, sh[rg], row, (int64_t)gridDim.x * ROWS);
}

// ---------------------------------------------------------------- launch
constexpr int MAX_SPLITS = 64;    // lanes of k_join
constexpr int WANT_WAVES = 2048;  // waves that fill the card: eight per CU

// Column-major scores of few rows: column splits of at least 64 columns.  Two splits
// of a long list's row cost more for their two lists than they gain (60,000 x 300 with
// 64 alternatives 91 us whole, 119 in two; 20,000 x 300 90 whole, 76 in four).
int column_splits(int64_t n, int32_t d, int32_t k) {
  const int64_t tiles = (n + 63) / 64;
  int64_t s = tiles >= WANT_WAVES ? 1 : WANT_WAVES / tiles;
  if (s > d / 64) s = d / 64;
  if (s > MAX_SPLITS) s = MAX_SPLITS;
  return s < 1 || (s == 2 && k > 32) ? 1 : (int)s;
}

template <template <int> class Launch, typename... Args>
void by_list(int k, Args... args) {
  if (k == 0) Launch<0>::run(args...);
  else if (k == 1) Launch<1>::run(args...);
  else if (k <= 4) Launch<4>::run(args...);
  else if (k <= 8) Launch<8>::run(args...);
  else if (k <= 12) Launch<12>::run(args...);
  else if (k <= 16) Launch<16>::run(args...);
  else if (k <= 32) Launch<32>::run(args...);
  else Launch<64>::run(args...);
}
template <int KM>
struct ColsByLane {
  static void run(LogProbArgs a, dim3 blocks, hipStream_t st) {
    hipLaunchKernelGGL(k_cols_by_lane<KM>, blocks, dim3(256), 0, st, a);
  }
};
template <typename T>
struct RowsByLane {
  template <int KM>
  struct With {
    static void run(LogProbArgs a, dim3 blocks, hipStream_t st) {
      hipLaunchKernelGGL((k_rows_by_lane<T, KM>), blocks, dim3(256), 0, st, a);
    }
  };
};

template <typename T>
void launch_rows(LogProbArgs a, hipStream_t st) {
  // A lane per row where there are rows for the lanes of the card: its time is that of
  // d columns until there are some 100,000 rows, a wave's that of the rows.  16-bit
  // scores are half the bytes for a wave and the same work for a lane.  (us by lane and
  // by wave: fp32, 5 alternatives, 20,000 x 125 20 and 20, 50,000 x 312 41 and 46,
  // 200,000 x 640 134 and 189, x 1000 246 and 212; 64 alternatives, 100,000 x 300 108 and
  // 233, 200,000 x 640 313 and 487; fp16, 16 alternatives, 20,000 x 125 30 and 24, 200,000
  // x 300 138 and 180, x 640 238 and 208, 500,000 x 600 400 and 508, x 1000 596 and 515; 64
  // alternatives, 500,000 x 600 720 and 1155.)  The limit of 640 columns is the same for
  // every size and list: 200,000 x 800 fp32 with 5 is taken by wave, 204, where a lane per
  // row takes 162.
  if (a.n >= (int64_t)(sizeof(T) == 2 ? 480 : 160) * a.d && a.d <= 640) {
    by_list<RowsByLane<T>::template With>(a.k, a, dim3((a.tiles + 3) / 4), st);
    return;
  }
  // else a wave or a block; few rows take more threads each
  auto blocks = [](int64_t b, int most = 256 * 8) { return dim3((unsigned)(b < most ? b : most)); };
  if (a.d <= 1024)
    hipLaunchKernelGGL((k_row_in_block<T, 64, 16>), blocks((a.n + 3) / 4), dim3(256), 0, st, a);
  else if (a.d <= 4096 && a.n >= WANT_WAVES)
    hipLaunchKernelGGL((k_row_in_block<T, 64, 64>), blocks((a.n + 3) / 4), dim3(256), 0, st, a);
  else if (a.d <= 4096)
    hipLaunchKernelGGL((k_row_in_block<T, 256, 16>), blocks(a.n), dim3(256), 0, st, a);
  else if (a.d <= 16384 && a.n >= WANT_WAVES / 4)
    hipLaunchKernelGGL((k_row_in_block<T, 256, 64>), blocks(a.n, 1024), dim3(256), 0, st, a);
  else if (a.d <= 16384)
    hipLaunchKernelGGL((k_row_in_block<T, 1024, 16>), blocks(a.n), dim3(1024), 0, st, a);
  else if constexpr (sizeof(T) == 2)  // two blocks share a CU: one row's loads meet another's arithmetic
    hipLaunchKernelGGL((k_row_in_block<T, 512, 128>), blocks(a.n, 512), dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL((k_row_in_block<T, 1024, 64>), blocks(a.n, 256), dim3(1024), 0, st, a);
}

}  // namespace

// Workspace: the column splits' statistics and lists.
int64_t log_probs_ws_bytes(int64_t n, int32_t d, int32_t k) {
  const int s = column_splits(n, d, k);
  return s == 1 ? 0 : align256((int64_t)s * (2 + k) * n * 8);
}

int32_t launch_log_probs(const void* F, int32_t dtype, int32_t order, int64_t n, int32_t d, int64_t ld_f, double T,
                         const int32_t* labels, float* logp, int32_t* rank, float* lse, float* entropy, int32_t k,
                         int32_t* top_id, float* top_logp, int64_t ld_top, void* ws, hipStream_t st) {
  LogProbArgs a{F, n, d, ld_f, (float)(1.0 / T), (float)(1.4426950408889634 / T), labels, logp, rank, lse, entropy, k,
                top_id, top_logp, ld_top, (int)((n + 63) / 64), 1, d, nullptr};
  if (order == SB_COLUMN_MAJOR && n == 1 && ld_f == 1) {  // one row without gaps is a row-major row
    order = SB_ROW_MAJOR;
    a.ld = d;
  }
  if (order == SB_COLUMN_MAJOR) {
    // whole steps, so that none but the row's end is filled up: a filled column is an
    // excluded class, which would count among those before an excluded one
    a.splits = column_splits(n, d, k);
    a.per = ((d + a.splits - 1) / a.splits + CH - 1) / CH * CH;
    a.splits = (d + a.per - 1) / a.per;
    a.part = static_cast<double*>(ws);
    const int64_t units = (int64_t)a.tiles * a.splits;
    by_list<ColsByLane>(k, a, dim3((unsigned)((units + 3) / 4)), st);
    auto blocks = [&](int g) { return dim3((unsigned)((n * g + 255) / 256)); };
    if (a.splits > 16) hipLaunchKernelGGL(k_join<64>, blocks(64), dim3(256), 0, st, a);
    else if (a.splits > 8) hipLaunchKernelGGL(k_join<16>, blocks(16), dim3(256), 0, st, a);
    else if (a.splits > 1) hipLaunchKernelGGL(k_join<8>, blocks(8), dim3(256), 0, st, a);
  } else if (dtype == SB_F32) {
    launch_rows<float>(a, st);
  } else if (dtype == SB_F16) {
    launch_rows<__half>(a, st);
  } else {
    launch_rows<__hip_bfloat16>(a, st);
  }
  return check_launch("sb_log_probs");
}

}  // namespace sb
