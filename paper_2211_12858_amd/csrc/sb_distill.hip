// Distillation from a teacher's top classes: the loss of every row and its
// first and second derivatives by the scores (sb_distill_loss,
// sb_distill_gradients).
//
// For a row with scores a, z = a - max a, s1 = sum exp(z_j), sT = sum exp(z_j / T),
// teacher's probabilities q_t of classes c_t, Q = sum q_t, A = w where the row has
// a label (else 0), B = (1 - w) T:
//   target_j = A [j == label] + B sum_{t: c_t == j} q_t
//   loss = A log s1 + B T (sum q_t log q_t + Q log sT) - sum_j target_j z_j
//   g_j  = A p1_j + B Q pT_j - target_j
//   h_j  = A p1_j (1 - p1_j) + (B / T) Q pT_j (1 - pT_j)
// (0 log 0 = 0; a score of -inf has p = 0, and a target on it makes the loss +inf),
// so the teacher's list and the label are one sparse target row, and at T = 1 the
// two softmaxes are one.
//
// k_distill_regs (rows of up to 1024 scores): a row tile's scores stay in the
//   registers of a block's waves, lanes on consecutive rows, c columns per lane, so
//   F is read once and every load and store is a run of a column.  Waves exchange
//   maxima and sums in LDS; each handles its share of the tile's list places, and
//   all waves then look through all places for the classes of their own columns and
//   add their targets to the wave's LDS tile of 16 columns.  The gradients replace
//   the targets in that tile, from which 16 lanes per row segment add the squared
//   column norms in fp64, in a fixed order; a block's sums are one partial.  While a
//   tile's gradients go out the same registers take the next tile's scores.
//   2M x 100 with labels and 10 places 402 us, 4.4 TB/s of 4.7 in a copy: the bytes.
//   300,007 x 1000 with hessians and 32 places 1280 us, 2.9 TB/s: one block of 16
//   waves per CU holds 32 rows, and columns of an odd number of rows start anywhere in
//   a cache line, so that half as many requests again go to the L2 (300,032 rows 950 us);
//   vector instructions take a third of the issue slots.
//   The loss alone: 1,000,003 x 100 with 10 places 104 us, 4.7 TB/s: the bytes (134 us
//   with the listed scores read from memory).
// k_loss_by_lane: the loss alone of many rows with short lists, a wave per tile.
// k_distill_stats, k_distill_rows, k_distill_range (wider rows): maxima and sums of
//   column ranges, then every row's statistics, targets and loss, then the outputs range
//   by range, with what each range's targets take off the loss (k_distill_join adds
//   them up; listed scores read from memory in k_distill_rows took 86 us more).  F is
//   read twice; 20,001 x 5003 with hessians and 64 places 455 us in all, of which 131, 11
//   and 294, the last 4.1 TB/s.
//
// k_hot_loss (with k_hot_stats): the loss at T > 4, whose terms are far larger than what
//   they add up to.
//
// exp(z / T) is 2^(z * log2(e) / T) by the hardware's exponential, which returns 0
// below 2^-126: probabilities under 2^-126 of the row's largest are 0.
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "sb_common.h"
#include "sb_distill_plan.h"

extern "C" __device__ float sb_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");  // v_mul_legacy_f32

namespace sb {
namespace {

constexpr float LOG2E = 1.44269504088896341f;

struct RowArgs {
  DistillArgs a;
  float inv_t;      // 1 / T
  float c2;         // log2(e) / T
  float w, b, bt;   // hard weight, B = (1 - w) T, B T
  double* npart;    // [d][parts] or NULL
  int parts;
  int waves, groups, tiles;
  int tile_bytes;  // of LDS per row tile
  float* stats;  // [ranges][3][n]: k_distill_stats; later [ranges][2][n]: k_distill_range
  float* row;    // [ROW_VALUES + k][n]: k_distill_rows
  int ranges, cols, slots;
};

// Other lanes of the wave see this wave's LDS writes; the compiler keeps the order.
__device__ inline void wave_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The product, 0 where a factor is: z is -inf for an excluded class, which adds nothing
// to the loss unless it is a target.
__device__ inline float product(float x, float z) { return sb_mul_legacy(x, z); }
// Of a row's sum of exponentials, 0 only where every class is excluded.
__device__ inline float inverse(float s) { return s > 0.0f ? 1.0f / s : 0.0f; }
__device__ inline float log_of(float s) { return s > 0.0f ? logf(s) : 0.0f; }

// A list place: class and value; unused ones have class -1 and a value of -inf,
// whatever they held.
struct Place {
  int id;
  float v;
};
__device__ inline Place load_place(const DistillArgs& a, int t, int64_t row) {
  return Place{a.t_id[t * a.ld_t + row], a.t_val[t * a.ld_t + row]};
}
__device__ inline Place usable(const DistillArgs& a, const Place& p) {
  return p.id >= 0 && p.id < a.d ? p : Place{-1, -INFINITY};
}

// The teacher's distribution from the sums over the used places: zs = sum e_t and
// us = sum e_t log-ish_t, e_t = exp(v_t / T - max) or exp(v_t).
struct Teacher {
  float Q;    // sum q
  float ent;  // sum q log q
  float wt;   // B * q_t = wt * e_t
};
__device__ inline Teacher teacher_of(const RowArgs& r, float zs, float us) {
  Teacher t;
  if (r.a.teacher == SB_TEACHER_LOGITS) {
    const bool any = zs > 0.0f;
    const float iz = any ? 1.0f / zs : 0.0f;
    t.Q = any ? 1.0f : 0.0f;
    t.ent = any ? us * iz - logf(zs) : 0.0f;
    t.wt = r.b * iz;
  } else {
    t.Q = zs;
    t.ent = us;
    t.wt = r.b;
  }
  return t;
}
// e_t and its term of us, from the value and the list's maximum
__device__ inline float place_exp(const RowArgs& r, float v, float vmax, float& us) {
  float u;
  if (r.a.teacher == SB_TEACHER_LOGITS) u = (v - (vmax == -INFINITY ? 0.0f : vmax)) * r.inv_t;
  else u = v;
  const float e = exp2_hw(u * LOG2E);
  us += e * fmaxf(u, -1000.0f);  // e = 0 at -inf
  return e;
}

// The listed places of the tile's rows, class and value or exponential, in LDS.
struct __align__(8) Listed {
  int id;
  float e;
};

// A target of the lane's row into its (zeroed) tile row of CG columns, where c is one
// of them.  A class listed again is added to what is there; a bit per column says
// which are (a float atomic per place instead takes the LDS three clocks a lane).
template <int CG>
__device__ inline void put_target(float* trow, uint32_t& seen, uint32_t c, float v) {
  if (c < (uint32_t)CG) {
    const uint32_t bit = 1u << c;
    if (seen & bit) v += trow[c];
    trow[c] = v;
    seen |= bit;
  }
}

// The targets of the columns from jg: the places', eight read at a time, and the
// label's (class y, weight A).
template <int CG, int ROWS>
__device__ inline void add_targets(const Listed* ent, int K, int rl, int jg, float wt, int y, float A, float* trow) {
  uint32_t seen = 0;
  int s = 0;
  for (; s + 8 <= K; s += 8) {
    Listed p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = ent[(s + u) * ROWS + rl];
#pragma unroll
    for (int u = 0; u < 8; ++u) put_target<CG>(trow, seen, column_from(p[u].id, jg), wt * p[u].e);
  }
  for (; s < K; ++s) {
    const Listed p = ent[s * ROWS + rl];
    put_target<CG>(trow, seen, column_from(p.id, jg), wt * p.e);
  }
  if (y >= 0) put_target<CG>(trow, seen, column_from(y, jg), A);
}

// Squared norms of a tile's columns: CG lanes take the columns of a segment's rows,
// every SEGSth of the part's (so that the segments' reads fall on different banks
// and one address with fixed offsets serves all rows).
template <int CG, int PARTS>
__device__ inline double tile_norms(const float* tile, int lane) {
  constexpr int SEGS = 64 / CG / PARTS, S = CG + 4;
  asm volatile("" : "+v"(lane));  // the address is formed here, not held across the tile loop
  const int c = lane % CG, seg = lane / CG;
  const float* p = tile + ((seg / SEGS) * (64 / PARTS) + seg % SEGS) * S + c;
  double acc = 0.0;
#pragma unroll
  for (int q = 0; q < CG; ++q) {
    const double g = p[q * SEGS * S];
    acc = fma(g, g, acc);
  }
  return acc;
}

// What a wave of k_distill_regs knows of its columns and lanes, and the exchange of
// values between the waves of a row tile.
// OFF: unsigned 64 bits where a row's lanes are columns further apart than 32 cover.
template <int ROWS, int C, bool FULLC, typename OFF>
struct WaveTile {
  static constexpr int PARTS = 64 / ROWS;
  static constexpr bool STEP = FULLC || PARTS == 1;  // a column is a step of a uniform pointer
  const DistillArgs& a;
  float* red;  // [DISTILL_RED][W][64]
  int W, w, lane, rl, hb;
  int groups, rg;
  int j0, last;  // the wave's first column, and its last one from there

  // byte offset of column i of the lane's in row `loc` of the tile
  __device__ OFF at(int i, uint32_t loc, int64_t ld) const {
    if (PARTS == 1) return 4 * loc;
    if (FULLC) return 4 * (loc + (OFF)(hb * C) * (OFF)ld);
    const int c = hb * C + i;
    return 4 * (loc + (OFF)(c < last ? c : last) * (OFF)ld);
  }
  // Rows past the end are row n - 1 again: they store its own values once more
  // and stay out of the norms.
  __device__ void rows_of(int tile_no, int64_t& base, uint32_t& loc) const {
    base = ((int64_t)tile_no * groups + rg) * ROWS;
    const int64_t left = a.n - 1 - base;
    if (left < 0) {
      base = a.n - 1;
      loc = 0;
    } else {
      loc = rl < left ? rl : (uint32_t)left;
    }
  }
  __device__ void load(float (&x)[C], int64_t base, uint32_t loc) const {
    int64_t ld = a.ld_f;
    const float* p = a.F + (int64_t)j0 * ld + base;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      // seen anew at every step: 64-bit offsets of all columns would otherwise be formed ahead and held, spilled
      if (sizeof(OFF) == 8) asm volatile("" : "+s"(ld));
      x[i] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p) + at(i, loc, ld));
      if (STEP && (FULLC || i < last)) p += ld;
    }
  }
  __device__ void put(int q, float v) const { red[(q * W + w) * 64 + lane] = v; }
  __device__ float max_of(int q) const {
    float v = red[q * W * 64 + lane];
    for (int u = 1; u < W; ++u) v = fmaxf(v, red[(q * W + u) * 64 + lane]);
    return v;
  }
  __device__ float sum_of(int q) const {
    float v = red[q * W * 64 + lane];
    for (int u = 1; u < W; ++u) v += red[(q * W + u) * 64 + lane];
    return v;
  }
  // over the lanes of a row
  __device__ float part_sum(float v) const {
#pragma unroll
    for (int off = 32; off >= ROWS; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
  }
  __device__ float part_max(float v) const {
#pragma unroll
    for (int off = 32; off >= ROWS; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
  }
};

// The loss alone: the tile's scores go into LDS, a run of rows per column, where the
// waves find those of the classes that their share of the places lists (in memory each
// is a cache line of its own); the next tile's are on their way from the sums on.
template <int ROWS, int C, bool MIX, bool FULLC, typename OFF>
__device__ __forceinline__ void loss_wave(const RowArgs& r, char* lds, int w, int rg, int bx, int grid) {
  constexpr int PARTS = 64 / ROWS;
  const DistillArgs& a = r.a;
  const int W = r.waves, K = a.k;
  const int lane = threadIdx.x & 63, hb = lane / ROWS;
  float* scores = reinterpret_cast<float*>(lds);  // [d][ROWS]
  const int rl = lane & (ROWS - 1);
  const WaveTile<ROWS, C, FULLC, OFF> wt{a, scores + a.d * ROWS, W, w, lane, rl, hb, r.groups, rg, w * C * PARTS,
                                         a.d - 1 - w * C * PARTS};
  const int s0 = w * PARTS + hb, step = W * PARTS;
  int64_t base;
  uint32_t loc;
  wt.rows_of(bx, base, loc);
  float x[C];
  wt.load(x, base, loc);
  constexpr int AHEAD = 4;
  Place ahead[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    ahead[u] = Place{-1, 0.0f};
    if (s0 + u * step < K) ahead[u] = load_place(a, s0 + u * step, base + loc);
  }
  int next_y = a.w > 0.0 ? a.labels[base + loc] : -1;
  for (int t = bx; t < r.tiles; t += grid) {
    const int64_t row = base + loc;
    auto score = [&](int id) { return scores[(id >= 0 ? id : 0) * ROWS + rl]; };
    Place now[AHEAD];
    float vm = -INFINITY;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      now[u] = usable(a, ahead[u]);
      vm = fmaxf(vm, now[u].v);
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (FULLC || hb * C + i <= wt.last) scores[(wt.j0 + hb * C + i) * ROWS + rl] = x[i];
#pragma unroll 4
    for (int sl = s0 + AHEAD * step; sl < K; sl += step) vm = fmaxf(vm, usable(a, load_place(a, sl, row)).v);
    const int y = next_y < a.d ? next_y : -1;
    float m = x[0];
#pragma unroll
    for (int i = 1; i < C; ++i) m = fmaxf(m, x[i]);
    m = wt.part_max(m);
    vm = wt.part_max(vm);
    if (W > 1) {
      wt.put(0, m);
      wt.put(1, vm);
      lds_barrier();
      m = wt.max_of(0);
      vm = wt.max_of(1);
    } else {
      wave_sync();
    }
    m = fmaxf(m, -FLT_MAX);  // a row of -inf has z = -inf, not differences of infinities
    float s1 = 0.0f, sT = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const float z = x[i] - m;
      const bool live = FULLC || hb * C + i <= wt.last;
      const float e = exp2_hw(z * r.c2);
      sT += live ? e : 0.0f;
      if (MIX) {
        const float e1 = exp2_hw(z * LOG2E);
        s1 += live ? e1 : 0.0f;
      }
    }
    asm volatile("" : "+v"(sT), "+v"(s1));
    // the next tile, past the last one this one again
    int64_t nbase;
    uint32_t nloc;
    wt.rows_of(t + grid < r.tiles ? t + grid : t, nbase, nloc);
    wt.load(x, nbase, nloc);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * step < K) ahead[u] = load_place(a, s0 + u * step, nbase + nloc);
    if (a.w > 0.0) next_y = a.labels[nbase + nloc];
    float zs = 0.0f, us = 0.0f, ds = 0.0f;  // ds: sum e_t (a_c - m)
    auto add = [&](const Place& p, float score_c) {
      const float e = place_exp(r, p.v, vm, us);
      zs += e;
      if (p.id >= 0) ds += product(e, score_c - m);
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * step < K) add(now[u], score(now[u].id));
    for (int sl = s0 + AHEAD * step; sl < K; sl += step) {
      const Place p = usable(a, load_place(a, sl, row));
      add(p, score(p.id));
    }
    const float xy = w == 0 ? score(y) : 0.0f;
    zs = wt.part_sum(zs);
    us = wt.part_sum(us);
    ds = wt.part_sum(ds);
    sT = wt.part_sum(sT);
    if (MIX) s1 = wt.part_sum(s1);
    if (W > 1) {
      wt.put(2, zs);
      wt.put(3, us);
      wt.put(4, sT);
      if (MIX) wt.put(5, s1);
      wt.put(6, ds);
      lds_barrier();
    }
    if (w == 0) {
      if (W > 1) {
        zs = wt.sum_of(2);
        us = wt.sum_of(3);
        sT = wt.sum_of(4);
        if (MIX) s1 = wt.sum_of(5);
        ds = wt.sum_of(6);
      }
      if (!MIX) s1 = sT;
      const Teacher te = teacher_of(r, zs, us);
      const float A = y >= 0 ? r.w : 0.0f;
      const float dot = product(te.wt, ds) + (y >= 0 ? product(A, xy - m) : 0.0f);
      if (hb == 0) a.loss[row] = A * log_of(s1) + r.bt * (te.ent + te.Q * log_of(sT)) - dot;
    }
    if (W == 1) wave_sync();  // the scores are read before the next tile's
    base = nbase;
    loc = nloc;
  }
}

// MODE 1: the gradients; 2: the hessians or their row sums too.
template <int ROWS, int C, int MODE, bool MIX, bool FULLC, typename OFF>
__device__ __forceinline__ void distill_wave(const RowArgs& r, char* lds, int w, int rg, int bx, int grid) {
  constexpr int PARTS = 64 / ROWS;
  constexpr int CG = C < 16 ? C : 16, S = CG + 4, NG = C / CG;
  constexpr bool STEP = WaveTile<ROWS, C, FULLC, OFF>::STEP;
  const DistillArgs& a = r.a;
  const int W = r.waves, K = a.k;
  const int lane = threadIdx.x & 63, rl = lane & (ROWS - 1), hb = lane / ROWS;
  Listed* ent = reinterpret_cast<Listed*>(lds);
  const int j0 = w * C * PARTS;  // the wave's first column
  const int jl = j0 + hb * C;    // the lane's first column
  WaveTile<ROWS, C, FULLC, OFF> wt{a, reinterpret_cast<float*>(lds) + 2 * K * ROWS, W, w, lane, rl, hb, r.groups, rg, j0,
                              a.d - 1 - j0};
  int& last = wt.last;
  float* tile = wt.red + DISTILL_RED * W * 64 + w * distill_tile_floats(C);
  float* trow = tile + lane * S;
  auto load_at = [](const float* p, OFF bytes) {
    return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p) + bytes);
  };
  auto store_at = [](float* p, OFF bytes, float v) {
    *reinterpret_cast<float*>(reinterpret_cast<char*>(p) + bytes) = v;
  };
  int64_t base;
  uint32_t loc;
  wt.rows_of(bx, base, loc);
  float x[C];
  wt.load(x, base, loc);
  // the first places of the wave, and the labels, a tile ahead
  constexpr int AHEAD = PARTS == 1 ? 4 : 2;
  const int s0 = w * PARTS + hb;
  Place ahead[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (s0 + u * W * PARTS < K) ahead[u] = load_place(a, s0 + u * W * PARTS, base + loc);
  int next_y = a.w > 0.0 ? a.labels[base + loc] : -1;
  double total[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) total[g] = 0.0;

  for (int t = bx; t < r.tiles; t += grid) {
    const int64_t row = base + loc;
    const bool ok = ((int64_t)t * r.groups + rg) * ROWS + rl < a.n;
    // the wave's places: class and value into LDS
    float vm = -INFINITY;
    auto stage = [&](int sl, const Place& p) {
      ent[sl * ROWS + rl] = Listed{p.id, p.v};
      vm = fmaxf(vm, p.v);
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * W * PARTS < K) stage(s0 + u * W * PARTS, usable(a, ahead[u]));
    for (int sl = s0 + AHEAD * W * PARTS; sl < K; sl += W * PARTS) stage(sl, usable(a, load_place(a, sl, row)));
    const int y = next_y < a.d ? next_y : -1;
    const float A = y >= 0 ? r.w : 0.0f;
    float m = x[0];
#pragma unroll
    for (int i = 1; i < C; ++i) m = fmaxf(m, x[i]);
    m = wt.part_max(m);
    vm = wt.part_max(vm);
    if (W > 1) {
      wt.put(0, m);
      wt.put(1, vm);
      lds_barrier();
      m = wt.max_of(0);
      vm = wt.max_of(1);
    } else {
      wave_sync();
    }
    m = fmaxf(m, -FLT_MAX);
    float zs = 0.0f, us = 0.0f, s1 = 0.0f, sT = 0.0f;
    for (int sl = s0; sl < K; sl += W * PARTS) {
      const float e = place_exp(r, ent[sl * ROWS + rl].e, vm, us);
      ent[sl * ROWS + rl].e = e;
      zs += e;
    }
    // the compiler sees the last column anew: the tests of columns would otherwise
    // be held as lane masks, spilled, across the tile loop
    asm volatile("" : "+s"(last));
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const float z = x[i] - m;
      const bool live = FULLC || hb * C + i <= last;
      const float e = exp2_hw(z * r.c2);
      sT += live ? e : 0.0f;
      if (MIX) {
        const float e1 = exp2_hw(z * LOG2E);
        s1 += live ? e1 : 0.0f;
      }
    }
    zs = wt.part_sum(zs);
    us = wt.part_sum(us);
    sT = wt.part_sum(sT);
    if (MIX) s1 = wt.part_sum(s1);
    if (W > 1) {
      wt.put(2, zs);
      wt.put(3, us);
      wt.put(4, sT);
      if (MIX) wt.put(5, s1);
      lds_barrier();
      zs = wt.sum_of(2);
      us = wt.sum_of(3);
      sT = wt.sum_of(4);
      if (MIX) s1 = wt.sum_of(5);
    } else {
      wave_sync();
    }
    if (!MIX) s1 = sT;
    const Teacher te = teacher_of(r, zs, us);
    const float BQ = r.b * te.Q;
    const float iT = inverse(sT), i1 = inverse(s1);
    const float kT = (MIX ? BQ : A + BQ) * iT, k1 = A * i1;          // coefficients of the exponentials in g
    const float hT = MIX ? BQ * r.inv_t : A + BQ * r.inv_t, h1 = A;  // of p (1 - p) in h

    // the exponentials are formed again below: kept, they take the registers of two rows more
    asm volatile("" : "+v"(m));
    int64_t nbase;
    uint32_t nloc;
    wt.rows_of(t + grid < r.tiles ? t + grid : t, nbase, nloc);
    // the next tile's places and labels, which arrive while this one goes out
    const int64_t nrow = nbase + nloc;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * W * PARTS < K) ahead[u] = load_place(a, s0 + u * W * PARTS, nrow);
    if (a.w > 0.0) next_y = a.labels[nrow];
    float hsum = 0.0f, dot = 0.0f;
    {
      // the leading dimensions are seen anew at every step: all column offsets
      // would otherwise be formed before the loop and held, spilled, across it
      int64_t ld_f = a.ld_f, ld_g = a.ld_g, ld_h = a.ld_h;
      const float* Fc = a.F + (int64_t)j0 * ld_f + nbase;
      float* Gc = a.G + (int64_t)j0 * ld_g + base;
      float* Hc = a.hess ? a.hess + (int64_t)j0 * ld_h + base : nullptr;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        wave_sync();  // the norms of the group before are read
        float4* t4 = reinterpret_cast<float4*>(trow);
#pragma unroll
        for (int q = 0; q < CG / 4; ++q) t4[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        add_targets<CG, ROWS>(ent, K, rl, jl + g * CG, te.wt, y, A, trow);
#pragma unroll
        for (int q = 0; q < CG / 4; ++q) {
          const float4 t4v = t4[q];
          const float tv[4] = {t4v.x, t4v.y, t4v.z, t4v.w};
          float gv[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int i = g * CG + q * 4 + u;
            asm volatile("" : "+s"(ld_f), "+s"(ld_g), "+s"(last));
            const bool live = FULLC || hb * C + i <= last;
            const float z = x[i] - m;
            const float eT = exp2_hw(z * r.c2);
            float gr = fmaf(kT, eT, -tv[u]);
            float e1 = 0.0f;
            if (MIX) {
              e1 = exp2_hw(z * LOG2E);
              gr = fmaf(k1, e1, gr);
            }
            dot += product(tv[u], z);
            if (live) store_at(Gc, wt.at(i, loc, ld_g), gr);
            if (MODE == 2) {
              const float pT = eT * iT;
              float h = hT * fmaf(-pT, pT, pT);
              if (MIX) {
                const float p1 = e1 * i1;
                h = fmaf(h1, fmaf(-p1, p1, p1), h);
              }
              hsum += live ? h : 0.0f;
              if (a.hess) {
                asm volatile("" : "+s"(ld_h));
                if (live) store_at(Hc, wt.at(i, loc, ld_h), h);
                if (STEP && (FULLC || i < last)) Hc += ld_h;
              }
            }
            gv[u] = ok && live ? gr : 0.0f;
            x[i] = load_at(Fc, wt.at(i, nloc, ld_f));
            if (STEP && (FULLC || i < last)) {
              Fc += ld_f;
              Gc += ld_g;
            }
          }
          t4[q] = make_float4(gv[0], gv[1], gv[2], gv[3]);
          // the sums are taken here, whether or not they are asked for: put off to
          // where they are, their terms are held, spilled, until then
          asm volatile("" : "+v"(dot));
          if (MODE == 2) asm volatile("" : "+v"(hsum));
          __builtin_amdgcn_sched_barrier(0);
        }
        if (r.npart) {
          wave_sync();
          total[g] += tile_norms<CG, PARTS>(tile, lane);
        }
      }
    }
    if (W > 1 || a.loss || a.h_row) {
      if (a.loss) dot = wt.part_sum(dot);
      if (MODE == 2 && a.h_row) hsum = wt.part_sum(hsum);
      if (W > 1) {
        if (a.loss) wt.put(6, dot);
        if (MODE == 2 && a.h_row) wt.put(7, hsum);
        lds_barrier();  // and all waves are through with the places
      }
      if (w == 0 && hb == 0) {
        if (a.loss) {
          if (W > 1) dot = wt.sum_of(6);
          a.loss[row] = A * log_of(s1) + r.bt * (te.ent + te.Q * log_of(sT)) - dot;
        }
        if (MODE == 2 && a.h_row) {
          if (W > 1) hsum = wt.sum_of(7);
          a.h_row[row] = hsum * (1.0f / (float)a.d);
        }
      }
    }
    if (W == 1) wave_sync();  // the places are read before the next tile's
    base = nbase;
    loc = nloc;
  }
  if (r.npart) {
    // the row segments of a column, in order
    const int c = lane % CG;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      double s = total[g];
      for (int off = CG; off < 64 / PARTS; off <<= 1) s += __shfl_xor(s, off, 64);
      const int col = jl + g * CG + c;
      if ((lane & (64 / PARTS - 1)) < CG && col < a.d)
        r.npart[(int64_t)col * r.parts + bx * r.groups + rg] = s;
    }
  }
}

// Blocks go to the 8 XCDs in turn; each XCD takes a run of neighbouring tiles, which
// share cache lines where columns do not start on a line.  The launch has a multiple
// of 8 blocks.
template <int ROWS, int C, int MODE, bool MIX, typename OFF>
__global__ void __launch_bounds__(64 * DISTILL_MAX_WAVES) k_distill_regs(RowArgs r, int grid) {
  extern __shared__ __align__(16) char smem[];
  const int bx = (int)(blockIdx.x & 7) * ((grid + 7) >> 3) + (int)(blockIdx.x >> 3);
  if (bx >= grid) return;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wv / r.waves, w = wv - rg * r.waves;
  const int bytes =
      MODE == 0 ? r.tile_bytes : 4 * (2 * r.a.k * ROWS + DISTILL_RED * r.waves * 64 + r.waves * distill_tile_floats(C));
  char* lds = smem + rg * bytes;
  const bool full = (w + 1) * C * (64 / ROWS) <= r.a.d;  // all columns of the wave exist
  if constexpr (MODE == 0) {
    if (full) loss_wave<ROWS, C, MIX, true, OFF>(r, lds, w, rg, bx, grid);
    else loss_wave<ROWS, C, MIX, false, OFF>(r, lds, w, rg, bx, grid);
  } else {
    if (full) distill_wave<ROWS, C, MODE, MIX, true, OFF>(r, lds, w, rg, bx, grid);
    else distill_wave<ROWS, C, MODE, MIX, false, OFF>(r, lds, w, rg, bx, grid);
  }
}

// ---------------------------------------------------------------- the loss of many rows
// One lane per row, one wave per 64-row tile: a running maximum and sums over the
// columns in order, then the places, eight at a time, twice: their largest value, which
// the sums are relative to (a place is a target or not by its distance from it, wherever
// in the list it stands), then the sums.  No wave waits for another.
template <bool MIX>
__global__ void __launch_bounds__(256) k_loss_by_lane(RowArgs r) {
  const DistillArgs& a = r.a;
  const int lane = threadIdx.x & 63;
  const int64_t base = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 64;
  if (base >= a.n) return;
  const int64_t left = a.n - 1 - base;  // rows past the end read row n - 1 and store nothing
  const int loc = lane < left ? lane : (int)left;
  const int64_t row = base + loc;
  const float* F = a.F + base;
  float m = -FLT_MAX, s1 = 0.0f, sT = 0.0f;
  float x[2][16];
  auto load = [&](float (&to)[16], int j) {
    const float* p = F + (int64_t)j * a.ld_f;
    if (j + 16 <= a.d) {
#pragma unroll
      for (int i = 0; i < 16; ++i, p += a.ld_f) to[i] = p[loc];
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i, p += a.ld_f) {
        to[i] = -INFINITY;
        if (j + i < a.d) to[i] = p[loc];
      }
    }
  };
  auto step = [&](const float (&now)[16]) {
    float mn = m;
#pragma unroll
    for (int i = 0; i < 16; ++i) mn = fmaxf(mn, now[i]);
    float a1 = 0.0f, aT = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float z = now[i] - mn;
      aT += exp2_hw(z * r.c2);
      if (MIX) a1 += exp2_hw(z * LOG2E);
      if (i % 4 == 3) asm volatile("" : "+v"(aT), "+v"(a1));  // here and now: put off, the terms take registers
    }
    sT = fmaf(sT, exp2_hw((m - mn) * r.c2), aT);
    if (MIX) s1 = fmaf(s1, exp2_hw((m - mn) * LOG2E), a1);
    m = mn;
  };
  load(x[0], 0);
  for (int j = 0; j < a.d; j += 32) {
    wait_loads();
    if (j + 16 < a.d) load(x[1], j + 16);
    step(x[0]);
    if (j + 16 < a.d) {
      wait_loads();
      if (j + 32 < a.d) load(x[0], j + 32);
      step(x[1]);
    }
  }
  if (!MIX) s1 = sT;
  float vm = -INFINITY, zs = 0.0f, us = 0.0f, ds = 0.0f;
  auto places = [&](Place (&p)[8], int s) {
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = s + u < a.k ? load_place(a, s + u, row) : Place{-1, 0.0f};
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = usable(a, p[u]);
  };
  Place p[8];
  // back to front, so that a list of up to eight is read once (log probabilities need no largest value)
  for (int s = a.teacher == SB_TEACHER_LOGITS ? (a.k - 1) & ~7 : 0; s >= 0; s -= 8) {
    places(p, s);
#pragma unroll
    for (int u = 0; u < 8; ++u) vm = fmaxf(vm, p[u].v);
  }
  for (int s = 0; s < a.k; s += 8) {
    if (s > 0) places(p, s);
    float xc[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) xc[u] = p[u].id >= 0 ? F[(int64_t)p[u].id * a.ld_f + loc] : m;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float e = place_exp(r, p[u].v, vm, us);
      zs += e;
      ds += product(e, xc[u] - m);
    }
  }
  const Teacher te = teacher_of(r, zs, us);
  float dot = product(te.wt, ds), A = 0.0f;
  if (a.w > 0.0) {
    const int y = a.labels[row];
    if (y >= 0 && y < a.d) {
      A = r.w;
      dot += product(A, F[(int64_t)y * a.ld_f + loc] - m);
    }
  }
  if (lane <= left) a.loss[row] = A * log_of(s1) + r.bt * (te.ent + te.Q * log_of(sT)) - dot;
}

// ---------------------------------------------------------------- wider rows
constexpr int WIDE_WAVES = 4;

// XCD x takes a run of units (range, row tile or slot), so that neighbouring tiles of a
// range, which share cache lines where columns do not start on a line, meet in its L2.
__device__ inline int unit_of(int units) {
  return (int)(blockIdx.x & 7) * ((units + 7) >> 3) + (int)(blockIdx.x >> 3);
}

// Maximum and sums of exponentials of a 64-row tile's columns in one range: the
// waves' running maxima and sums, joined in LDS.
template <bool MIX>
__global__ void __launch_bounds__(64 * WIDE_WAVES) k_distill_stats(RowArgs r, int units) {
  __shared__ float red[3][WIDE_WAVES][64];
  const DistillArgs& a = r.a;
  const int unit = unit_of(units);
  if (unit >= units) return;
  const int range = unit / r.tiles;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t base = (int64_t)(unit - range * r.tiles) * 64;
  const int64_t left = a.n - 1 - base;
  const int loc = lane < left ? lane : (int)left;
  const int per = r.cols / WIDE_WAVES, j0 = range * r.cols + w * per;
  const int j1 = j0 + per < a.d ? j0 + per : a.d;
  float m = -FLT_MAX, s1 = 0.0f, sT = 0.0f;
  // two sets of registers in turn: one is read while the other is summed
  float x[2][16];
  auto load = [&](float (&to)[16], int j) {
#pragma unroll
    for (int i = 0; i < 16; ++i) to[i] = (a.F + (int64_t)(j + i < j1 ? j + i : j1 - 1) * a.ld_f + base)[loc];
  };
  auto step = [&](const float (&now)[16], float (&next)[16], int j) {
    wait_loads();
    if (j + 16 < j1) load(next, j + 16);
    float mn = m;
#pragma unroll
    for (int i = 0; i < 16; ++i) mn = fmaxf(mn, now[i]);
    float a1 = 0.0f, aT = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float z = now[i] - mn;
      const bool live = j + i < j1;  // columns past the last repeat it
      aT += live ? exp2_hw(z * r.c2) : 0.0f;
      if (MIX) a1 += live ? exp2_hw(z * LOG2E) : 0.0f;
    }
    sT = fmaf(sT, exp2_hw((m - mn) * r.c2), aT);
    if (MIX) s1 = fmaf(s1, exp2_hw((m - mn) * LOG2E), a1);
    m = mn;
  };
  if (j0 < j1) load(x[0], j0);
  for (int j = j0; j < j1; j += 32) {
    step(x[0], x[1], j);
    if (j + 16 < j1) step(x[1], x[0], j + 16);
  }
  red[0][w][lane] = m;
  red[1][w][lane] = sT;
  red[2][w][lane] = s1;
  __syncthreads();
  if (w != 0 || lane > left) return;
  float mm = red[0][0][lane];
#pragma unroll
  for (int u = 1; u < WIDE_WAVES; ++u) mm = fmaxf(mm, red[0][u][lane]);
  sT = s1 = 0.0f;
#pragma unroll
  for (int u = 0; u < WIDE_WAVES; ++u) {
    const float z = red[0][u][lane] - mm;
    sT += red[1][u][lane] * exp2_hw(z * r.c2);
    if (MIX) s1 += red[2][u][lane] * exp2_hw(z * LOG2E);
  }
  float* out = r.stats + (int64_t)range * 3 * a.n + base + lane;
  out[0] = mm;
  out[a.n] = sT;
  if (MIX) out[2 * a.n] = s1;
}

// What the rows' outputs need besides their scores: the joined statistics, the
// targets of the listed places and the loss (with gradients, its part without scores).  64 rows per block, ranges and places
// shared out among its waves.  In the workspace of n floats each:
//   row[0] max, row[1] coefficient of 2^(z c2) in g, row[2] of 2^(z log2 e),
//   row[3] 1 / sT, row[4] 1 / s1, row[5] Q, then the targets of the K places.
constexpr int ROW_VALUES = 6;

template <bool MIX, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_distill_rows(RowArgs r) {
  __shared__ float red[6][WAVES][64];
  const DistillArgs& a = r.a;
  const int K = a.k;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t base = (int64_t)blockIdx.x * 64;
  const int64_t left = a.n - 1 - base;  // rows past the end are row n - 1 again, whose values they store once more
  const int64_t row = base + (lane < left ? lane : left);
  float* targets = r.row + ROW_VALUES * a.n + row;
  auto sum_of = [&](int q) {
    float s = red[q][0][lane];
#pragma unroll
    for (int u = 1; u < WAVES; ++u) s += red[q][u][lane];
    return s;
  };
  auto max_of = [&](int q) {
    float s = red[q][0][lane];
#pragma unroll
    for (int u = 1; u < WAVES; ++u) s = fmaxf(s, red[q][u][lane]);
    return s;
  };
  float m = -INFINITY, vm = -INFINITY;
#pragma unroll 4
  for (int q = w; q < r.ranges; q += WAVES) m = fmaxf(m, r.stats[(int64_t)q * 3 * a.n + row]);
#pragma unroll 4
  for (int s = w; s < K; s += WAVES) vm = fmaxf(vm, usable(a, load_place(a, s, row)).v);
  red[0][w][lane] = m;
  red[1][w][lane] = vm;
  __syncthreads();
  m = max_of(0);
  vm = max_of(1);
  float sT = 0.0f, s1 = 0.0f, zs = 0.0f, us = 0.0f;
#pragma unroll 4
  for (int q = w; q < r.ranges; q += WAVES) {
    const float* st = r.stats + (int64_t)q * 3 * a.n + row;
    const float z = st[0] - m;
    sT = fmaf(st[a.n], exp2_hw(z * r.c2), sT);
    if (MIX) s1 = fmaf(st[2 * a.n], exp2_hw(z * LOG2E), s1);
  }
#pragma unroll 4
  for (int s = w; s < K; s += WAVES) zs += place_exp(r, usable(a, load_place(a, s, row)).v, vm, us);
  red[2][w][lane] = sT;
  red[3][w][lane] = s1;
  red[4][w][lane] = zs;
  red[5][w][lane] = us;
  __syncthreads();
  sT = sum_of(2);
  s1 = MIX ? sum_of(3) : sT;
  zs = sum_of(4);
  us = sum_of(5);
  const Teacher te = teacher_of(r, zs, us);
  int y = -1;
  if (a.w > 0.0) {
    y = a.labels[row];
    if (y >= a.d) y = -1;
  }
  const float A = y >= 0 ? r.w : 0.0f;
  float dot = 0.0f, unused = 0.0f;
  for (int s = w; s < K; s += WAVES) {
    const Place p = usable(a, load_place(a, s, row));
    const float t = te.wt * place_exp(r, p.v, vm, unused);
    if (a.G) targets[s * a.n] = t;
    // with gradients the ranges, which have the scores at hand, form the products
    if (!a.G && p.id >= 0) dot += product(t, a.F[(int64_t)p.id * a.ld_f + row] - m);
  }
  if (a.loss && a.G) {
    if (w == 0) a.loss[row] = A * log_of(s1) + r.bt * (te.ent + te.Q * log_of(sT));
  } else if (a.loss) {
    if (w == 0 && y >= 0) dot += product(A, a.F[(int64_t)y * a.ld_f + row] - m);
    red[0][w][lane] = dot;  // the maxima are read before the barrier above
    __syncthreads();
    if (w == 0) a.loss[row] = A * log_of(s1) + r.bt * (te.ent + te.Q * log_of(sT)) - sum_of(0);
  }
  if (w == 0 && a.G) {
    const float BQ = r.b * te.Q, iT = inverse(sT), i1 = inverse(s1);
    float* out = r.row + row;
    out[0] = m;
    out[a.n] = (MIX ? BQ : A + BQ) * iT;
    out[2 * a.n] = A * i1;
    out[3 * a.n] = iT;
    out[4 * a.n] = i1;
    out[5 * a.n] = te.Q;
  }
}

// The outputs of a 64-row tile's columns in one range.
template <int MODE, bool MIX>
__global__ void __launch_bounds__(64 * WIDE_WAVES) k_distill_range(RowArgs r, int units) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[2][WIDE_WAVES][64];
  const DistillArgs& a = r.a;
  const int K = a.k;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Listed* ent = reinterpret_cast<Listed*>(smem);  // [K][64]
  float* tile = reinterpret_cast<float*>(smem) + 2 * K * 64 + w * distill_tile_floats(16);
  float* trow = tile + lane * 20;
  const int unit = unit_of(units);
  if (unit >= units) return;
  const int range = unit / r.slots, slot = unit - range * r.slots;
  const int per = r.cols / WIDE_WAVES, j0 = range * r.cols + w * per;
  const int cols = a.d - j0 < per ? a.d - j0 : per;  // may be <= 0
  for (int64_t t = slot; t < r.tiles; t += r.slots) {
    const int64_t base = t * 64;
    const int64_t left_rows = a.n - 1 - base;
    const int loc = lane < left_rows ? lane : (int)left_rows;
    const bool ok = lane <= left_rows;
    const int64_t row = base + loc;
    float nx[16];
    auto load = [&](int c0) {
      const int last = cols - 1 - c0;
#pragma unroll
      for (int i = 0; i < 16; ++i) nx[i] = (a.F + (int64_t)(j0 + c0 + (i < last ? i : last)) * a.ld_f + base)[loc];
    };
    if (cols > 0) load(0);
#pragma unroll 4
    for (int s = w; s < K; s += WIDE_WAVES)
      ent[s * 64 + lane] = Listed{a.t_id[s * a.ld_t + row], r.row[(ROW_VALUES + s) * a.n + row]};
    const float* rv = r.row + row;
    const float m = rv[0], kT = rv[a.n], k1 = rv[2 * a.n], iT = rv[3 * a.n], i1 = rv[4 * a.n], Q = rv[5 * a.n];
    int y = -1;
    if (a.w > 0.0) {
      y = a.labels[row];
      if (y >= a.d) y = -1;
    }
    const float A = y >= 0 ? r.w : 0.0f;
    const float hQ = r.b * Q * r.inv_t;
    const float hT = MIX ? hQ : A + hQ, h1 = A;
    __syncthreads();
    float hsum = 0.0f, dot = 0.0f;
    // the places of the wave's columns, a bit each; every group takes its own out
    uint64_t mine = 0;
#pragma unroll 8
    for (int s = 0; s < K; ++s)
      mine |= (uint64_t)(column_from(ent[s * 64 + lane].id, j0) < (uint32_t)(cols > 0 ? cols : 0)) << s;
    // 16 columns from c0; all of them exist (FULL), or those up to `last`
    auto group = [&](auto full, int c0, int last) {
      constexpr bool FULL = decltype(full)::value;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = nx[i];
      if (c0 + 16 < cols) load(c0 + 16);
      wave_sync();
      float4* t4 = reinterpret_cast<float4*>(trow);
#pragma unroll
      for (int q = 0; q < 4; ++q) t4[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      uint32_t seen = 0;
      uint64_t left = mine;
      while (left) {
        const int s = __builtin_ctzll(left);
        left &= left - 1;
        const Listed p = ent[s * 64 + lane];
        const uint32_t c = column_from(p.id, j0 + c0);
        if (c < 16) mine &= ~(uint64_t(1) << s);
        put_target<16>(trow, seen, c, p.e);
      }
      if (y >= 0) put_target<16>(trow, seen, column_from(y, j0 + c0), A);
      float* Gc = a.G + (int64_t)(j0 + c0) * a.ld_g + base;
      float* Hc = MODE == 2 && a.hess ? a.hess + (int64_t)(j0 + c0) * a.ld_h + base : nullptr;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 t4v = t4[q];
        const float tv[4] = {t4v.x, t4v.y, t4v.z, t4v.w};
        float gv[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int i = q * 4 + u;
          const bool live = FULL || i <= last;
          const float z = x[i] - m;
          const float eT = exp2_hw(z * r.c2);
          float gr = fmaf(kT, eT, -tv[u]);
          float e1 = 0.0f;
          if (MIX) {
            e1 = exp2_hw(z * LOG2E);
            gr = fmaf(k1, e1, gr);
          }
          dot += product(tv[u], z);  // columns past the last repeat it without a target
          // rows past the end store row n - 1's own values once more
          if (live) Gc[loc] = gr;
          Gc += a.ld_g;
          if (MODE == 2) {
            const float pT = eT * iT;
            float h = hT * fmaf(-pT, pT, pT);
            if (MIX) {
              const float p1 = e1 * i1;
              h = fmaf(h1, fmaf(-p1, p1, p1), h);
            }
            hsum += live ? h : 0.0f;
            if (a.hess) {
              if (live) Hc[loc] = h;
              Hc += a.ld_h;
            }
          }
          gv[u] = ok && live ? gr : 0.0f;
        }
        t4[q] = make_float4(gv[0], gv[1], gv[2], gv[3]);
      }
      if (r.npart) {
        wave_sync();
        double s = tile_norms<16, 1>(tile, lane);
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        if (lane < 16 && lane <= last) {
          // the slot belongs to this lane: its first tile writes it, the others add in order
          double* pp = r.npart + (int64_t)(j0 + c0 + lane) * r.parts + slot;
          *pp = t == slot ? s : *pp + s;
        }
      }
    };
    for (int c0 = 0; c0 < cols; c0 += 16) {
      const int last = cols - 1 - c0;
      if (last >= 15) group(std::true_type(), c0, last);
      else group(std::false_type(), c0, last);
    }
    if (a.loss || (MODE == 2 && a.h_row)) {
      red[0][w][lane] = dot;
      red[1][w][lane] = hsum;
      __syncthreads();
      if (w == 0 && ok) {  // the ranges' statistics are read by now
        for (int u = 1; u < WIDE_WAVES; ++u) {
          dot += red[0][u][lane];
          hsum += red[1][u][lane];
        }
        r.stats[(int64_t)range * 2 * a.n + row] = dot;
        r.stats[((int64_t)range * 2 + 1) * a.n + row] = hsum;
      }
    }
    __syncthreads();  // the places and exchanged values are read before the next tile's
  }
}

// The ranges' sums of a row: what its targets take off the loss, and its hessians' mean.
__global__ void __launch_bounds__(256) k_distill_join(const float* sums, int ranges, int64_t n, int d, float* loss,
                                                      float* h_row) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float dot = 0.0f, h = 0.0f;
  for (int q = 0; q < ranges; ++q) {
    dot += sums[(int64_t)q * 2 * n + i];
    h += sums[((int64_t)q * 2 + 1) * n + i];
  }
  if (loss) loss[i] -= dot;
  if (h_row) h_row[i] = h * (1.0f / (float)d);
}

// ---------------------------------------------------------------- the loss at high temperatures
// The loss's terms are about T^2 log d, and what they add up to is about the squared
// differences of scores and values: in fp32 all of it is lost at T = 1000.  Their parts of
// order 1, 1 / T and 1 / T^2 are kept apart.  With x_j = (a_j - m) / T,
//   exp(x) = 1 + x + phi(x),  phi(x) = x^2 / 2 + x^3 / 6 + ...,
// 1 + x is summed in fp64 from the scores as they are, and phi, formed in fp32, carries
// fp32 roundings of x^2: after T^2 those of the squared differences.  Where x < -1/2 the
// exponential itself is as small as its roundings ask for.  The list's exponentials and
// all sums and logarithms of a row are fp64.
// Up to T = HOT the fp32 forms above lose at most four bits more than they do at T = 1.
// Bound by vector instructions (some 35 per score, two of them in fp64; 0.7 of the issue
// slots at 20,001 x 5003) and, in lists of many rows, by the listed scores, a cache line each: 1,000,003 x 100 with 10 places
// 213 us (107 by the fp32 form), 300,007 x 1000 with 25 397 (342), 20,001 x 5003 with 64
// 170 (111); 64 x 60,000 37 (23), of which a second launch is part.  A call for gradients
// reads the scores once more for it.
constexpr double HOT = 4.0;

struct HotArgs {
  RowArgs r;
  double inv_t, bt;  // 1 / T, (1 - w) T^2
  int waves, tiles;
  int ranges, cols;  // k_hot_stats: column ranges; 0 if there are none
  double* S;         // [ranges][n]
  float2* ms;        // [ranges][n]: maximum, sum at T = 1
};

struct HotSums {
  float m = -FLT_MAX, s1 = 0.0f;
  double S = 0.0;  // sum exp((a - m) / T)
};

// exp(x) - 1 - x for |x| <= 1/2: the Taylor series to x^9 / 9! (the next term is 2^-25 of it)
__device__ inline float phi(float x) {
  float p = 1.0f / 362880.0f;
  p = fmaf(p, x, 1.0f / 40320.0f);
  p = fmaf(p, x, 1.0f / 5040.0f);
  p = fmaf(p, x, 1.0f / 720.0f);
  p = fmaf(p, x, 1.0f / 120.0f);
  p = fmaf(p, x, 1.0f / 24.0f);
  p = fmaf(p, x, 1.0f / 6.0f);
  p = fmaf(p, x, 0.5f);
  return x * x * p;
}
__device__ inline double exp_fine(double x) {  // x <= 0
  const float f = (float)x;
  return f >= -0.5f ? 1.0 + (x + (double)phi(f)) : (double)exp2_hw(f * LOG2E);
}

// h joined with the sums o of other columns of the row.
template <bool MIX>
__device__ inline void hot_add(HotSums& h, const HotSums& o, double inv_t) {
  const float mn = fmaxf(h.m, o.m);
  h.S = h.S * exp_fine(((double)h.m - mn) * inv_t) + o.S * exp_fine(((double)o.m - mn) * inv_t);
  if (MIX) h.s1 = h.s1 * exp2_hw((h.m - mn) * LOG2E) + o.s1 * exp2_hw((o.m - mn) * LOG2E);
  h.m = mn;
}

// The sums of columns j0 .. j1 - 1 of a lane's row; the next 16 are on their way meanwhile.
template <bool MIX>
__device__ inline HotSums hot_columns(const HotArgs& h, const float* F, int loc, int j0, int j1) {
  const int64_t ld = h.r.a.ld_f;
  const float inv_t = h.r.inv_t, c2 = h.r.c2;
  HotSums o;
  float x[2][16];
  auto load = [&](float (&to)[16], int j) {
    const float* p = F + (int64_t)j * ld;
    if (j + 16 <= j1) {
#pragma unroll
      for (int i = 0; i < 16; ++i, p += ld) to[i] = p[loc];
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i, p += ld) {
        to[i] = -INFINITY;
        if (j + i < j1) to[i] = p[loc];
      }
    }
  };
  auto step = [&](const float (&now)[16]) {
    float mn = o.m;
#pragma unroll
    for (int i = 0; i < 16; ++i) mn = fmaxf(mn, now[i]);
    if (__any(mn > o.m)) {
      o.S *= exp_fine(((double)o.m - mn) * h.inv_t);
      if (MIX) o.s1 *= exp2_hw((o.m - mn) * LOG2E);
      o.m = mn;
    }
    int near = 0;
    double sum = 0.0;  // of the near scores
    float f = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float z = now[i] - mn, v = z * inv_t;
      const bool is_near = v >= -0.5f;
      const float p = phi(v), e = exp2_hw(z * c2);
      f += is_near ? p : e;
      sum += (double)(is_near ? now[i] : 0.0f);
      near += is_near;
      if (MIX) s1 += exp2_hw(z * LOG2E);
      if (i % 4 == 3) asm volatile("" : "+v"(f), "+v"(s1), "+v"(sum));  // here and now: put off, the terms take registers
    }
    o.S += ((double)near + (sum - (double)near * (double)mn) * h.inv_t) + (double)f;
    if (MIX) o.s1 += s1;
  };
  if (j0 < j1) load(x[0], j0);
  for (int j = j0; j < j1; j += 32) {
    wait_loads();
    if (j + 16 < j1) load(x[1], j + 16);
    step(x[0]);
    if (j + 16 < j1) {
      wait_loads();
      if (j + 32 < j1) load(x[0], j + 32);
      step(x[1]);
    }
  }
  return o;
}

// What the waves of a block exchange, 64 values each.
struct HotShared {
  double* d;  // [4][waves][64]
  float* f;   // [3][waves][64]
  int waves;
  __device__ HotShared(char* lds, int waves)
      : d(reinterpret_cast<double*>(lds)), f(reinterpret_cast<float*>(lds + 4 * 8 * 64 * waves)), waves(waves) {}
  __device__ double& at(int q, int w, int lane) const { return d[(q * waves + w) * 64 + lane]; }
  __device__ float& at_f(int q, int w, int lane) const { return f[(q * waves + w) * 64 + lane]; }
  __device__ double sum(int q, int lane) const {
    double s = at(q, 0, lane);
    for (int u = 1; u < waves; ++u) s += at(q, u, lane);
    return s;
  }
};
constexpr int HOT_WAVE_BYTES = 64 * (4 * 8 + 3 * 4);

template <bool MIX>
__device__ inline HotSums hot_join(const HotArgs& h, const HotShared& sh, HotSums o, int w, int lane) {
  if (sh.waves == 1) return o;
  sh.at(0, w, lane) = o.S;
  sh.at_f(0, w, lane) = o.m;
  sh.at_f(1, w, lane) = o.s1;
  __syncthreads();
  o = HotSums();
  for (int u = 0; u < sh.waves; ++u)
    hot_add<MIX>(o, HotSums{sh.at_f(0, u, lane), sh.at_f(1, u, lane), sh.at(0, u, lane)}, h.inv_t);
  return o;
}

// A 64-row tile's sums in one column range, for k_hot_loss of few rows with many classes.
template <bool MIX>
__global__ void __launch_bounds__(64 * WIDE_WAVES) k_hot_stats(HotArgs h) {
  extern __shared__ __align__(16) char smem[];
  const HotShared sh(smem, WIDE_WAVES);
  const DistillArgs& a = h.r.a;
  const int range = blockIdx.x / h.tiles, tile = blockIdx.x - range * h.tiles;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t base = (int64_t)tile * 64, left = a.n - 1 - base;
  const int loc = lane < left ? lane : (int)left;
  const int per = h.cols / WIDE_WAVES, j0 = range * h.cols + w * per;
  const HotSums o = hot_join<MIX>(h, sh, hot_columns<MIX>(h, a.F + base, loc, j0, j0 + per < a.d ? j0 + per : a.d), w, lane);
  if (w != 0 || lane > left) return;
  const int64_t at = (int64_t)range * a.n + base + lane;
  h.S[at] = o.S;
  h.ms[at] = make_float2(o.m, o.s1);
}

// A 64-row tile per block: its columns (or the ranges' sums) and its list places shared
// out among the waves.
template <bool MIX>
__global__ void __launch_bounds__(64 * DISTILL_MAX_WAVES) k_hot_loss(HotArgs h) {
  extern __shared__ __align__(16) char smem[];
  const HotShared sh(smem, h.waves);
  const DistillArgs& a = h.r.a;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = h.waves;
  const int64_t base = (int64_t)blockIdx.x * 64, left = a.n - 1 - base;  // rows past the end read row n - 1
  const int loc = lane < left ? lane : (int)left;
  const int64_t row = base + loc;
  HotSums o;
  if (h.ranges) {
    for (int q = w; q < h.ranges; q += W) {
      const float2 ms = h.ms[(int64_t)q * a.n + row];
      hot_add<MIX>(o, HotSums{ms.x, ms.y, h.S[(int64_t)q * a.n + row]}, h.inv_t);
    }
  } else {
    const int per = ((a.d + W - 1) / W + 15) / 16 * 16, j0 = w * per;
    o = hot_columns<MIX>(h, a.F + base, loc, j0, j0 + per < a.d ? j0 + per : a.d);
  }
  const bool logits = a.teacher == SB_TEACHER_LOGITS;
  float vm = -INFINITY;
  if (logits) {
#pragma unroll 4
    for (int s = w; s < a.k; s += W) vm = fmaxf(vm, usable(a, load_place(a, s, row)).v);
    sh.at_f(2, w, lane) = vm;
  }
  o = hot_join<MIX>(h, sh, o, w, lane);
  if (logits)
    for (int u = 0; u < W; ++u) vm = fmaxf(vm, sh.at_f(2, u, lane));
  // e_t and its products with the value and the listed score; a place with e_t = 0 is no target
  double zs = 0.0, us = 0.0, ds = 0.0;
  for (int s = w; s < a.k; s += 4 * W) {
    Place p[4];
    float score[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = s + u * W < a.k ? load_place(a, s + u * W, row) : Place{-1, 0.0f};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      p[u] = usable(a, p[u]);
      score[u] = a.F[(int64_t)(p[u].id >= 0 ? p[u].id : 0) * a.ld_f + row];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const double x = logits ? ((double)p[u].v - (double)vm) * h.inv_t : (double)p[u].v;
      // a value of -inf is left out here: with no finite one its difference is no number
      const double e = p[u].v == -INFINITY ? 0.0 : logits ? exp_fine(x) : (double)exp2_hw(p[u].v * LOG2E);
      if (e != 0.0) {
        zs += e;
        us += e * x;
        ds += e * ((double)score[u] - (double)o.m);
      }
    }
  }
  if (W > 1) {
    sh.at(1, w, lane) = zs;
    sh.at(2, w, lane) = us;
    sh.at(3, w, lane) = ds;
    __syncthreads();
  }
  if (w != 0) return;
  if (W > 1) {
    zs = sh.sum(1, lane);
    us = sh.sum(2, lane);
    ds = sh.sum(3, lane);
  }
  const double log_S = o.S > 0.0 ? log(o.S) : 0.0;
  double loss = 0.0;
  if (!logits) loss = h.bt * (us + zs * log_S - ds * h.inv_t);
  else if (zs != 0.0) loss = h.bt * ((us - ds * h.inv_t) / zs + (log_S - log(zs)));
  if (MIX) {
    const int y = a.labels[row];
    if (y >= 0 && y < a.d)
      loss += a.w * ((double)log_of(o.s1) - ((double)a.F[(int64_t)y * a.ld_f + row] - (double)o.m));
  }
  if (lane <= left) a.loss[row] = (float)loss;
}

// Few rows with many classes: column ranges over blocks.
DistillWidePlan hot_plan(int64_t n, int32_t d) {
  DistillWidePlan p{};
  const int tiles = (int)((n + 63) / 64);
  if (d > DISTILL_REGS_MAX_D && tiles < 128) p = distill_wide_plan(n, d);
  p.tiles = tiles;
  return p;
}
int64_t hot_bytes(int64_t n, int32_t d) { return align256((int64_t)hot_plan(n, d).ranges * n * 8) * 2; }

void launch_hot(const RowArgs& r, void* ws, bool mix, hipStream_t st) {
  const DistillArgs& a = r.a;
  const DistillWidePlan p = hot_plan(a.n, a.d);
  // eight waves per CU where the columns allow it
  int waves = (2048 + p.tiles - 1) / p.tiles;
  if (waves > DISTILL_MAX_WAVES) waves = DISTILL_MAX_WAVES;
  if (waves > (a.d + 15) / 16) waves = (a.d + 15) / 16;
  char* at = static_cast<char*>(ws);
  const HotArgs h{r, 1.0 / a.T, (1.0 - a.w) * a.T * a.T, waves, p.tiles, p.ranges, p.cols,
                  reinterpret_cast<double*>(at), reinterpret_cast<float2*>(at + align256((int64_t)p.ranges * a.n * 8))};
  auto run = [&](auto stats, auto loss) {
    if (p.ranges)
      hipLaunchKernelGGL(stats, dim3(p.ranges * p.tiles), dim3(64 * WIDE_WAVES), WIDE_WAVES * HOT_WAVE_BYTES, st, h);
    hipLaunchKernelGGL(loss, dim3(p.tiles), dim3(64 * waves), waves * HOT_WAVE_BYTES, st, h);
  };
  if (mix) run(k_hot_stats<true>, k_hot_loss<true>);
  else run(k_hot_stats<false>, k_hot_loss<false>);
}

// The loss alone, a wave per tile: where there are tiles for the waves of the card, and
// few listed scores, which by then are read from memory once more, a cache line each (us
// by lane and by blocks: 100,000 x 1000 with 10 places 86 and 118, with 25 113 and 120,
// x 400 with 10 42 and 53; 300,007 x 1000 with 25 349 and 380, with 32 387 and 388; 1M x
// 400 with 4 331 and 395, x 100 with 2 99 and 101, x 100 with 10 156 and 109; 100,003 x
// 1500 with 37 176 and 207).  It gives away 4% at 1M x 200 with 5 (199 and 192), and more
// where there are fewer rows (50,000 x 400 with 4 20 and 31).
bool loss_by_lane(const DistillArgs& a) { return a.n >= 100000 && a.d >= 40 * a.k; }

template <int ROWS, int C, int MODE, typename OFF>
void launch_regs(const RowArgs& r, const DistillPlan& p, bool mix, hipStream_t st) {
  const dim3 grid((p.grid + 7) / 8 * 8), block(64 * p.waves * p.groups);
  if (mix) hipLaunchKernelGGL((k_distill_regs<ROWS, C, MODE, true, OFF>), grid, block, p.lds, st, r, p.grid);
  else hipLaunchKernelGGL((k_distill_regs<ROWS, C, MODE, false, OFF>), grid, block, p.lds, st, r, p.grid);
}

template <int MODE>
void launch_mode(const RowArgs& r, const DistillPlan& p, bool mix, hipStream_t st) {
  const DistillArgs& a = r.a;
  const bool near = a.ld_f < DISTILL_NEAR_LD && (!a.G || a.ld_g < DISTILL_NEAR_LD) && (!a.hess || a.ld_h < DISTILL_NEAR_LD);
  if (p.rows == 32 && near) launch_regs<32, 32, MODE, uint32_t>(r, p, mix, st);
  else if (p.rows == 32) launch_regs<32, 32, MODE, uint64_t>(r, p, mix, st);
  else if (p.c == 32) launch_regs<64, 32, MODE, uint32_t>(r, p, mix, st);
  else if (p.c == 16) launch_regs<64, 16, MODE, uint32_t>(r, p, mix, st);
  else launch_regs<64, 8, MODE, uint32_t>(r, p, mix, st);
}

template <int MODE, bool MIX>
void launch_wide(const RowArgs& r, const DistillWidePlan& p, hipStream_t st) {
  const dim3 block(64 * WIDE_WAVES);
  auto blocks = [](int units) { return dim3((units + 7) / 8 * 8); };
  hipLaunchKernelGGL(k_distill_stats<MIX>, blocks(p.ranges * p.tiles), block, 0, st, r, p.ranges * p.tiles);
  // few tiles: more waves to a tile (one of 60,000 classes 26 us with 4, 12 with 16; 313 of 5003 12 with 16; 1563 of
  // 1030 9 and 17)
  if (p.tiles <= DISTILL_SLOTS) hipLaunchKernelGGL((k_distill_rows<MIX, 16>), dim3(p.tiles), dim3(64 * 16), 0, st, r);
  else hipLaunchKernelGGL((k_distill_rows<MIX, 4>), dim3(p.tiles), dim3(64 * 4), 0, st, r);
  if constexpr (MODE != 0) {
    const size_t lds = 4 * (2 * r.a.k * 64 + WIDE_WAVES * distill_tile_floats(16));
    hipLaunchKernelGGL((k_distill_range<MODE, MIX>), blocks(p.ranges * p.slots), block, lds, st, r, p.ranges * p.slots);
    if (r.a.loss || r.a.h_row)
      hipLaunchKernelGGL(k_distill_join, dim3((unsigned)((r.a.n + 255) / 256)), dim3(256), 0, st, r.stats, p.ranges, r.a.n,
                         r.a.d, r.a.loss, r.a.h_row);
  }
}

int64_t norm_bytes(int64_t n, int32_t d, int32_t k) {
  if (d > DISTILL_REGS_MAX_D) return align256((int64_t)d * distill_wide_plan(n, d).slots * 8);
  const DistillPlan p = distill_plan(n, d, k);
  return align256((int64_t)d * p.grid * p.groups * 8);
}

}  // namespace

// Workspace: [norm partials]; past 1024 classes [rows' values and targets][statistics of the ranges] too.
// A hot loss takes it from the start again.
int64_t distill_ws_bytes(int64_t n, int32_t d, int32_t k) {
  int64_t b = norm_bytes(n, d, k);
  if (d > DISTILL_REGS_MAX_D)
    b += align256((int64_t)(ROW_VALUES + k) * n * 4) + align256((int64_t)distill_wide_plan(n, d).ranges * 3 * n * 4);
  const int64_t hot = hot_bytes(n, d);
  return b > hot ? b : hot;
}

int32_t launch_distill(const DistillArgs& args, void* ws, hipStream_t st, const char* call) {
  // a hot loss is formed by kernels of its own, once the others are through with the workspace
  const bool hot = args.loss && args.T > HOT && args.w < 1.0;
  DistillArgs a = args;
  if (hot) a.loss = nullptr;
  const double b = (1.0 - a.w) * a.T;
  RowArgs r{};
  r.a = a;
  r.inv_t = (float)(1.0 / a.T);
  r.c2 = (float)(1.4426950408889634 / a.T);
  r.w = (float)a.w;
  r.b = (float)b;
  r.bt = (float)(b * a.T);
  r.npart = a.norm2 ? static_cast<double*>(ws) : nullptr;
  const bool mix = a.w > 0.0 && a.T != 1.0;
  const int mode = !a.G ? 0 : a.hess || a.h_row ? 2 : 1;
  if (mode == 0 && hot) {
    // nothing else is asked for
  } else if (mode == 0 && loss_by_lane(a)) {
    const dim3 blocks((unsigned)((a.n + 255) / 256));
    if (mix) hipLaunchKernelGGL(k_loss_by_lane<true>, blocks, dim3(256), 0, st, r);
    else hipLaunchKernelGGL(k_loss_by_lane<false>, blocks, dim3(256), 0, st, r);
  } else if (a.d <= DISTILL_REGS_MAX_D) {
    const DistillPlan p = distill_plan(a.n, a.d, a.k, mode == 0);
    r.tile_bytes = p.lds / p.groups;
    r.waves = p.waves;
    r.groups = p.groups;
    r.tiles = p.tiles;
    r.parts = p.grid * p.groups;
    if (mode == 0) launch_mode<0>(r, p, mix, st);
    else if (mode == 1) launch_mode<1>(r, p, mix, st);
    else launch_mode<2>(r, p, mix, st);
  } else {
    const DistillWidePlan p = distill_wide_plan(a.n, a.d);
    r.ranges = p.ranges;
    r.cols = p.cols;
    r.tiles = p.tiles;
    r.slots = p.slots;
    r.parts = p.slots;
    char* at = static_cast<char*>(ws) + norm_bytes(a.n, a.d, a.k);
    r.row = reinterpret_cast<float*>(at);
    r.stats = reinterpret_cast<float*>(at + align256((int64_t)(ROW_VALUES + a.k) * a.n * 4));
    if (mode == 0) mix ? launch_wide<0, true>(r, p, st) : launch_wide<0, false>(r, p, st);
    else if (mode == 1) mix ? launch_wide<1, true>(r, p, st) : launch_wide<1, false>(r, p, st);
    else mix ? launch_wide<2, true>(r, p, st) : launch_wide<2, false>(r, p, st);
  }
  if (a.norm2) launch_norm_final(r.npart, a.d, r.parts, a.norm2, st);
  if (hot) {
    r.a.loss = args.loss;
    launch_hot(r, ws, mix, st);
  }
  return check_launch(call);
}

}  // namespace sb
