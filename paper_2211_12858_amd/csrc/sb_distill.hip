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
// so the teacher's list and the label are one sparse target row, and at T = 1 the
// two softmaxes are one.
//
// k_distill_regs (rows of up to 1024 scores): a row tile's scores stay in the
// registers of a block's waves, lanes on consecutive rows, c columns per lane, so
// F is read once and every load and store is a run of a column.  Waves exchange
// maxima and sums in LDS; each handles its share of the tile's list places, and
// all waves then look through all places for the classes of their own columns and
// add their targets to the wave's LDS tile of 16 columns.  The gradients replace the targets in that tile,
// from which 16 lanes per row segment add the squared column norms in fp64, in a
// fixed order; a block's sums are one partial.  While a tile's gradients go out
// the same registers take the next tile's scores.
// k_distill_stats, k_distill_range (wider rows): maxima and sums of 512-column
// ranges, then the outputs range by range, the list places staged per block.
//
// exp(z / T) is 2^(z * log2(e) / T) by the hardware's exponential, which returns 0
// below 2^-126: probabilities under 2^-126 of the row's largest are 0.
#include <cmath>

#include "sb_common.h"
#include "sb_distill_plan.h"

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
  int waves, groups, tiles;  // k_distill_regs
  float* stats;              // [ranges][3][n]: k_distill_stats
  int ranges, slots;
};

// Other lanes of the wave see this wave's LDS writes; the compiler keeps the order.
__device__ inline void wave_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

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

// The targets of the lane's row in its CG columns from jg, into its (zeroed) tile row:
// the places' and the label's (class y - jg of weight A).  A class listed again is
// added to what is there; a bit per column says which are (a float atomic per place
// instead takes the LDS three clocks a lane).  Places are read eight at a time.
template <int CG, int ROWS>
__device__ inline void add_targets(const Listed* ent, int K, int rl, int jg, float wt, int y, float A, float* trow) {
  uint32_t seen = 0;
  auto put = [&](uint32_t c, float v) {
    if (c < (uint32_t)CG) {
      const uint32_t bit = 1u << c;
      if (seen & bit) v += trow[c];
      trow[c] = v;
      seen |= bit;
    }
  };
  int s = 0;
  for (; s + 8 <= K; s += 8) {
    Listed p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) p[u] = ent[(s + u) * ROWS + rl];
#pragma unroll
    for (int u = 0; u < 8; ++u) put((uint32_t)(p[u].id - jg), wt * p[u].e);
  }
  for (; s < K; ++s) {
    const Listed p = ent[s * ROWS + rl];
    put((uint32_t)(p.id - jg), wt * p.e);
  }
  if (y >= 0) put((uint32_t)(y - jg), A);
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

template <int ROWS, int C, int MODE, bool MIX, bool FULLC>
__device__ __forceinline__ void distill_wave(const RowArgs& r, char* lds, int w, int rg, int bx, int grid) {
  constexpr int PARTS = 64 / ROWS;
  constexpr int CG = C < 16 ? C : 16, S = CG + 4, NG = C / CG;
  const DistillArgs& a = r.a;
  const int W = r.waves, K = a.k;
  const int lane = threadIdx.x & 63, rl = lane & (ROWS - 1), hb = lane / ROWS;
  Listed* ent = reinterpret_cast<Listed*>(lds);
  float* red = reinterpret_cast<float*>(lds) + 2 * K * ROWS;  // [DISTILL_RED][W][64]
  float* tile = red + DISTILL_RED * W * 64 + w * distill_tile_floats(C);
  float* trow = tile + lane * S;
  const int j0 = w * C * PARTS;    // the wave's first column
  int last = a.d - 1 - j0;         // its last one, from there
  const int jl = j0 + hb * C;      // the lane's first column
  constexpr bool STEP = FULLC || PARTS == 1;  // a column is a step of a uniform pointer
  auto at = [&](int i, uint32_t loc, int64_t ld) -> uint32_t {
    if (PARTS == 1) return 4 * loc;
    if (FULLC) return 4 * (loc + (uint32_t)(hb * C) * (uint32_t)ld);
    const int c = hb * C + i;
    return 4 * (loc + (uint32_t)(c < last ? c : last) * (uint32_t)ld);
  };
  // Rows past the end are row n - 1 again: they store its own values once more
  // and stay out of the norms.
  auto rows_of = [&](int tile_no, int64_t& base, uint32_t& loc) {
    base = ((int64_t)tile_no * r.groups + rg) * ROWS;
    const int64_t left = a.n - 1 - base;
    if (left < 0) {
      base = a.n - 1;
      loc = 0;
    } else {
      loc = rl < left ? rl : (uint32_t)left;
    }
  };
  auto load_at = [](const float* p, uint32_t bytes) {
    return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p) + bytes);
  };
  auto store_at = [](float* p, uint32_t bytes, float v) {
    *reinterpret_cast<float*>(reinterpret_cast<char*>(p) + bytes) = v;
  };
  auto red_put = [&](int q, float v) { red[(q * W + w) * 64 + lane] = v; };
  auto red_max = [&](int q) {
    float v = red[q * W * 64 + lane];
    for (int u = 1; u < W; ++u) v = fmaxf(v, red[(q * W + u) * 64 + lane]);
    return v;
  };
  auto red_sum = [&](int q) {
    float v = red[q * W * 64 + lane];
    for (int u = 1; u < W; ++u) v += red[(q * W + u) * 64 + lane];
    return v;
  };
  // over the lanes of a row
  auto part_sum = [&](float v) {
#pragma unroll
    for (int off = 32; off >= ROWS; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
  };
  auto part_max = [&](float v) {
#pragma unroll
    for (int off = 32; off >= ROWS; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
  };

  int64_t base;
  uint32_t loc;
  rows_of(bx, base, loc);
  float x[C];
  {
    const float* p = a.F + (int64_t)j0 * a.ld_f + base;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      x[i] = load_at(p, at(i, loc, a.ld_f));
      if (STEP && (FULLC || i < last)) p += a.ld_f;
    }
  }
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
    m = part_max(m);
    vm = part_max(vm);
    if (W > 1) {
      red_put(0, m);
      red_put(1, vm);
      lds_barrier();
      m = red_max(0);
      vm = red_max(1);
    } else {
      wave_sync();
    }
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
    zs = part_sum(zs);
    us = part_sum(us);
    sT = part_sum(sT);
    if (MIX) s1 = part_sum(s1);
    if (W > 1) {
      red_put(2, zs);
      red_put(3, us);
      red_put(4, sT);
      if (MIX) red_put(5, s1);
      lds_barrier();
      zs = red_sum(2);
      us = red_sum(3);
      sT = red_sum(4);
      if (MIX) s1 = red_sum(5);
    } else {
      wave_sync();
    }
    if (!MIX) s1 = sT;
    const Teacher te = teacher_of(r, zs, us);
    const float BQ = r.b * te.Q;
    const float iT = 1.0f / sT, i1 = 1.0f / s1;
    const float kT = (MIX ? BQ : A + BQ) * iT, k1 = A * i1;          // coefficients of the exponentials in g
    const float hT = MIX ? BQ * r.inv_t : A + BQ * r.inv_t, h1 = A;  // of p (1 - p) in h

    // the exponentials are formed again below: kept, they take the registers of two rows more
    asm volatile("" : "+v"(m));
    int64_t nbase;
    uint32_t nloc;
    rows_of(t + grid < r.tiles ? t + grid : t, nbase, nloc);
    // the next tile's places and labels, which arrive while this one goes out
    const int64_t nrow = nbase + nloc;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * W * PARTS < K) ahead[u] = load_place(a, s0 + u * W * PARTS, nrow);
    if (a.w > 0.0) next_y = a.labels[nrow];
    float hsum = 0.0f, dot = 0.0f;
    if (MODE == 0) {
      // the loss alone: the scores of the listed classes, through the tile
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        wave_sync();
#pragma unroll
        for (int i = 0; i < CG; ++i) trow[i] = x[g * CG + i];
        for (int sl = 0; sl < K; ++sl) {
          const Listed p = ent[sl * ROWS + rl];
          const uint32_t c = (uint32_t)(p.id - jl - g * CG);
          if (c < CG) dot += te.wt * p.e * (trow[c] - m);
        }
        const uint32_t cy = (uint32_t)(y - jl - g * CG);
        if (y >= 0 && cy < CG) dot += A * (trow[cy] - m);
      }
      const float* p = a.F + (int64_t)j0 * a.ld_f + nbase;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        x[i] = load_at(p, at(i, nloc, a.ld_f));
        if (STEP && (FULLC || i < last)) p += a.ld_f;
      }
    } else {
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
            dot = fmaf(tv[u], z, dot);
            // columns past the last repeat it: same address, same value, but no target there
            if (live) store_at(Gc, at(i, loc, ld_g), gr);
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
                if (live) store_at(Hc, at(i, loc, ld_h), h);
                if (STEP && (FULLC || i < last)) Hc += ld_h;
              }
            }
            gv[u] = ok && live ? gr : 0.0f;
            x[i] = load_at(Fc, at(i, nloc, ld_f));
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
      if (a.loss) dot = part_sum(dot);
      if (MODE == 2 && a.h_row) hsum = part_sum(hsum);
      if (W > 1) {
        if (a.loss) red_put(6, dot);
        if (MODE == 2 && a.h_row) red_put(7, hsum);
        lds_barrier();  // and all waves are through with the places
      }
      if (w == 0 && hb == 0) {
        if (a.loss) {
          if (W > 1) dot = red_sum(6);
          a.loss[row] = A * logf(s1) + r.bt * (te.ent + te.Q * logf(sT)) - dot;
        }
        if (MODE == 2 && a.h_row) {
          if (W > 1) hsum = red_sum(7);
          a.h_row[row] = hsum * (1.0f / (float)a.d);
        }
      }
    }
    if (W == 1) wave_sync();  // the places are read before the next tile's
    base = nbase;
    loc = nloc;
  }
  if (MODE != 0 && r.npart) {
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
template <int ROWS, int C, int MODE, bool MIX>
__global__ void __launch_bounds__(64 * DISTILL_MAX_WAVES) k_distill_regs(RowArgs r, int grid) {
  extern __shared__ __align__(16) char smem[];
  const int bx = (int)(blockIdx.x & 7) * ((grid + 7) >> 3) + (int)(blockIdx.x >> 3);
  if (bx >= grid) return;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wv / r.waves, w = wv - rg * r.waves;
  const int bytes = 4 * (2 * r.a.k * ROWS + DISTILL_RED * r.waves * 64 + r.waves * distill_tile_floats(C));
  char* lds = smem + rg * bytes;
  if ((w + 1) * C * (64 / ROWS) <= r.a.d) distill_wave<ROWS, C, MODE, MIX, true>(r, lds, w, rg, bx, grid);
  else distill_wave<ROWS, C, MODE, MIX, false>(r, lds, w, rg, bx, grid);
}

// ---------------------------------------------------------------- wider rows
constexpr int WIDE_WAVES = 4;
constexpr int WIDE_COLS = DISTILL_RANGE / WIDE_WAVES;  // columns per wave

// Maximum and sums of exponentials of a 64-row tile's columns in one range: the
// waves' running maxima and sums, joined in LDS.
template <bool MIX>
__global__ void __launch_bounds__(64 * WIDE_WAVES) k_distill_stats(RowArgs r) {
  __shared__ float red[3][WIDE_WAVES][64];
  const DistillArgs& a = r.a;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int range = blockIdx.y;
  const int64_t base = (int64_t)blockIdx.x * 64;
  const int64_t left = a.n - 1 - base;
  const int loc = lane < left ? lane : (int)left;
  const int j0 = range * DISTILL_RANGE + w * WIDE_COLS;
  const int j1 = j0 + WIDE_COLS < a.d ? j0 + WIDE_COLS : a.d;
  float m = -INFINITY, s1 = 0.0f, sT = 0.0f;
  for (int j = j0; j < j1; j += 16) {
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = (a.F + (int64_t)(j + i < j1 ? j + i : j1 - 1) * a.ld_f + base)[loc];
    float cm = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) cm = fmaxf(cm, x[i]);
    const float mn = fmaxf(m, cm);
    float a1 = 0.0f, aT = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float z = x[i] - mn;
      const bool live = j + i < j1;
      aT += live ? exp2_hw(z * r.c2) : 0.0f;
      if (MIX) a1 += live ? exp2_hw(z * LOG2E) : 0.0f;
    }
    sT = fmaf(sT, exp2_hw((m - mn) * r.c2), aT);
    if (MIX) s1 = fmaf(s1, exp2_hw((m - mn) * LOG2E), a1);
    m = mn;
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
    const float z = red[0][u][lane] - mm;  // -inf for a wave without columns, whose sums are 0
    sT += red[1][u][lane] * exp2_hw(z * r.c2);
    if (MIX) s1 += red[2][u][lane] * exp2_hw(z * LOG2E);
  }
  float* out = r.stats + (int64_t)range * 3 * a.n + base + lane;
  out[0] = mm;
  out[a.n] = sT;
  if (MIX) out[2 * a.n] = s1;
}

// The outputs of a 64-row tile's columns in one range.  MODE 0 (the loss alone) has
// one range: listed scores are gathered.
template <int MODE, bool MIX>
__global__ void __launch_bounds__(64 * WIDE_WAVES) k_distill_range(RowArgs r) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float red[3][WIDE_WAVES][64];
  const DistillArgs& a = r.a;
  const int K = a.k;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Listed* ent = reinterpret_cast<Listed*>(smem);  // [K][64]
  float* tile = reinterpret_cast<float*>(smem) + 2 * K * 64 + w * distill_tile_floats(16);
  float* trow = tile + lane * 20;
  const int j0 = blockIdx.x * DISTILL_RANGE + w * WIDE_COLS;
  const int cols = a.d - j0 < WIDE_COLS ? a.d - j0 : WIDE_COLS;  // may be <= 0
  for (int64_t t = blockIdx.y; t * 64 < a.n; t += gridDim.y) {
    const int64_t base = t * 64;
    const int64_t left_rows = a.n - 1 - base;
    const int loc = lane < left_rows ? lane : (int)left_rows;
    const bool ok = lane <= left_rows;
    const int64_t row = base + loc;
    float vm = -INFINITY;
    for (int s = w; s < K; s += WIDE_WAVES) {
      const Place p = usable(a, load_place(a, s, row));
      ent[s * 64 + lane] = Listed{p.id, p.v};
      vm = fmaxf(vm, p.v);
    }
    int y = -1;
    if (a.w > 0.0) {
      y = a.labels[row];
      if (y >= a.d) y = -1;
    }
    const float A = y >= 0 ? r.w : 0.0f;
    // the row's statistics from the ranges'
    float m = -INFINITY, sT = 0.0f, s1 = 0.0f;
    for (int q = 0; q < r.ranges; ++q) m = fmaxf(m, r.stats[(int64_t)q * 3 * a.n + row]);
    for (int q = 0; q < r.ranges; ++q) {
      const float* st = r.stats + (int64_t)q * 3 * a.n + row;
      const float z = st[0] - m;
      sT = fmaf(st[a.n], exp2_hw(z * r.c2), sT);
      if (MIX) s1 = fmaf(st[2 * a.n], exp2_hw(z * LOG2E), s1);
    }
    red[0][w][lane] = vm;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < WIDE_WAVES; ++u) vm = fmaxf(vm, red[0][u][lane]);
    float zs = 0.0f, us = 0.0f;
    for (int s = w; s < K; s += WIDE_WAVES) {
      const float e = place_exp(r, ent[s * 64 + lane].e, vm, us);
      ent[s * 64 + lane].e = e;
      zs += e;
    }
    red[1][w][lane] = zs;
    red[2][w][lane] = us;
    __syncthreads();
    zs = us = 0.0f;
#pragma unroll
    for (int u = 0; u < WIDE_WAVES; ++u) {
      zs += red[1][u][lane];
      us += red[2][u][lane];
    }
    if (!MIX) s1 = sT;
    const Teacher te = teacher_of(r, zs, us);
    const float BQ = r.b * te.Q;
    const float iT = 1.0f / sT, i1 = 1.0f / s1;
    const float kT = (MIX ? BQ : A + BQ) * iT, k1 = A * i1;
    const float hT = MIX ? BQ * r.inv_t : A + BQ * r.inv_t, h1 = A;
    if (a.loss && blockIdx.x == 0) {
      // the listed scores, each wave its places
      float dot = 0.0f;
      for (int s = w; s < K; s += WIDE_WAVES) {
        const Listed p = ent[s * 64 + lane];
        if (p.id >= 0) dot += te.wt * p.e * (a.F[(int64_t)p.id * a.ld_f + row] - m);
      }
      if (w == 0 && y >= 0) dot += A * (a.F[(int64_t)y * a.ld_f + row] - m);
      red[0][w][lane] = dot;  // vm is read before the barrier above
      __syncthreads();
      if (w == 0) {
        for (int u = 1; u < WIDE_WAVES; ++u) dot += red[0][u][lane];
        if (ok) a.loss[row] = A * logf(s1) + r.bt * (te.ent + te.Q * logf(sT)) - dot;
      }
      __syncthreads();
    }
    if (MODE != 0) {
      float hsum = 0.0f;
      for (int c0 = 0; c0 < cols; c0 += 16) {
        const int last = cols - 1 - c0;  // of the group's columns, from its first
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          x[i] = (a.F + (int64_t)(j0 + c0 + (i < last ? i : last)) * a.ld_f + base)[loc];
        wave_sync();
        float4* t4 = reinterpret_cast<float4*>(trow);
#pragma unroll
        for (int q = 0; q < 4; ++q) t4[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        add_targets<16, 64>(ent, K, lane, j0 + c0, te.wt, y, A, trow);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 t4v = t4[q];
          const float tv[4] = {t4v.x, t4v.y, t4v.z, t4v.w};
          float gv[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int i = q * 4 + u;
            const float z = x[i] - m;
            const float eT = exp2_hw(z * r.c2);
            float gr = fmaf(kT, eT, -tv[u]);
            float e1 = 0.0f;
            if (MIX) {
              e1 = exp2_hw(z * LOG2E);
              gr = fmaf(k1, e1, gr);
            }
            if (ok && i <= last) (a.G + (int64_t)(j0 + c0 + i) * a.ld_g + base)[loc] = gr;
            if (MODE == 2) {
              const float pT = eT * iT;
              float h = hT * fmaf(-pT, pT, pT);
              if (MIX) {
                const float p1 = e1 * i1;
                h = fmaf(h1, fmaf(-p1, p1, p1), h);
              }
              hsum += i <= last ? h : 0.0f;
              if (a.hess && ok && i <= last) (a.hess + (int64_t)(j0 + c0 + i) * a.ld_h + base)[loc] = h;
            }
            gv[u] = ok && i <= last ? gr : 0.0f;
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
            double* pp = r.npart + (int64_t)(j0 + c0 + lane) * r.parts + blockIdx.y;
            *pp = t == blockIdx.y ? s : *pp + s;
          }
        }
      }
      if (MODE == 2 && a.h_row) {
        red[0][w][lane] = hsum;
        __syncthreads();
        if (w == 0 && ok) {
          for (int u = 1; u < WIDE_WAVES; ++u) hsum += red[0][u][lane];
          r.stats[(int64_t)r.ranges * 3 * a.n + (int64_t)blockIdx.x * a.n + row] = hsum;
        }
      }
    }
    __syncthreads();  // the places and exchanged values are read before the next tile's
  }
}

// Row means of the hessians from the ranges' sums.
__global__ void __launch_bounds__(256) k_distill_hrow(const float* sums, int ranges, int64_t n, int d, float* h_row) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float s = 0.0f;
  for (int q = 0; q < ranges; ++q) s += sums[(int64_t)q * n + i];
  h_row[i] = s * (1.0f / (float)d);
}

bool in_regs(const DistillArgs& a) {
  if (a.d > DISTILL_REGS_MAX_D) return false;
  if (a.d <= DISTILL_ONE_PART_D) return true;
  return a.ld_f < DISTILL_PARTS_MAX_LD && (!a.G || a.ld_g < DISTILL_PARTS_MAX_LD) &&
         (!a.hess || a.ld_h < DISTILL_PARTS_MAX_LD);
}

template <int ROWS, int C, int MODE>
void launch_regs(const RowArgs& r, const DistillPlan& p, bool mix, hipStream_t st) {
  const dim3 grid((p.grid + 7) / 8 * 8), block(64 * p.waves * p.groups);
  if (mix) hipLaunchKernelGGL((k_distill_regs<ROWS, C, MODE, true>), grid, block, p.lds, st, r, p.grid);
  else hipLaunchKernelGGL((k_distill_regs<ROWS, C, MODE, false>), grid, block, p.lds, st, r, p.grid);
}

template <int MODE>
void launch_mode(const RowArgs& r, const DistillPlan& p, bool mix, hipStream_t st) {
  if (p.rows == 32) launch_regs<32, 32, MODE>(r, p, mix, st);
  else if (p.c == 32) launch_regs<64, 32, MODE>(r, p, mix, st);
  else if (p.c == 16) launch_regs<64, 16, MODE>(r, p, mix, st);
  else launch_regs<64, 8, MODE>(r, p, mix, st);
}

template <int MODE>
void launch_range(const RowArgs& r, const DistillWidePlan& p, bool mix, hipStream_t st) {
  const dim3 grid(MODE == 0 ? 1 : p.ranges, p.slots), block(64 * WIDE_WAVES);
  const size_t lds = 4 * (2 * r.a.k * 64 + WIDE_WAVES * distill_tile_floats(16));
  if (mix) hipLaunchKernelGGL((k_distill_range<MODE, true>), grid, block, lds, st, r);
  else hipLaunchKernelGGL((k_distill_range<MODE, false>), grid, block, lds, st, r);
}

int64_t norm_bytes(int64_t n, int32_t d, int32_t k) {
  int64_t parts = distill_wide_plan(n, d).slots;
  if (d <= DISTILL_REGS_MAX_D) {
    const DistillPlan p = distill_plan(n, d, k);
    if ((int64_t)p.grid * p.groups > parts) parts = (int64_t)p.grid * p.groups;
  }
  return align256((int64_t)d * parts * 8);
}

}  // namespace

// Workspace: [norm partials][statistics of the ranges, 3 n each][row sums of the hessians, n per range]
int64_t distill_ws_bytes(int64_t n, int32_t d, int32_t k) {
  int64_t b = norm_bytes(n, d, k);
  // narrower rows never take the ranges
  if (d > DISTILL_ONE_PART_D) b += align256((int64_t)distill_wide_plan(n, d).ranges * 4 * n * 4);
  return b;
}

int32_t launch_distill(const DistillArgs& a, void* ws, hipStream_t st, const char* call) {
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
  if (in_regs(a)) {
    const DistillPlan p = distill_plan(a.n, a.d, a.k);
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
    r.slots = p.slots;
    r.parts = p.slots;
    r.stats = reinterpret_cast<float*>(static_cast<char*>(ws) + norm_bytes(a.n, a.d, a.k));
    const dim3 grid(p.tiles, p.ranges), block(64 * WIDE_WAVES);
    if (mix) hipLaunchKernelGGL(k_distill_stats<true>, grid, block, 0, st, r);
    else hipLaunchKernelGGL(k_distill_stats<false>, grid, block, 0, st, r);
    if (mode == 0) launch_range<0>(r, p, mix, st);
    else if (mode == 1) launch_range<1>(r, p, mix, st);
    else launch_range<2>(r, p, mix, st);
    if (mode == 2 && a.h_row)
      hipLaunchKernelGGL(k_distill_hrow, dim3((unsigned)((a.n + 255) / 256)), dim3(256), 0, st,
                         r.stats + (int64_t)p.ranges * 3 * a.n, p.ranges, a.n, a.d, a.h_row);
  }
  if (a.norm2) launch_norm_final(r.npart, a.d, r.parts, a.norm2, st);
  return check_launch(call);
}

}  // namespace sb
