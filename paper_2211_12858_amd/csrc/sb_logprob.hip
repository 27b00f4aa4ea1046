// Log probability and rank of a given class, log normaliser, entropy and the
// best classes of every row of scores (sb_log_probs).
//
// With m = max_j a_j and c = 1 / T, e_j = exp((a_j - m) c), s = sum e_j,
// t = sum e_j (a_j - m) c:
//   lse = m c + log s,  log p_y = (a_y - m) c - log s,  entropy = log s - t / s
// (log s >= 0 >= t, so the entropy has no cancellation).
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <cmath>

#include "sb_common.h"

namespace sb {
namespace {

struct LogProbArgs {
  const void* F;
  int64_t n;
  int32_t d;
  int64_t rs, cs;  // element (i, j) at F[i * rs + j * cs]
  float c;         // 1 / T
  const int32_t* labels;
  float* logp;
  int32_t* rank;
  float* lse;
  float* entropy;
  int32_t k;
  int32_t* top_id;
  float* top_logp;
  int64_t ld_top;
};

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(__half x) { return __half2float(x); }
__device__ inline float to_f32(__hip_bfloat16 x) { return __bfloat162float(x); }

// One wave per row: the maximum, the sums and the rank, then the alternatives one
// at a time, each the best class after the one before.
template <typename T>
__global__ void __launch_bounds__(256) k_log_probs(LogProbArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.n) return;
  const T* x = static_cast<const T*>(a.F) + row * a.rs;
  float m = -INFINITY;
  for (int j = lane; j < a.d; j += 64) m = fmaxf(m, to_f32(x[j * a.cs]));
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  const float mm = m == -INFINITY ? 0.0f : m;
  const int y = a.labels ? a.labels[row] : -1;
  const bool has = y >= 0 && y < a.d;
  const float ay = has ? to_f32(x[y * a.cs]) : 0.0f;
  float s = 0.0f, t = 0.0f;
  int before = 0;
  for (int j = lane; j < a.d; j += 64) {
    const float v = to_f32(x[j * a.cs]);
    const float u = (v - mm) * a.c, e = expf(u);
    s += e;
    t += e * fmaxf(u, -1000.0f);
    before += v > ay || (v == ay && j < y);
  }
  for (int off = 32; off > 0; off >>= 1) {
    s += __shfl_xor(s, off, 64);
    t += __shfl_xor(t, off, 64);
    before += __shfl_xor(before, off, 64);
  }
  const float log_s = logf(s);
  const bool none = m == -INFINITY && s == 0.0f;
  if (lane == 0) {
    if (a.lse) a.lse[row] = mm * a.c + log_s;
    if (a.entropy) a.entropy[row] = none ? 0.0f : log_s - t / s;
    if (a.logp) a.logp[row] = !has ? 0.0f : none ? -INFINITY : (ay - mm) * a.c - log_s;
    if (a.rank) a.rank[row] = has ? before : -1;
  }
  float pv = INFINITY;
  int pj = -1;
  bool first = true;
  for (int q = 0; q < a.k; ++q) {
    float bv = -INFINITY;
    int bj = -1;
    for (int j = lane; j < a.d; j += 64) {
      const float v = to_f32(x[j * a.cs]);
      const bool after = first || v < pv || (v == pv && j > pj);
      if (after && v > bv) {
        bv = v;
        bj = j;
      }
    }
    for (int off = 32; off > 0; off >>= 1) {
      const float ov = __shfl_xor(bv, off, 64);
      const int oj = __shfl_xor(bj, off, 64);
      if (oj >= 0 && (bj < 0 || ov > bv || (ov == bv && oj < bj))) {
        bv = ov;
        bj = oj;
      }
    }
    if (lane == 0) {
      a.top_id[q * a.ld_top + row] = bj;
      a.top_logp[q * a.ld_top + row] = bj < 0 ? -INFINITY : (bv - mm) * a.c - log_s;
    }
    pv = bj < 0 ? -INFINITY : bv;
    pj = bj < 0 ? a.d : bj;
    first = false;
  }
}

}  // namespace

int64_t log_probs_ws_bytes(int64_t, int32_t, int32_t) { return 0; }

int32_t launch_log_probs(const void* F, int32_t dtype, int32_t order, int64_t n, int32_t d, int64_t ld_f, double T,
                         const int32_t* labels, float* logp, int32_t* rank, float* lse, float* entropy, int32_t k,
                         int32_t* top_id, float* top_logp, int64_t ld_top, void*, hipStream_t st) {
  const bool col = order == SB_COLUMN_MAJOR;
  const LogProbArgs a{F,    n,   d,       col ? 1 : ld_f, col ? ld_f : 1, (float)(1.0 / T), labels, logp, rank,
                      lse,  entropy, k,   top_id,         top_logp,       ld_top};
  const dim3 blocks((unsigned)((n + 3) / 4)), threads(256);
  if (dtype == SB_F32) hipLaunchKernelGGL(k_log_probs<float>, blocks, threads, 0, st, a);
  else if (dtype == SB_F16) hipLaunchKernelGGL(k_log_probs<__half>, blocks, threads, 0, st, a);
  else hipLaunchKernelGGL(k_log_probs<__hip_bfloat16>, blocks, threads, 0, st, a);
  return check_launch("sb_log_probs");
}

}  // namespace sb
