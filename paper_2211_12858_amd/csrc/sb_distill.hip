// Distillation from a teacher's top classes: the loss of every row and its
// first and second derivatives by the scores (sb_distill_loss,
// sb_distill_gradients).
//
// For a row with scores a, m = max a, s1 = sum exp(a_j - m),
// sT = sum exp((a_j - m) / T), teacher's probabilities q_t of classes c_t,
// Q = sum q_t, A = w where the row has a label (else 0), B = (1 - w) T:
//   target_j = A [j == label] + B sum_{t: c_t == j} q_t
//   loss = A log s1 + B T (sum q_t log q_t + Q log sT) - sum_j target_j (a_j - m)
//   g_j  = A p1_j + B Q pT_j - target_j
//   h_j  = A p1_j (1 - p1_j) + (B / T) Q pT_j (1 - pT_j)
// so the teacher's list and the label are one sparse target row.
#include <cmath>

#include "sb_common.h"

namespace sb {
namespace {

struct RowArgs {
  DistillArgs a;
  float inv_t, w, b, bt;  // 1 / T, hard weight, B = (1 - w) T, B T
};

// One wave per row.
__global__ void __launch_bounds__(256) k_distill(RowArgs r) {
  const DistillArgs& a = r.a;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.n) return;
  const float* x = a.F + row;
  float m = -INFINITY;
  for (int j = lane; j < a.d; j += 64) m = fmaxf(m, x[j * a.ld_f]);
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  float s1 = 0.0f, sT = 0.0f;
  for (int j = lane; j < a.d; j += 64) {
    const float z = x[j * a.ld_f] - m;
    s1 += expf(z);
    sT += expf(z * r.inv_t);
  }
  for (int off = 32; off > 0; off >>= 1) {
    s1 += __shfl_xor(s1, off, 64);
    sT += __shfl_xor(sT, off, 64);
  }
  // lane t holds place t of the list
  const int y = a.w > 0.0 ? a.labels[row] : -1;
  const float A = y >= 0 && y < a.d ? r.w : 0.0f;
  int id = -1;
  float v = -INFINITY;
  if (lane < a.k) {
    id = a.t_id[lane * a.ld_t + row];
    if (id >= 0 && id < a.d) v = a.t_val[lane * a.ld_t + row];
    else id = -1;
  }
  float q, lq;
  if (a.teacher == SB_TEACHER_LOGITS) {
    float vm = v;
    for (int off = 32; off > 0; off >>= 1) vm = fmaxf(vm, __shfl_xor(vm, off, 64));
    const float u = v == -INFINITY ? -INFINITY : (v - vm) * r.inv_t;
    const float e = expf(u);
    float z = e;
    for (int off = 32; off > 0; off >>= 1) z += __shfl_xor(z, off, 64);
    q = e > 0.0f ? e / z : 0.0f;
    lq = e > 0.0f ? u - logf(z) : 0.0f;
  } else {
    q = expf(v);
    lq = q > 0.0f ? v : 0.0f;
  }
  float Q = q, ent = q * lq;
  float dot = q > 0.0f ? r.b * q * (x[id * a.ld_f] - m) : 0.0f;
  for (int off = 32; off > 0; off >>= 1) {
    Q += __shfl_xor(Q, off, 64);
    ent += __shfl_xor(ent, off, 64);
    dot += __shfl_xor(dot, off, 64);
  }
  if (a.loss && lane == 0) {
    if (A > 0.0f) dot += A * (x[y * a.ld_f] - m);
    a.loss[row] = A * logf(s1) + r.bt * (ent + Q * logf(sT)) - dot;
  }
  if (!a.G) return;
  const float BQ = r.b * Q;
  float hsum = 0.0f;
  for (int j0 = 0; j0 < a.d; j0 += 64) {
    const int j = j0 + lane;
    float target = j == y ? A : 0.0f;
    for (int t = 0; t < a.k; ++t) {
      const int c = __shfl(id, t, 64);
      const float qt = __shfl(q, t, 64);
      if (c == j) target += r.b * qt;
    }
    if (j < a.d) {
      const float z = x[j * a.ld_f] - m;
      const float p1 = expf(z) / s1, pT = expf(z * r.inv_t) / sT;
      a.G[j * a.ld_g + row] = A * p1 + BQ * pT - target;
      const float h = A * (p1 * (1.0f - p1)) + BQ * r.inv_t * (pT * (1.0f - pT));
      if (a.hess) a.hess[j * a.ld_h + row] = h;
      hsum += h;
    }
  }
  for (int off = 32; off > 0; off >>= 1) hsum += __shfl_xor(hsum, off, 64);
  if (a.h_row && lane == 0) a.h_row[row] = hsum * (1.0f / (float)a.d);
}

// One block per column of G.
__global__ void __launch_bounds__(256) k_distill_norms(const float* G, int64_t n, int64_t ld_g, double* norm2) {
  __shared__ double part[4];
  const float* g = G + (int64_t)blockIdx.x * ld_g;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 256) s += (double)g[i] * g[i];
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) norm2[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

}  // namespace

int64_t distill_ws_bytes(int64_t, int32_t, int32_t) { return 0; }

int32_t launch_distill(const DistillArgs& a, void*, hipStream_t st, const char* call) {
  const double b = (1.0 - a.w) * a.T;
  const RowArgs r{a, (float)(1.0 / a.T), (float)a.w, (float)b, (float)(b * a.T)};
  hipLaunchKernelGGL(k_distill, dim3((unsigned)((a.n + 3) / 4)), dim3(256), 0, st, r);
  if (a.norm2) hipLaunchKernelGGL(k_distill_norms, dim3(a.d), dim3(256), 0, st, a.G, a.n, a.ld_g, a.norm2);
  return check_launch(call);
}

}  // namespace sb
