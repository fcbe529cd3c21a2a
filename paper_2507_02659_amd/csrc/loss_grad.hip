// Gradient of the hybrid cross-vocabulary distillation loss with respect to the drafter's logits.
//
// With r(v) = ln q'(v) - ln p(v) + 1 (the derivative of q' ln(q'/p) by q'), a draft row with distribution q at temperature Td, and
// c = grad_loss / (tokens considered) / Td, times the token's lambda for n-grams:
//   direct token:     dz_i = c q_i (a_i - A),  a_i = r(image of i), 0 where i has none,  A = sum q a
//   n-gram, NLL:      dz_i = c (q_i - [i is the row's sub-token])                         in the rows of all its sub-tokens
//   n-gram, KL:       dz_i = D ([i is the row's sub-token] - q_i) in the rows of all its sub-tokens, D = c pi (r(t_ng) - r(t_pre)),
//                     and in the first one c q_i (a_i - A) as above with Eq. 2's overrides: a_i = r(t_pre) at the first sub-token,
//                     0 at the pre-image of t_ng.  (pi, the product of the sub-tokens' q, moves q'(t_ng) = pi and
//                     q'(t_pre) = q(d_1) - pi against each other.)
// A needs no sum of its own over the target row: the loss has left sum q' (ln q' - ln p), so A is that plus the mass of q on the ids that
// have an image (less and plus the overrides' terms).
#include "device_math.h"
#include "otv_internal.h"

namespace otv {
namespace {

struct RowGrad {
  double mxq, invTd, lnSq;      // ln q(i) = (zq_i - mxq) * invTd - lnSq
  double mx, invT, lnS;         // ln p(v) = (z_v - mx) * invT - lnS
  double c, A, D;
  int32_t kind;                 // 0: zeros, 1: the KL part, 2: D alone, 3: both
  int32_t sub;                  // the row's drafted id
  int32_t out, pre;             // draft ids whose a is 0 / a_pre, or -1
  double a_pre;
  int32_t row;
};

__device__ inline double draft_logit(const LossGradArgs& a, int64_t drow, int i) {
  const int64_t at = drow * a.V_d + i;
  return a.dtype == OT_BF16 ? bf16_to_f32(static_cast<const uint16_t*>(a.draft_logits)[at]) : static_cast<const float*>(a.draft_logits)[at];
}
__device__ inline uint16_t f32_to_bf16(float x) {         // to nearest, ties to even; NaN stays one
  const uint32_t u = __float_as_uint(x);
  return x != x ? 0x7FC0 : (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}

// What draft row `drow` needs, all but the mass of its mapped ids in A; by one wavefront.
__device__ inline RowGrad make_row(const LossGradArgs& a, int drow, int lane) {
  RowGrad R = {};
  const int b = uniform(find_sequence(a.row_off, a.B, drow, 1, lane));
  const int r0 = a.row_off[b], at = drow - (r0 - b), m = a.n_mapped[b];
  bool covers = false;
  if (lane < m) {
    const int s = a.span_start[r0 + lane];
    covers = s <= at && at < s + a.span_len[r0 + lane];
  }
  const unsigned long long who = __ballot(covers);
  if (!who) return R;
  const int row = r0 + (int)__builtin_ctzll(who), kind = a.kind[row];
  if (kind == 0) return R;
  const int s = a.span_start[row], L = a.span_len[row], first = r0 - b + s;
  const double T = a.temperature[b], Td = a.draft_temperature ? a.draft_temperature[b] : a.temperature[b];
  R.row = row;
  R.sub = a.draft_ids[drow]; R.out = -1; R.pre = -1;
  R.mxq = a.drow_max[drow]; R.invTd = 1.0 / Td; R.lnSq = log(a.drow_sum[drow]);
  R.mx = a.row_max[row]; R.invT = 1.0 / T; R.lnS = log(a.row_sum[row]);
  R.c = (a.grad_loss ? (double)*a.grad_loss : 1.0) / fmax(1.0, a.totals[2] + a.totals[3]) * R.invTd;
  if (kind == 1) {
    R.kind = 1;
    R.A = a.kl[row];
    return R;
  }
  R.c *= a.weight[row];
  R.D = -R.c;
  R.kind = 2;
  if (!a.approx_kl) return R;
  const int t = a.mapped_ids[row], d1 = a.draft_ids[first], t_pre = a.dmap[d1];
  double lq = 0.0;
  if (lane < L) lq = (draft_logit(a, first + lane, a.draft_ids[first + lane]) - (double)a.drow_max[first + lane]) * R.invTd - log(a.drow_sum[first + lane]);
  double ln_pi = 0.0;
  for (int l = 0; l < L; ++l) ln_pi += __shfl(lq, l);
  const double lq_first = __shfl(lq, 0), pi = exp(ln_pi), q_pre = -exp(lq_first) * expm1(ln_pi - lq_first);   // q(d_1) - pi
  const float* z = a.Z + (int64_t)row * a.ldz;
  const double lp_ng = ((double)z[t] - R.mx) * R.invT - R.lnS;
  const bool has_pre = t_pre >= 0 && t_pre != t && q_pre > 0.0;
  double pull = pi > 0.0 ? ln_pi - lp_ng + 1.0 : 0.0;
  double A = a.kl[row] - (pi > 0.0 ? pi * (ln_pi - lp_ng) : 0.0);
  R.out = a.tmap[t];
  if (t_pre >= 0 && t_pre != t) R.pre = d1;
  if (has_pre) {
    const double lp_pre = ((double)z[t_pre] - R.mx) * R.invT - R.lnS;
    R.a_pre = log(q_pre) - lp_pre + 1.0;
    pull -= R.a_pre;
    A += pi * R.a_pre + q_pre;                           // q(d_1) a_pre in place of q_pre (a_pre - 1)
  }
  R.D = R.c * pi * pull;
  R.A = A;
  if (drow == first) R.kind = 3;
  return R;
}

// One workgroup per draft row.
__global__ __launch_bounds__(256) void loss_grad_kernel(LossGradArgs a) {
  __shared__ RowGrad s_row;
  __shared__ double s_sum[4];
  const int drow = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  if (wave == 0) {
    const RowGrad R = make_row(a, drow, lane);
    if (lane == 0) s_row = R;
  }
  __syncthreads();
  RowGrad R = s_row;
  if (R.kind & 1) {
    double mass = 0.0;
    for (int i = tid; i < a.V_d; i += 256)
      if (a.dmap[i] >= 0 && i != R.out && i != R.pre) mass += exp_neg_fast((draft_logit(a, drow, i) - R.mxq) * R.invTd - R.lnSq);
    mass = wave_sum(mass);
    if (lane == 0) s_sum[wave] = mass;
    __syncthreads();
    R.A += s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
  }
  const float* z = a.Z + (int64_t)R.row * a.ldz;
  for (int i = tid; i < a.V_d; i += 256) {
    double g = 0.0;
    if (R.kind) {
      const double lq = (draft_logit(a, drow, i) - R.mxq) * R.invTd - R.lnSq, q = exp_neg_fast(lq);
      if ((R.kind & 1) && q > 0.0) {
        double e = 0.0;
        if (i == R.pre) e = R.a_pre;
        else if (i != R.out && a.dmap[i] >= 0) e = lq - (((double)z[a.dmap[i]] - R.mx) * R.invT - R.lnS) + 1.0;
        g = R.c * q * (e - R.A);
      }
      if (R.kind & 2) g += R.D * ((i == R.sub ? 1.0 : 0.0) - q);
    }
    const int64_t at = (int64_t)drow * a.V_d + i;
    if (a.dtype == OT_BF16) static_cast<uint16_t*>(a.grad)[at] = f32_to_bf16((float)g);
    else static_cast<float*>(a.grad)[at] = (float)g;
  }
}

}  // namespace

hipError_t launch_loss_grad(const LossGradArgs& a, hipStream_t stream) {
  if (a.K == 0) return hipSuccess;
  hipLaunchKernelGGL(loss_grad_kernel, dim3((unsigned)a.K), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace otv
