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
  double c, A, D, a_pre;
  int32_t kind;                 // 0: zeros, 1: the KL part, 2: D alone, 3: both
  int32_t row, sub;             // the token's target row; the draft row's drafted id
  int32_t out, pre;             // draft ids whose a is 0 / a_pre, or -1
};

template <typename T> struct Draft;
template <> struct Draft<float> {
  static constexpr int kElems = 4;
  __device__ static float one(const float* p) { return *p; }
  __device__ static void load(const float* p, float* x) {
    typedef float raw_t __attribute__((ext_vector_type(4)));
    const raw_t r = *reinterpret_cast<const raw_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = r[i];
  }
  __device__ static void store_one(float* p, float x) { *p = x; }
  __device__ static void store(float* p, const float* x) {
    typedef float raw_t __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(raw_t{x[0], x[1], x[2], x[3]}, reinterpret_cast<raw_t*>(p));
  }
};
template <> struct Draft<uint16_t> {
  static constexpr int kElems = 8;
  typedef uint32_t raw_t __attribute__((ext_vector_type(4)));
  __device__ static float one(const uint16_t* p) { return bf16_to_f32(*p); }
  __device__ static void load(const uint16_t* p, float* x) {
    const raw_t r = *reinterpret_cast<const raw_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(r[i] << 16); x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u); }
  }
  __device__ static void store_one(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }   // to nearest
  __device__ static void store(uint16_t* p, const float* x) {
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
    typedef float two_t __attribute__((ext_vector_type(2)));
    raw_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two_t{x[2 * i], x[2 * i + 1]}, pair_t));
    __builtin_nontemporal_store(r, reinterpret_cast<raw_t*>(p));
  }
};

// What draft row `drow` needs; by one wavefront.  Everything about its sequence's window is asked for at once, lane j holding mapped token j,
// or drafted token j; what hangs on the token that covers the row comes with one round trip more.
template <typename T>
__device__ inline RowGrad make_row(const LossGradArgs& a, int drow, int lane) {
  RowGrad R = {};
  const int b = uniform(find_sequence(a.row_off, a.B, drow, 1, lane));
  const int r0 = uniform(a.row_off[b]), r1 = uniform(a.row_off[b + 1]), q0 = r0 - b, at = drow - q0;
  const int r = min(r0 + lane, r1 - 1), q = max(q0, min(q0 + lane, r1 - b - 2));
  const int m = a.n_mapped[b], s_l = a.span_start[r], len_l = a.span_len[r], kind_l = a.kind[r], t_l = a.mapped_ids[r], id_l = a.draft_ids[q];
  const float T_b = a.temperature[b], Td_b = a.draft_temperature ? a.draft_temperature[b] : T_b;
  const double kl_l = a.kl[r], mass_l = a.mass[r], weight_l = a.weight[r], sum_l = a.row_sum[r], dsum_l = a.drow_sum[q];
  const float mx_l = a.row_max[r], dmx_l = a.drow_max[q], up = a.grad_loss ? *a.grad_loss : 1.f;
  const double n = fmax(1.0, a.totals[2] + a.totals[3]);
  const unsigned long long who = __ballot(lane < m && s_l <= at && at < s_l + len_l);
  if (!who) return R;
  const int j = (int)__builtin_ctzll(who), kind = __shfl(kind_l, j), s = __shfl(s_l, j), L = __shfl(len_l, j);
  if (kind == 0) return R;
  R.row = r0 + j;
  R.sub = __shfl(id_l, at); R.out = -1; R.pre = -1;
  R.invTd = 1.0 / (double)Td_b; R.invT = 1.0 / (double)T_b;
  const double lnSq_l = log(dsum_l);
  R.mxq = (double)__shfl(dmx_l, at); R.lnSq = __shfl(lnSq_l, at);
  R.mx = (double)__shfl(mx_l, j); R.lnS = log(__shfl(sum_l, j));
  R.c = (double)up / n * R.invTd;
  R.kind = 1;
  R.A = __shfl(kl_l, j) + __shfl(mass_l, j);
  if (kind == 1) return R;
  R.c *= __shfl(weight_l, j);
  R.D = -R.c;
  R.kind = 2;
  if (!a.approx_kl) return R;
  const int t = __shfl(t_l, j), d1 = __shfl(id_l, s);
  const float* z = a.Z + (int64_t)R.row * a.ldz;
  const float zq = Draft<T>::one(static_cast<const T*>(a.draft_logits) + (int64_t)q * a.V_d + id_l), z_t = z[t];
  const int t_pre = a.dmap[d1];
  R.out = a.tmap[t];
  const double lq = ((double)zq - (double)dmx_l) * R.invTd - lnSq_l;   // of the lane's drafted token
  double ln_pi = 0.0;
  for (int l = s; l < s + L; ++l) ln_pi += __shfl(lq, l);
  // q(d_1) - pi as a product: next to each other (a drafter sure of the other sub-tokens) the difference would keep nothing
  const double lq_first = __shfl(lq, s), pi = exp(ln_pi), q_pre = -exp(lq_first) * expm1(ln_pi - lq_first);
  const double lp_ng = ((double)z_t - R.mx) * R.invT - R.lnS;
  const bool has_pre = t_pre >= 0 && t_pre != t && q_pre > 0.0;
  double pull = pi > 0.0 ? ln_pi - lp_ng + 1.0 : 0.0;
  double A = R.A - (pi > 0.0 ? pi * (ln_pi - lp_ng) : 0.0);
  if (t_pre >= 0 && t_pre != t) R.pre = d1;
  if (has_pre) {
    const double lp_pre = ((double)z[t_pre] - R.mx) * R.invT - R.lnS;
    R.a_pre = log(q_pre) - lp_pre + 1.0;
    pull -= R.a_pre;
    A += pi * R.a_pre + q_pre;                           // q(d_1) a_pre in place of q_pre (a_pre - 1)
  }
  R.D = R.c * pi * pull;
  R.A = A;
  if (at == s) R.kind = 3;
  return R;
}

// Grid = groups of draft ids x draft rows, the groups of a row on one XCD back to back, so that its L2 holds the target row that they gather
// from (across all of them: 58 us for 128 rows of 32000 ids with the loss in front).  A thread has whole vectors of its row, laid out from the 16-byte boundary at or before the row's
// start; the row's ends go element by element.
constexpr int kGradVecs = 2;
template <typename T>
constexpr int kGradIds = 256 * kGradVecs * Draft<T>::kElems;
template <typename T>
__global__ __launch_bounds__(256) void loss_grad_kernel(LossGradArgs a, int groups) {
  constexpr int kVec = Draft<T>::kElems, kEach = kGradVecs * kVec;
  typedef int image_t __attribute__((ext_vector_type(4), aligned(4)));
  __shared__ RowGrad s_row;
  const int slot = (int)(blockIdx.x >> 3), drow = slot / groups * 8 + (int)(blockIdx.x & 7u), tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  if (drow >= a.K) return;                               // padding of the id space
  const T* zq = static_cast<const T*>(a.draft_logits) + (int64_t)drow * a.V_d;
  T* grad = static_cast<T*>(a.grad) + (int64_t)drow * a.V_d;
  const int shift = (int)(reinterpret_cast<uintptr_t>(zq) / sizeof(T)) & (kVec - 1);
  const bool vectors = ((int)(reinterpret_cast<uintptr_t>(grad) / sizeof(T)) & (kVec - 1)) == shift;
  const int v0 = slot % groups * kGradIds<T> - shift + tid * kVec;
  auto first = [&](int i) { return v0 + i * 256 * kVec; };
  auto whole = [&](int i) { return vectors && first(i) >= 0 && first(i) + kVec <= a.V_d; };
  float x[kEach];
  int image[kEach];
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) {
    if (whole(i)) {
      Draft<T>::load(zq + first(i), x + i * kVec);
#pragma unroll
      for (int e = 0; e < kVec; e += 4) {
        const image_t r = *reinterpret_cast<const image_t*>(a.dmap + first(i) + e);
#pragma unroll
        for (int f = 0; f < 4; ++f) image[i * kVec + e + f] = r[f];
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const bool in_it = first(i) + e >= 0 && first(i) + e < a.V_d;
        x[i * kVec + e] = in_it ? Draft<T>::one(zq + first(i) + e) : -INFINITY;
        image[i * kVec + e] = in_it ? a.dmap[first(i) + e] : -1;
      }
    }
  }
  if (wave == 0) {
    const RowGrad R = make_row<T>(a, drow, lane);
    if (lane == 0) s_row = R;
  }
  __syncthreads();
  const RowGrad R = s_row;
  float out[kEach];
  if (R.kind & 1) {
    const float* z = a.Z + (int64_t)R.row * a.ldz;
    float zv[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) zv[e] = z[max(image[e], 0)];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = first(e / kVec) + e % kVec;
      const double lq = ((double)x[e] - R.mxq) * R.invTd - R.lnSq, q = exp_neg_fast(lq);
      double r = image[e] >= 0 && i != R.out ? lq - (((double)zv[e] - R.mx) * R.invT - R.lnS) + 1.0 : 0.0;
      if (i == R.pre) r = R.a_pre;
      double g = q > 0.0 ? R.c * q * (r - R.A) : 0.0;
      if (R.kind & 2) g += R.D * ((i == R.sub ? 1.0 : 0.0) - q);
      out[e] = (float)g;
    }
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = first(e / kVec) + e % kVec;
      out[e] = R.kind ? (float)(R.D * ((i == R.sub ? 1.0 : 0.0) - exp_neg_fast(((double)x[e] - R.mxq) * R.invTd - R.lnSq))) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kGradVecs; ++i) {
    if (whole(i)) {
      Draft<T>::store(grad + first(i), out + i * kVec);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (first(i) + e >= 0 && first(i) + e < a.V_d) Draft<T>::store_one(grad + first(i) + e, out[i * kVec + e]);
    }
  }
}

template <typename T>
hipError_t launch(const LossGradArgs& a, hipStream_t stream) {
  const int groups = ceil_div((int64_t)a.V_d + 7, kGradIds<T>);   // a row starts up to 7 elements into its first vector
  const int64_t grid = (int64_t)groups * ceil_div(a.K, 8) * 8;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL(loss_grad_kernel<T>, dim3((unsigned)grid), dim3(256), 0, stream, a, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_loss_grad(const LossGradArgs& a, hipStream_t stream) {
  if (a.K == 0) return hipSuccess;
  return a.dtype == OT_BF16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}

}  // namespace otv
