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
// A draft row that the drafter's mask leaves empty has no mass: nothing is added for it, and its gradient is 0.  One with a NaN or +inf has
// no distribution: its KL value and gradient are NaN.
// A needs no sum of its own over the target row: it is sum q' (ln q' - ln p), the loss's value, plus the mass of q on the ids that
// have an image (less and plus the overrides' terms).
//
// Two forms (loss_grad_in_one): behind the loss's launch, which leaves that value and the mass, a gather from the target row by
// draft id (loss_grad_kernel); or loss and gradient of a draft row in one workgroup (loss_row_kernel), which reads the target row in order.
// Bound by memory: every 128-byte line of a target row holds an image, so it is read whole.  128 rows of 32000 ids against 128256 30 us
// (2.7 TB/s: a chain of steps per row, one row per workgroup, below), 384 against 152064 65 us (3.7 TB/s).
#include "device_math.h"
#include "otv_internal.h"

namespace otv {
namespace {

// 0, or NaN where the row's sum is.
__device__ inline double nan_of(double lnS) { return lnS != lnS ? lnS : 0.0; }

// A drafter is sure of a row's likeliest id where the others' sum of exponentials is below an eighth of its own.
constexpr double kSureSum = 1.125;

struct RowGrad {
  double mxq, invTd, lnSq;      // ln q(i) = (zq_i - mxq) * invTd - lnSq
  double mx, invT, lnS;         // ln p(v) = (z_v - mx) * invT - lnS
  double c, A, D, a_pre;
  double none;                  // what an id with q = 0 gets: 0, or NaN in a row without a distribution
  int32_t kind;                 // 0: zeros, 1: the KL part, 2: D alone, 3: both
  int32_t row, sub;             // the token's target row; the draft row's drafted id
  int32_t out, pre;             // draft ids whose a is 0 / a_pre, or -1
  int32_t top;                  // the likeliest id of a sure drafter, or -1
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
  const int arg_l = a.drow_arg[q];
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
  R.none = nan_of(R.lnSq);
  const int arg = __shfl(arg_l, at);
  const double Sq = __shfl(dsum_l, at);
  R.top = Sq > 0.0 && Sq < kSureSum ? arg : -1;
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

// ln q of a draft logit, and ln p of a target logit, of a row.
__device__ inline double ln_q(const RowGrad& R, float x) { return ((double)x - R.mxq) * R.invTd - R.lnSq; }
__device__ inline double ln_p(const RowGrad& R, float z) { return ((double)z - R.mx) * R.invT - R.lnS; }
// The gradient at draft id i of a row with (kKl) or without a KL part; x: its logit, z: the target's logit at its image.
template <bool kKl>
__device__ inline float grad_at(const RowGrad& R, int i, float x, int image, float z) {
  const double lq = ln_q(R, x), q = exp_neg_fast(lq), pull = R.D * ((i == R.sub ? 1.0 : 0.0) - q) + R.none;
  if (!kKl) return (float)pull;
  double r = image >= 0 && i != R.out ? lq - ln_p(R, z) + 1.0 : 0.0;
  if (i == R.pre) r = R.a_pre;
  double g = q > 0.0 ? R.c * q * (r - R.A) : R.none;
  if (R.kind & 2) g += pull;
  return (float)g;
}

// The gradient at a sure drafter's likeliest id, by a workgroup: what loss_row_kernel says of it, with the others' mass summed here.  q a of that
// id comes off A as the loss's launch put it there, in 64 bits.  s_sum: 4 numbers of shared memory.
template <typename T>
__device__ inline float grad_at_top(const LossGradArgs& a, const RowGrad& R, const T* zq, int shift, int tid, double* s_sum) {
  constexpr int kVec = Draft<T>::kElems, kAtOnce = 32 / kVec;
  const float mxq = (float)R.mxq, s2 = (float)(R.invTd * 1.4426950408889634);
  auto q_of = [&](float x) { return __builtin_amdgcn_exp2f(fmaxf(x - mxq, -1e30f) * s2); };   // times the row's sum
  double rest = 0.0;
  const int vecs = (a.V_d + shift) / kVec;               // whole ones, from the 16-byte boundary at or before the row's start; its ends one by one
  for (int v = tid + 1; v < vecs; v += 256 * kAtOnce) {
    float x[kAtOnce][kVec];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) Draft<T>::load(zq - shift + min(v + 256 * j, vecs - 1) * kVec, x[j]);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < kVec; ++e) part += (v + 256 * j) * kVec - shift + e != R.top ? q_of(x[j][e]) : 0.f;
      if (v + 256 * j < vecs) rest += (double)part;
    }
  }
  const int first = min(kVec - shift, a.V_d), last = max(vecs * kVec - shift, first), i = tid < first ? tid : last + tid - first;
  if (i < a.V_d && i != R.top) rest += (double)q_of(Draft<T>::one(zq + i));
  rest = wave_sum(rest);
  if ((tid & 63) == 0) s_sum[tid >> 6] = rest;
  __syncthreads();
  const double others = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), mass = others / (1.0 + others), q_top = 1.0 - mass;
  const double pull = R.kind & 2 ? R.D * (R.top == R.sub ? mass : -q_top) : 0.0;
  if (!(R.kind & 1)) return (float)pull;
  const double lq = -R.lnSq;
  const int image = a.dmap[R.top];
  double a_top = 0.0, A_rest = R.A;
  if (R.top == R.pre) {
    a_top = R.a_pre;
    A_rest -= exp(lq) * a_top;
  } else if (image >= 0 && R.top != R.out) {
    a_top = lq - ln_p(R, a.Z[(int64_t)R.row * a.ldz + image]) + 1.0;
    A_rest -= exp_neg_fast(lq) * a_top;
  }
  return (float)(pull + R.c * q_top * (a_top * mass - A_rest));
}

// Grid = groups of draft ids x draft rows, the groups of a row on one XCD back to back, so that its L2 holds the target row that they gather
// from (across all of them: 58 us for 128 rows of 32000 ids with the loss in front).  A thread has whole vectors of its row, laid out from
// the 16-byte boundary at or before the row's start; the row's ends go element by element.
constexpr int kGradVecs = 2;
template <typename T>
constexpr int kGradIds = 256 * kGradVecs * Draft<T>::kElems;
template <typename T>
__global__ __launch_bounds__(256) void loss_grad_kernel(LossGradArgs a, int groups) {
  constexpr int kVec = Draft<T>::kElems, kEach = kGradVecs * kVec;
  typedef int image_t __attribute__((ext_vector_type(4), aligned(4)));
  __shared__ RowGrad s_row;
  __shared__ double s_sum[4];
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
    for (int e = 0; e < kEach; ++e) out[e] = grad_at<true>(R, first(e / kVec) + e % kVec, x[e], image[e], zv[e]);
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e) out[e] = R.kind ? grad_at<false>(R, first(e / kVec) + e % kVec, x[e], -1, 0.f) : 0.f;
  }
  const int first_id = slot % groups * kGradIds<T> - shift;
  if (R.kind != 0 && R.top >= max(first_id, 0) && R.top < first_id + kGradIds<T>) {   // the same in the whole workgroup
    const float g = grad_at_top(a, R, zq, shift, tid, s_sum);
#pragma unroll
    for (int e = 0; e < kEach; ++e) out[e] = first(e / kVec) + e % kVec == R.top ? g : out[e];
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

// ------------------------------------------------------------------------------------------------ loss and gradient of a row in one workgroup
// Where a row of draft ids fits LDS, 4 bytes each, and the q' rows are not wanted, two launches do the loss's work as well:
//   loss_prepare_kernel  one wavefront per sequence: kinds, NLL and weights of its tokens, the number of drafted tokens considered (whole
//                        numbers added by atomics: the order does not matter), and a record of what every draft row needs;
//   loss_row_kernel      one workgroup per draft row.  It walks the mapped pairs in ascending target id, so that the target row is read in
//                        order, and leaves each logit in LDS at its draft id; then it walks its draft row, which it holds in registers, for
//                        q, r and their sums, and a second time for the gradient.  The last workgroup of all forms the loss's totals.
// Of 30 us for 128 rows of 32000 ids the record's round trip takes 2.7, clearing LDS 1.7, the pairs 9.7, the two sweeps 2.2 and 1.4, the sums
// 2.6, arrival and totals 2.4, and the launch in front 4.
// What the row kernel computes is float32 with the constants (maxima, ln S) apart: t = (zq - mxq)/Td - (z - mx)/T is formed without them, and
// sum q t gets the constants' part as their 64-bit difference times the mass of q.
// The likeliest id of a row of which it has nearly all of q (kSureSum) is left out of the sums: with `rest` the mass of the others, its 1 - q is
// rest, and a - A = a rest - (sum q a of the others).  Formed from q, both would be what is left of numbers next to each other: the rows'
// sums, which the step leaves, know 1 - q to 2^-24 at best, and with float32 q nothing below that came out right (rows of 1 - q = 1e-8 were
// off by 14 times their gradient).
// Rows for which that arithmetic leaves float32's range are done as the other form does all of them, in 64 bits and from memory: those of
// temperatures below 2.1e-8 (kMostScale), where exponents overflow; and those that propose an id which the target masks (with -inf, or with a
// number as low as -1e20): its term is infinite or nearly, however small q is, and a q below 2^-126 is not there in float32.  An n-gram's
// overrides that the target masks show in the record's numbers.
constexpr float kMostScale = 0x1p26f;
struct alignas(16) GradRow {
  float mx, mxq;                // t = (zq - mxq) * s2q and (z - mx) * s2: exponents to base 2, s2 as two floats
  float s2, s2_lo, s2q;         // (the row sums' exponents were formed with one float of log2(e)/Td as well)
  float r0, inv_Sq;             // q = 2^t / Sq;  r = (tq - t) ln 2 + r0, r0 = lnS - lnSq + 1
  double dlnS;                  // lnS - lnSq
  double c, D, a_pre;           // c and D without grad_loss / n
  double kl_more, A_more;       // what Eq. 2's overrides add to the KL sum and to A
  double invTd, lnSq, invT, lnS;   // for rows in 64 bits
  int32_t kind;                 // RowGrad's, and 4: in 64 bits
  int32_t row, sub, out, pre;
  int32_t top;                  // the likeliest id of a sure drafter, or -1
};
static_assert(sizeof(GradRow) % 16 == 0, "read as 16-byte units");

template <typename T>
__global__ __launch_bounds__(256) void loss_prepare_kernel(LossGradArgs a) {
  const int lane = threadIdx.x & 63, b = (int)blockIdx.x * 4 + uniform((int)threadIdx.x >> 6);
  if (b >= a.B) return;
  const int r0 = uniform(a.row_off[b]), r1 = uniform(a.row_off[b + 1]), q0 = r0 - b, k = r1 - r0 - 1;
  const int r = min(r0 + lane, r1 - 1), q = q0 + max(0, min(lane, k - 1));
  const float T_b = a.temperature[b], Td_b = a.draft_temperature ? a.draft_temperature[b] : T_b;
  const int m = a.n_mapped[b], n_accept = a.n_accept[b], s = a.span_start[r], L = a.span_len[r], t = a.mapped_ids[r];
  const float p_tok = a.p_tok[r], mx = a.row_max[r];
  const double lnS = log(a.row_sum[r]);
  int id = 0;
  float mxq = 0.f;
  double Sq = 1.0, lq = 0.0;
  const double invT = 1.0 / (double)T_b, invTd = 1.0 / (double)Td_b;
  const bool counts = T_b > 0.f && Td_b > 0.f;
  int top = -1;
  if (k > 0 && counts && m > 0) {                        // (ids outside the vocabulary: nothing is mapped)
    id = a.draft_ids[q];
    mxq = a.drow_max[q];
    Sq = a.drow_sum[q];
    if (Sq > 0.0 && Sq < kSureSum) top = a.drow_arg[q];
    lq = ((double)Draft<T>::one(static_cast<const T*>(a.draft_logits) + (int64_t)q * a.V_d + id) - (double)mxq) * invTd - log(Sq);
  }
  const double lnSq = log(Sq);
  // lane j: mapped token j
  const bool mine = lane < k + 1;
  int kind = 0;
  if (mine && lane < m && counts) kind = L == 1 ? 1 : (!a.accepted_only || lane < n_accept) ? 2 : 0;
  const int first = max(s, 0), d1 = __shfl(id, first);
  double ln_pi = 0.0;
  const double lq_first = __shfl(lq, first);
  for (int l = 0; l < OT_MAX_NGRAM_LEN; ++l) {
    const double x = __shfl(lq, min(first + l, 63));
    if (l < L) ln_pi += x;
  }
  const double weight = kind != 2 ? 0.0 : a.lambda_mode == OT_LAMBDA_TARGET_PROB ? (double)p_tok : (double)a.lambda;
  int n = kind == 1 ? 1 : kind == 2 ? L : 0;
  double D = -weight * invTd, c = kind == 1 ? invTd : weight * invTd, a_pre = 0.0, kl_more = 0.0, A_more = 0.0;
  int out = -1, pre = -1;
  const bool ngram_kl = kind == 2 && a.approx_kl;
  if (ngram_kl) {
    const float* z = a.Z + (int64_t)r * a.ldz;
    const int t_pre = a.dmap[d1];
    out = a.tmap[t];
    const double pi = exp(ln_pi), q_pre = -exp(lq_first) * expm1(ln_pi - lq_first);   // q(d_1) - pi, as in make_row
    const double lp_ng = ((double)z[t] - (double)mx) * invT - lnS;
    double pull = 0.0;
    if (pi > 0.0) {
      pull = ln_pi - lp_ng + 1.0;
      kl_more = pi * (ln_pi - lp_ng);
    }
    if (t_pre >= 0 && t_pre != t) {
      pre = d1;
      if (q_pre > 0.0) {
        const double lp_pre = ((double)z[t_pre] - (double)mx) * invT - lnS;
        a_pre = log(q_pre) - lp_pre + 1.0;
        pull -= a_pre;
        kl_more += q_pre * (a_pre - 1.0);
        A_more = exp(lq_first) * a_pre;
      }
    }
    D = c * pi * pull;
  }
  if (mine) {
    a.out.kind[r0 + lane] = kind;
    a.out.nll[r0 + lane] = kind == 2 ? -ln_pi : 0.0;
    a.out.weight[r0 + lane] = weight;
    a.out.kl[r0 + lane] = 0.0;                           // of rows without a KL term; the others' workgroups write theirs
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) n += __shfl_xor(n, o);
  if (lane == 0 && n > 0) __hip_atomic_fetch_add(a.n_tokens, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // lane i: draft row i, covered by the last token that starts at or before it
  unsigned long long starts = mine && lane < m ? 1ull << (first & 63) : 0ull;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) starts |= __shfl_xor(starts, o);
  const int j = max(0, (int)__popcll(starts & ((2ull << lane) - 1)) - 1);
  const int s_j = __shfl(first, j), L_j = __shfl(L, j), kind_j = __shfl(kind, j);
  const bool covered = (starts & ((2ull << lane) - 1)) != 0 && lane < s_j + L_j && kind_j != 0, is_first = lane == s_j;
  GradRow R = {};
  R.row = r0 + j;
  R.mx = __shfl(mx, j); R.mxq = mxq;
  const double s2 = 1.4426950408889634 * invT, s2q = 1.4426950408889634 * invTd;
  R.s2 = (float)s2; R.s2_lo = (float)(s2 - (double)R.s2);
  R.s2q = (float)s2q;
  R.inv_Sq = Sq == 0.0 ? 0.f : (float)(1.0 / Sq);
  R.lnS = __shfl(lnS, j);
  R.dlnS = Sq == 0.0 ? 0.0 : R.lnS - lnSq;               // (times the mass, which is 0 then)
  R.r0 = (float)(R.dlnS + 1.0);
  R.c = __shfl(c, j); R.D = __shfl(D, j); R.a_pre = __shfl(a_pre, j);
  R.kl_more = __shfl(kl_more, j); R.A_more = __shfl(A_more, j);
  R.out = __shfl(out, j); R.pre = __shfl(pre, j); R.sub = id; R.top = top;
  const int ngram_kl_j = __shfl((int)ngram_kl, j);
  R.invTd = invTd; R.lnSq = lnSq; R.invT = invT;
  R.kind = !covered ? 0 : kind_j == 1 ? 1 : !ngram_kl_j ? 2 : is_first ? 3 : 2;
  const double most = fmax(fmax(fabs(R.a_pre), fabs(R.A_more)), fabs(R.D) + fabs(R.c));   // (a NaN of D shows in the comparison)
  if (R.kind != 0 && !(fmaxf(R.s2, R.s2q) <= kMostScale && most <= 1e20)) R.kind |= 4;
  if (lane < k) static_cast<GradRow*>(a.rows)[q0 + lane] = R;
}

// The sums over all rows and the mean, by a workgroup.
__device__ inline void grad_totals(const LossGradArgs& a, int tid, int wave, int lane, double (*s_term)[16]) {
  double term[4] = {0.0, 0.0, 0.0, 0.0};                // direct, n-gram, direct tokens, n-gram sub-tokens
  for (int row = tid; row < a.M; row += 1024) {
    const int kind = a.out.kind[row];
    const double kl = observe(a.out.kl + row), nll = a.out.nll[row], weight = a.out.weight[row];
    if (kind == 1) {
      term[0] += kl;
      term[2] += 1.0;
    } else if (kind == 2) {
      term[1] += weight * (a.approx_kl ? kl : nll);
      term[3] += (double)a.span_len[row];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double t = wave_sum(term[i]);
    if (lane == 0) s_term[i][wave] = t;
  }
  __syncthreads();
  if (wave != 0) return;
  double t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = wave_sum(lane < 16 ? s_term[i][lane] : 0.0);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a.out.totals[i] = t[i];
    a.out.totals[4] = (t[0] + t[1]) / fmax(1.0, t[2] + t[3]);
  }
}

constexpr uint32_t kNoImage = 0x7FC0D0E5u;               // in LDS: the draft id has no image (a NaN that no arithmetic gives)
constexpr int kRowThreads = 1024;
template <typename T, int kVecs>
__global__ __launch_bounds__(kRowThreads) void loss_row_kernel(LossGradArgs a) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  constexpr int kVec = Draft<T>::kElems, kEach = kVecs * kVec, kPairs = 8;
  extern __shared__ __attribute__((aligned(16))) float s_z[];   // [shift + id]: the target's logit at the id's image, then r
  __shared__ double s_term[5][16];                       // a row for each sum: nothing is written again before the totals
  __shared__ int s_last, s_far;
  __shared__ float s_top;                                // the target's logit at the likeliest id's image
  const int drow = blockIdx.x, tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const T* zq = static_cast<const T*>(a.draft_logits) + (int64_t)drow * a.V_d;
  T* grad = static_cast<T*>(a.grad) + (int64_t)drow * a.V_d;
  const int shift = (int)(reinterpret_cast<uintptr_t>(zq) / sizeof(T)) & (kVec - 1);
  const bool vectors = ((int)(reinterpret_cast<uintptr_t>(grad) / sizeof(T)) & (kVec - 1)) == shift;
  const GradRow R = static_cast<const GradRow*>(a.rows)[drow];
  const int n_tokens = *a.n_tokens;
  const float up = a.grad_loss ? *a.grad_loss : 1.f;
  const int v0 = tid * kVec - shift;                     // the thread's vector i holds ids v0 + i * kRowThreads * kVec ..
  auto first = [&](int i) { return v0 + i * kRowThreads * kVec; };
  auto whole = [&](int i) { return vectors && first(i) >= 0 && first(i) + kVec <= a.V_d; };
  int2 id[kPairs] = {};
  auto load_pairs = [&](int at, int2* to) {
#pragma unroll
    for (int e = 0; e < kPairs; ++e) to[e] = a.pairs[max(0, min(at + e * kRowThreads, a.n_pairs - 1))];
  };
  if (a.n_pairs > 0) load_pairs(tid, id);
  float x[kEach];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    if (whole(i)) {
      Draft<T>::load(zq + first(i), x + i * kVec);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[i * kVec + e] = first(i) + e >= 0 && first(i) + e < a.V_d ? Draft<T>::one(zq + first(i) + e) : -INFINITY;
    }
  }
  const float scale = up / (float)max(1, n_tokens), c = (float)R.c * scale, D = (float)R.D * scale;
  auto q_of = [&](float zq_i, float* tq) {
    const float d = fmaxf(zq_i - R.mxq, -1e30f);         // an id masked with -inf: q = 0, and no -inf times a low part of 0
    *tq = d * R.s2q;
    return __builtin_amdgcn_exp2f(*tq) * R.inv_Sq;
  };
  const int top_vec = R.kind != 0 && R.top >= 0 ? (shift + R.top) / (kRowThreads * kVec) : -1;   // the vectors that hold the likeliest id
  // while the record and the pairs are on their way
  const int slots = (a.V_d + shift + kVec - 1) / kVec * (kVec / 4);   // whole vectors, as they are read
  for (int i = tid; i < slots; i += kRowThreads) {
    const float none = __uint_as_float(kNoImage);
    reinterpret_cast<f32x4*>(s_z)[i] = f32x4{none, none, none, none};
  }
  // Counts the row in: its KL value has reached memory, and every wavefront has read the number of tokens (a barrier lies in front), which
  // the last workgroup of all puts back to 0.
  auto count_in = [&]() {
    s_last = arrive(a.count, a.K);
    if (s_last) publish(a.n_tokens, 0);
  };
  float A = 0.f, out_top = 0.f;
  asm volatile("" ::"v"(scale));                         // read by now
  if (tid == 0) s_far = R.kind & 4;
  __syncthreads();
  const float* z = a.Z + (int64_t)R.row * a.ldz;
  bool wide = (R.kind & 4) != 0;                         // in 64 bits; the same in all threads
  if ((R.kind & 1) && !wide) {
    // a turn's logits are asked for a turn ahead, their ids two
    float zv[kPairs];
    int2 id_next[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) zv[e] = z[id[e].x];
    if (kPairs * kRowThreads < a.n_pairs) load_pairs(tid + kPairs * kRowThreads, id_next);
    for (int at = tid; at - tid < a.n_pairs; at += kPairs * kRowThreads) {
      float z_next[kPairs] = {};
      int2 id_after[kPairs] = {};
      if (at - tid + kPairs * kRowThreads < a.n_pairs) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) z_next[e] = z[id_next[e].x];
      }
      if (at - tid + 2 * kPairs * kRowThreads < a.n_pairs) load_pairs(at + 2 * kPairs * kRowThreads, id_after);
#pragma unroll
      for (int e = 0; e < kPairs; ++e)
        if (at + e * kRowThreads < a.n_pairs) s_z[shift + id[e].y] = zv[e];
#pragma unroll
      for (int e = 0; e < kPairs; ++e) { id[e] = id_next[e]; id_next[e] = id_after[e]; zv[e] = z_next[e]; }
    }
    __syncthreads();
    if ((R.kind & 2) && tid == 0) {                      // Eq. 2's overrides are not among the ordinary ids
      if (R.out >= 0) s_z[shift + R.out] = __uint_as_float(kNoImage);
      if (R.pre >= 0) s_z[shift + R.pre] = __uint_as_float(kNoImage);
    }
    if (R.kind & 2) __syncthreads();
    if (R.top >= 0 && tid == (shift + R.top) / kVec % kRowThreads) s_top = s_z[shift + R.top];   // its own word, below
    double kl = 0.0, mass = 0.0;
    float rest_own = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int base = (i * kRowThreads + tid) * kVec;   // slot of the vector's first id
      if (base < shift + a.V_d) {
        float zr[kVec], kl_i = 0.f, mass_i = 0.f;
#pragma unroll
        for (int e = 0; e < kVec; e += 4) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(s_z + base + e);
#pragma unroll
          for (int f = 0; f < 4; ++f) zr[e + f] = w[f];
        }
        if (i == top_vec) {                              // the likeliest id stays out of the sums
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[i * kVec + e] = base - shift + e == R.top ? -INFINITY : x[i * kVec + e];
        }
        bool far = false;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          float tq;
          const float q = q_of(x[i * kVec + e], &tq), d = zr[e] - R.mx;
          const bool ordinary = __float_as_uint(zr[e]) != kNoImage, near = ordinary && !(d < -1e20f);
          const float diff = near ? (tq - fmaf(d, R.s2, d * R.s2_lo)) * 0.69314718f : 0.f;
          kl_i = fmaf(q, diff, kl_i);
          mass_i += ordinary ? q : 0.f;
          rest_own += q;
          far |= ordinary && !near && tq > -1080.f;      // in 64 bits q may be above 0
          zr[e] = near ? diff + R.r0 : 0.f;
          x[i * kVec + e] = q;
        }
        if (far) s_far = 4;
#pragma unroll
        for (int e = 0; e < kVec; e += 4) *reinterpret_cast<f32x4*>(s_z + base + e) = f32x4{zr[e], zr[e + 1], zr[e + 2], zr[e + 3]};
        kl += (double)kl_i;
        mass += (double)mass_i;
      }
    }
    kl = wave_sum(kl);
    mass = wave_sum(mass);
    double rest = wave_sum((double)rest_own);
    if (lane == 0) { s_term[0][wave] = kl; s_term[1][wave] = mass; s_term[4][wave] = rest; }
    __syncthreads();
    wide = s_far != 0;
    kl = wave_sum(lane < 16 ? s_term[0][lane] : 0.0);
    mass = wave_sum(lane < 16 ? s_term[1][lane] : 0.0);
    rest = wave_sum(lane < 16 ? s_term[4][lane] : 0.0);
    kl += R.dlnS * mass;                                 // sum over ordinary ids of q (ln q - ln p)
    double A_rest = kl + mass + (R.pre == R.top ? 0.0 : R.A_more), a_top = 0.0;
    if (R.top >= 0) {
      const double q_top = 1.0 - rest;
      if (R.pre == R.top) {
        a_top = R.a_pre;
      } else if (__float_as_uint(s_top) != kNoImage) {
        const double diff = -R.lnSq - (((double)s_top - (double)R.mx) * R.invT - R.lnS);
        a_top = diff + 1.0;
        kl += q_top * diff;
        wide |= diff > 1e20;                             // masked by the target
      }
      A = (float)(A_rest + q_top * a_top);
      out_top = (float)(R.c * (double)scale * q_top * (a_top * rest - A_rest));
      if (R.kind & 2) out_top += (float)(R.D * (double)scale * (R.top == R.sub ? rest : -q_top));
    } else {
      A = (float)A_rest;
    }
    if (R.kind & 2) {
      if (tid == 0 && R.pre >= 0) s_z[shift + R.pre] = (float)R.a_pre;
      __syncthreads();
    }
    if (tid == 0 && !wide) {
      publish(a.out.kl + R.row, kl + R.kl_more);
      count_in();
    }
  } else if (R.kind == 2 && R.top >= 0) {                // without a KL part: what is left of the likeliest id
    float rest_own = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      float tq;
      rest_own += q_of(first(i / kVec) + i % kVec == R.top ? -INFINITY : x[i], &tq);
    }
    double rest = wave_sum((double)rest_own);
    if (lane == 0) s_term[4][wave] = rest;
    __syncthreads();
    rest = wave_sum(lane < 16 ? s_term[4][lane] : 0.0);
    out_top = (float)(R.D * (double)scale * (R.top == R.sub ? rest : rest - 1.0));
    if (tid == 0) count_in();
  } else if (!wide && tid == 0) {
    count_in();
  }
  if (wide) {
    RowGrad X;
    X.mxq = (double)R.mxq; X.invTd = R.invTd; X.lnSq = R.lnSq; X.mx = (double)R.mx; X.invT = R.invT; X.lnS = R.lnS;
    X.c = R.c * (double)up / (double)max(1, n_tokens); X.D = R.D * (double)up / (double)max(1, n_tokens);
    X.a_pre = R.a_pre; X.kind = R.kind; X.sub = R.sub; X.out = R.out; X.pre = R.pre;
    X.none = nan_of(X.lnSq);
    double kl = X.none, mass = 0.0;
    for (int i = tid; (R.kind & 1) && i < a.V_d; i += kRowThreads) {
      const int image = a.dmap[i];
      if (image < 0 || i == R.out || i == R.pre) continue;
      const double lq = ln_q(X, Draft<T>::one(zq + i)), q = exp_neg_fast(lq);
      mass += q;
      if (q > 0.0) kl += q * (lq - ln_p(X, z[image]));
    }
    kl = wave_sum(kl);
    mass = wave_sum(mass);
    if (lane == 0) { s_term[2][wave] = kl; s_term[3][wave] = mass; }
    __syncthreads();
    kl = wave_sum(lane < 16 ? s_term[2][lane] : 0.0);
    mass = wave_sum(lane < 16 ? s_term[3][lane] : 0.0);
    X.A = kl + mass + R.A_more;
    for (int i = tid; i < a.V_d; i += kRowThreads) {
      const float xi = Draft<T>::one(zq + i);
      const int image = R.kind & 1 ? a.dmap[i] : -1;
      Draft<T>::store_one(grad + i, R.kind & 1 ? grad_at<true>(X, i, xi, image, z[max(image, 0)]) : grad_at<false>(X, i, xi, -1, 0.f));
    }
    if (tid == 0) {
      if (R.kind & 1) publish(a.out.kl + R.row, kl + R.kl_more);
      count_in();
    }
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int base = (i * kRowThreads + tid) * kVec;
    if (wide || base >= shift + a.V_d) break;
    float out[kVec];
    if (R.kind & 1) {                                    // the thread's own words, which it wrote above, but for R.pre's
#pragma unroll
      for (int e = 0; e < kVec; e += 4) {
        const f32x4 r = *reinterpret_cast<const f32x4*>(s_z + base + e);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const float q = x[i * kVec + e + f];
          out[e + f] = q > 0.f ? c * q * (r[f] - A) : q;   // (NaN stays one)
          if (R.kind & 2) out[e + f] = fmaf(D, (base - shift + e + f == R.sub ? 1.f : 0.f) - q, out[e + f]);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float tq;
        out[e] = R.kind ? D * ((base - shift + e == R.sub ? 1.f : 0.f) - q_of(x[i * kVec + e], &tq)) : 0.f;
      }
    }
    if (i == top_vec) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) out[e] = base - shift + e == R.top ? out_top : out[e];
    }
    if (whole(i)) {
      Draft<T>::store(grad + first(i), out);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (first(i) + e >= 0 && first(i) + e < a.V_d) Draft<T>::store_one(grad + first(i) + e, out[e]);
    }
  }
  __syncthreads();
  if (s_last) grad_totals(a, tid, wave, lane, s_term);
}

template <typename T>
hipError_t launch(const LossGradArgs& a, hipStream_t stream) {
  const int groups = ceil_div((int64_t)a.V_d + 7, kGradIds<T>);   // a row starts up to 7 elements into its first vector
  const int64_t grid = (int64_t)groups * ceil_div(a.K, 8) * 8;
  if (!grid_fits(grid, 256)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(loss_grad_kernel<T>, dim3((unsigned)grid), dim3(256), 0, stream, a, groups);
  return hipGetLastError();
}

}  // namespace

// LDS for a row of 4-byte slots, and the vectors per thread that hold one.
constexpr int64_t kRowLdsBytes = 150 << 10;
constexpr int64_t row_lds_bytes(int V_d) { return 16 * (((int64_t)V_d + 16 + 3) / 4); }   // a row shifted by up to 7, in whole vectors of 8
// One workgroup per row costs its chain of steps, about 20 us for 32000 ids, and from a quarter of the compute units on less than the loss's
// launch and the gather; short rows are short chains.  Measured, us per call in one / with the gather: 6 rows of 32000 ids against 128256
// 25.9 / 19.4, 24 28.7 / 22.0, 96 30.2 / 36.8, 288 60.6 / 80.5, 600 90.3 / 160.7; of 8000 against 50257 17.7 / 19.1 (6), 35.7 / 58.3 (600); one
// vocabulary of 32000 ids on both sides 22.8 / 19.4 (6), 26.7 / 28.7 (96), 75.2 / 101.2 (600).
bool loss_grad_in_one(int K, int V_d, int n_cu) { return K > 0 && row_lds_bytes(V_d) <= kRowLdsBytes && (4 * K >= n_cu || V_d <= 16384); }
size_t loss_grad_row_bytes() { return sizeof(GradRow); }

template <typename T>
static hipError_t launch_rows(const LossGradArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(loss_prepare_kernel<T>, dim3((unsigned)ceil_div(a.B, 4)), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int kMost = (int)(kRowLdsBytes / 4 / (kRowThreads * Draft<T>::kElems)) + 1;
  const int vecs = ceil_div(a.V_d + Draft<T>::kElems - 1, kRowThreads * Draft<T>::kElems);
  const size_t lds = (size_t)row_lds_bytes(a.V_d);
  const auto kernel = vecs <= kMost / 5 ? loss_row_kernel<T, kMost / 5> : vecs <= 2 * kMost / 5 ? loss_row_kernel<T, 2 * kMost / 5>
                      : vecs <= 4 * kMost / 5 ? loss_row_kernel<T, 4 * kMost / 5> : loss_row_kernel<T, kMost>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.K), dim3(kRowThreads), lds, stream, a);
  return hipGetLastError();
}
hipError_t launch_loss_and_grad(const LossGradArgs& a, hipStream_t stream) {
  return a.dtype == OT_BF16 ? launch_rows<uint16_t>(a, stream) : launch_rows<float>(a, stream);
}

hipError_t launch_loss_grad(const LossGradArgs& a, hipStream_t stream) {
  if (a.K == 0) return hipSuccess;
  return a.dtype == OT_BF16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}

}  // namespace otv
