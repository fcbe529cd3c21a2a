// Distillation from a teacher's top logits: the loss of a row of a student's logits against the teacher's most likely ids, and its gradient.
//
// With p_i the teacher's probabilities of the ids K that are kept, P their sum (1 where they are renormalised), q = softmax(z / T):
//   loss = sum p_i (ln p_i - ln q_i)                dz_v = (P q_v - p_v) / T
//   bucket: + (1 - P) ln((1 - P) / (1 - Q))         dz_v = (q_v - p_v) / T in K, q_v (1 - (1 - P) / (1 - Q)) / T elsewhere.
// The sums over the kept ids and over the others are held apart, each with its own largest logit: 1 - Q and q_v - p_v then keep their
// digits where the student is sure.
#include <math.h>

#include <algorithm>

#include "otv_host.h"
#include "rows.h"

namespace otv {
namespace {

struct TopDistillArgs {
  ot_top_distill_in in;
  const int32_t* tmap;      // target id -> draft id or -1, with through_map
  int32_t V_t;
  float *loss, *kept;
  const float* grad_loss;
  void* grad;
  int64_t ld_grad;
};

// What the first wavefront hands to the others.
struct RowCoef {
  float rest;               // of exp((z - mx) / T), mx the others' largest logit, in a gradient outside K
  int32_t zero;             // the row adds nothing
};

// Grid = rows.  A workgroup holds the vectors of its row that fit its registers (kHeld per thread) from the sums to the gradient and reads what is
// beyond them twice.  The kept ids, of which the first wavefront has up to four per lane, are taken in 64 bits; the others through a bitmap in
// LDS that tells them apart, in float32 exponentials of their distance to their largest.
template <typename T, int kThreads, int kHeld, bool kGrad>
__global__ __launch_bounds__(kThreads) void top_distill_kernel(TopDistillArgs a) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kWaves = kThreads / 64, kEach = OT_MAX_TEACHER_TOP / 64;
  constexpr uint32_t kAll = (1u << kVec) - 1;
  extern __shared__ uint32_t s_keep[];                   // [V / 32 + 2]
  __shared__ int s_id[OT_MAX_TEACHER_TOP];
  __shared__ double s_p[OT_MAX_TEACHER_TOP], s_sum[kWaves];
  __shared__ float s_max[kWaves];
  __shared__ int s_state;
  __shared__ RowCoef s_coef;
  const ot_top_distill_in& in = a.in;
  const int row = (int)blockIdx.x, tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, V = in.V;
  const T* z = static_cast<const T*>(in.logits) + (int64_t)row * in.ld;
  T* grad = kGrad ? static_cast<T*>(a.grad) + (int64_t)row * a.ld_grad : nullptr;
  const RowSplit<T> split(z, V);
  const Raw* zv = reinterpret_cast<const Raw*>(z + split.head);
  const float temperature = row_temperature(in.temperature, in.row_off, in.B, row, lane), scale = kLog2e / temperature;

  // the teacher's entries, entry lane + 64 j of the first wavefront's lanes
  for (int i = tid; i < V / 32 + 2; i += kThreads) s_keep[i] = 0;
  int id[kEach];
  float lp[kEach], zk[kEach];
  bool broken = false;
  if (wave == 0) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int i = lane + 64 * j;
      id[j] = -1;
      lp[j] = -INFINITY;
      if (i < in.n_top) {
        int v = in.top_ids[(int64_t)row * in.n_top + i];
        lp[j] = in.top_logprobs[(int64_t)row * in.n_top + i];
        const bool inside = v >= -1 && v < (in.through_map ? a.V_t : V);
        broken |= !inside;
        if (in.through_map && inside && v >= 0) v = a.tmap[v];
        id[j] = inside && v >= 0 && v < V ? v : -1;
        if (id[j] >= 0) broken |= isnan(lp[j]) || lp[j] == INFINITY;
      }
      any |= id[j] >= 0;
    }
    broken = __any(broken);
    const int state = (__any(any) || broken) ? 1 : 0;
    if (lane == 0) s_state = state;
  }
  __syncthreads();
  if (s_state == 0) {                                    // no ids: nothing is read
    if (tid == 0) {
      a.loss[row] = 0.f;
      if (a.kept) a.kept[row] = 0.f;
    }
    if (kGrad) {
      const RowSplit<T> to(grad, V);
      const float zero[kVec] = {};
      for (int k = tid; k < to.vecs; k += kThreads) store_vec(grad + to.head + k * kVec, zero);
      if (tid < to.head + to.tail) store_one(grad + to.edge(tid), 0.f);
    }
    return;
  }
  Raw raw[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int at = k * kThreads + tid;
    raw[k] = Raw{};
    if (at < split.vecs) raw[k] = kGrad ? zv[at] : __builtin_nontemporal_load(zv + at);
  }
  const bool has_edge = tid < split.head + split.tail;
  const int edge_id = has_edge ? split.edge(tid) : 0;
  const float edge = has_edge ? Vec<T>::one(z + edge_id) : -INFINITY;
  bool twice = false;
  if (wave == 0) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      zk[j] = -INFINITY;
      if (id[j] < 0) continue;
      zk[j] = Vec<T>::one(z + id[j]);
      const uint32_t bit = 1u << (id[j] & 31);
      twice |= (atomicOr(&s_keep[id[j] >> 5], bit) & bit) != 0;
    }
  }
  __syncthreads();

  auto keep_at = [&](int v) { return (uint32_t)((((uint64_t)s_keep[(v >> 5) + 1] << 32) | s_keep[v >> 5]) >> (v & 31)) & kAll; };
  const bool edge_kept = has_edge && (keep_at(edge_id) & 1);
  // the others' largest logit
  float mx = has_edge && !edge_kept ? edge : -INFINITY;
  auto vector_max = [&](const Raw& x, int v0) {
    float v[kVec];
    Vec<T>::unpack(x, v);
    const uint32_t keep = keep_at(v0);
#pragma unroll
    for (int e = 0; e < kVec; ++e) mx = fmaxf(mx, keep >> e & 1 ? -INFINITY : v[e]);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (const int at = k * kThreads + tid; at < split.vecs) vector_max(raw[k], split.head + at * kVec);
  for (int at = kHeld * kThreads + tid; at < split.vecs; at += kThreads) vector_max(zv[at], split.head + at * kVec);
  mx = wave_max(mx);
  if (lane == 0) s_max[wave] = mx;
  __syncthreads();
  mx = wave_max(lane < kWaves ? s_max[lane] : -INFINITY);
  const float ref = mx == -INFINITY ? 0.f : mx;
  // and the sum of their exponentials
  double sum = 0.0;
  auto vector_sum = [&](const Raw& x, int v0) {
    float v[kVec];
    Vec<T>::unpack(x, v);
    const uint32_t keep = keep_at(v0);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = keep >> e & 1 ? 0.f : __builtin_amdgcn_exp2f((v[e] - ref) * scale);
    sum += (double)tree_sum<kVec>(v);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (const int at = k * kThreads + tid; at < split.vecs) vector_sum(raw[k], split.head + at * kVec);
  for (int at = kHeld * kThreads + tid; at < split.vecs; at += kThreads) vector_sum(zv[at], split.head + at * kVec);
  if (has_edge && !edge_kept) sum += (double)__builtin_amdgcn_exp2f((edge - ref) * scale);
  sum = wave_sum(sum);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();

  if (wave == 0) {
    const double S_rest = wave_sum(lane < kWaves ? s_sum[lane] : 0.0), temp = (double)temperature;
    // entries of the same id: the first of them has the id's part in Q and its gradient
    bool first[kEach];
    double p[kEach], p_id[kEach];
    double P = 0.0;
    float top = mx;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      first[j] = id[j] >= 0;
      p_id[j] = p[j] = id[j] >= 0 ? exp((double)lp[j]) : 0.0;
      P += p[j];
      top = fmaxf(top, zk[j]);
    }
    P = wave_sum(P);
    top = wave_max(top);
    if (__any(twice)) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        *(volatile int*)&s_id[lane + 64 * j] = id[j];
        *(volatile double*)&s_p[lane + 64 * j] = p[j];
      }
      __builtin_amdgcn_wave_barrier();
      for (int i = 0; i < in.n_top; ++i) {
        const int other = *(volatile int*)&s_id[i];
        const double more = *(volatile double*)&s_p[i];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          if (id[j] < 0 || other != id[j]) continue;
          if (i < lane + 64 * j) first[j] = false;
          if (i > lane + 64 * j) p_id[j] += more;
        }
      }
    }
    const double ref_top = top == -INFINITY ? 0.0 : (double)top;
    const double rest = mx == -INFINITY && !isnan(S_rest) ? 0.0 : S_rest * exp(((double)mx - ref_top) / temp);   // of exp((z - top) / T)
    double e[kEach], S = 0.0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      e[j] = id[j] >= 0 ? exp(((double)zk[j] - ref_top) / temp) : 0.0;
      if (first[j]) S += e[j];
    }
    S = wave_sum(S) + rest;
    const double lnS = log(S), norm = in.rest == OT_REST_RENORMALISE ? P : 1.0, ln_norm = log(norm);
    double loss = 0.0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (id[j] >= 0 && p[j] != 0.0 && norm > 0.0) loss += p[j] / norm * ((double)lp[j] - ln_norm - (((double)zk[j] - ref_top) / temp - lnS));
    loss = wave_sum(loss);
    const double left = in.rest == OT_REST_BUCKET && P < 1.0 ? 1.0 - P : 0.0;
    if (left > 0.0) loss += left * (log(left) - (S_rest == 0.0 ? -INFINITY : log(S_rest) + ((double)mx - ref_top) / temp - lnS));
    const bool nothing = S == 0.0 && top == -INFINITY && !broken;       // masked whole
    if (broken) loss = (double)kNan;
    if (lane == 0) {
      a.loss[row] = nothing ? 0.f : (float)loss;
      if (a.kept) a.kept[row] = broken ? kNan : (float)P;
    }
    if (kGrad) {
      const double each = (a.grad_loss ? (double)a.grad_loss[row] : 1.0) / temp;
      const double mass = in.rest == OT_REST_BUCKET ? 1.0 : in.rest == OT_REST_RENORMALISE ? (P > 0.0 ? 1.0 : 0.0) : P;   // in front of q_v
      if (lane == 0) {
        double c = mx == -INFINITY && !isnan(S) ? 0.0 : each * mass * exp(((double)mx - ref_top) / temp) / S;
        if (left > 0.0 && S_rest > 0.0) c -= each * left / S_rest;
        s_coef.rest = broken ? kNan : (float)c;
        s_coef.zero = nothing;
      }
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        if (!first[j]) continue;
        double g = each * (mass * e[j] / S - (norm > 0.0 ? p_id[j] / norm : 0.0));
        if (nothing || (zk[j] == -INFINITY && !isnan(S))) g = 0.0;
        if (broken) g = (double)kNan;
        store_one(grad + id[j], (float)g);
      }
    }
  }
  if (!kGrad) return;
  __syncthreads();
  const float c = s_coef.zero ? 0.f : s_coef.rest;
  const bool zero = s_coef.zero;
  const bool vectors = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0;
  const float none = isnan(c) ? c : 0.f;                 // where the exponential is 0, also beside an infinite factor
  auto gradient = [&](float x) {
    const float e = __builtin_amdgcn_exp2f((x - ref) * scale);
    return zero ? 0.f : e == 0.f ? none : c * e;
  };
  auto vector_grad = [&](const Raw& x, int v0) {
    float v[kVec];
    Vec<T>::unpack(x, v);
    const uint32_t keep = keep_at(v0);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = gradient(v[e]);
    if (vectors && keep == 0) {
      store_vec(grad + v0, v);
    } else {                                             // the kept ids' are there already
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (!(keep >> e & 1)) store_one(grad + v0 + e, v[e]);
    }
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (const int at = k * kThreads + tid; at < split.vecs) vector_grad(raw[k], split.head + at * kVec);
  for (int at = kHeld * kThreads + tid; at < split.vecs; at += kThreads) vector_grad(zv[at], split.head + at * kVec);
  if (has_edge && !edge_kept) store_one(grad + edge_id, gradient(edge));
}

template <typename T, bool kGrad>
hipError_t launch(const TopDistillArgs& a, hipStream_t stream) {
  constexpr int kVec = Vec<T>::kElems;
  const size_t lds = sizeof(uint32_t) * ((size_t)a.in.V / 32 + 2);
  auto go = [&](auto kernel, int threads) {
    if (lds > (60 << 10)) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.in.M), dim3(threads), lds, stream, a);
    return hipGetLastError();
  };
  if (a.in.V <= 256 * 4 * kVec) return go(top_distill_kernel<T, 256, 4, kGrad>, 256);
  if (a.in.V <= 1024 * 8 * kVec) return go(top_distill_kernel<T, 1024, 8, kGrad>, 1024);
  return go(top_distill_kernel<T, 1024, 16, kGrad>, 1024);
}

int run(const char* who, const ot_ctx* ctx, const ot_top_distill_in* in, float* loss, float* kept, const float* grad_loss, void* grad, int64_t ld_grad, bool with_grad) {
  if (!ctx || !in) return ot_fail(OT_ERR_NULL, "%s: ctx and in must not be NULL", who);
  if (in->dtype != OT_BF16 && in->dtype != OT_F32) return ot_fail(OT_ERR_DTYPE, "%s: logits are OT_BF16 or OT_F32 (%d)", who, in->dtype);
  const int64_t size = in->dtype == OT_BF16 ? 2 : 4;
  if (in->M < 0 || in->V < 1 || in->V > OT_MAX_STUDENT_V || in->ld < in->V)
    return ot_fail(OT_ERR_SHAPE, "%s: need M >= 0, 1 <= V <= %d and ld >= V (M = %d, V = %d, ld = %lld)", who, OT_MAX_STUDENT_V, in->M, in->V, (long long)in->ld);
  if (in->n_top < 1 || in->n_top > OT_MAX_TEACHER_TOP) return ot_fail(OT_ERR_SHAPE, "%s: n_top must be in 1..%d (%d)", who, OT_MAX_TEACHER_TOP, in->n_top);
  if (in->rest < OT_REST_DROP || in->rest > OT_REST_BUCKET) return ot_fail(OT_ERR_SHAPE, "%s: rest must be one of OT_REST_* (%d)", who, in->rest);
  if (in->reserved != 0) return ot_fail(OT_ERR_SHAPE, "%s: reserved must be 0", who);
  if (in->through_map && in->V != ctx->V_d) return ot_fail(OT_ERR_SHAPE, "%s: through the map the logits are the drafter's, V = V_d = %d (%d)", who, ctx->V_d, in->V);
  if (in->row_off && (in->B < 1 || !in->temperature)) return ot_fail(OT_ERR_SHAPE, "%s: row_off needs B >= 1 sequences and their temperatures", who);
  if (with_grad && ld_grad < in->V) return ot_fail(OT_ERR_SHAPE, "%s: ld_grad = %lld is below V = %d", who, (long long)ld_grad, in->V);
  if (in->M == 0) return OT_OK;
  if (!in->logits || !in->top_ids || !in->top_logprobs || !loss || (with_grad && !grad))
    return ot_fail(OT_ERR_NULL, "%s: logits, top_ids, top_logprobs, loss and grad must not be NULL", who);
  if (reinterpret_cast<uintptr_t>(in->logits) % size || (with_grad && reinterpret_cast<uintptr_t>(grad) % size))
    return ot_fail(OT_ERR_SHAPE, "%s: logits and grad must be aligned to their type", who);
  if (with_grad && grad == in->logits && ld_grad != in->ld) return ot_fail(OT_ERR_SHAPE, "%s: in place, ld_grad must be ld", who);
  if (with_grad && ot_rows_overlap(in->logits, in->ld, grad, ld_grad, in->M, in->V, size))
    return ot_fail(OT_ERR_SHAPE, "%s: rows of grad overlap other places of the logits' rows", who);
  if (!grid_fits(in->M, 1024)) return ot_fail(OT_ERR_SHAPE, "%s: %d rows are too many for a launch", who, in->M);
  if (const int bad = ot_check_device(ctx, who)) return bad;
  const TopDistillArgs a{*in, ctx->tmap, ctx->V_t, loss, kept, grad_loss, grad, ld_grad};
  const hipError_t e = in->dtype == OT_BF16 ? (with_grad ? launch<uint16_t, true>(a, ctx->stream) : launch<uint16_t, false>(a, ctx->stream))
                                            : (with_grad ? launch<float, true>(a, ctx->stream) : launch<float, false>(a, ctx->stream));
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, who);
}

}  // namespace
}  // namespace otv

using namespace otv;

#pragma GCC visibility push(default)
extern "C" {

int ot_top_distill_loss(ot_ctx* ctx, const ot_top_distill_in* in, float* loss, float* kept) {
  return run("ot_top_distill_loss", ctx, in, loss, kept, nullptr, nullptr, 0, false);
}

int ot_top_distill_loss_grad(ot_ctx* ctx, const ot_top_distill_in* in, float* loss, float* kept, const float* grad_loss, void* grad, int64_t ld_grad) {
  return run("ot_top_distill_loss_grad", ctx, in, loss, kept, grad_loss, grad, ld_grad, true);
}

}  // extern "C"
#pragma GCC visibility pop
