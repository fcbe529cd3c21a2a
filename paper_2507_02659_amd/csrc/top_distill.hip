// Distillation from a teacher's top logits: the loss of a row of a student's logits against the teacher's most likely ids, and its gradient.
//
// With p_i the teacher's probabilities of the ids K that are kept, P their sum (1 where they are renormalised), q = softmax(z / T):
//   loss = sum p_i (ln p_i - ln q_i)                dz_v = (P q_v - p_v) / T
//   bucket: + (1 - P) ln((1 - P) / (1 - Q))         dz_v = (q_v - p_v) / T in K, q_v (1 - (1 - P) / (1 - Q)) / T elsewhere; P >= 1: as without.
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

// Grid = rows.  A workgroup holds the vectors of its row that fit its registers (kHeld per thread; kWhole: all of them) from the sums to the
// gradient and reads what is beyond them again.  The kept ids, one a thread of the first four wavefronts, are taken in 64 bits; where they lie
// among the others a bitmap in LDS says, by which the held vectors have -inf in their places.  The others' sum is one of float32 exponentials of
// their distance to their largest, added in 64 bits.
// 512 rows of 128256 float32 logits with 50 ids, gradient included, 114 to 116 us (525 MB, 4.6 TB/s; a copy of the logits takes 99): bound by memory,
// and by the 60 % of a row that is read again, from a cache.  16 vectors held 119 to 133 us, 8 123, in workgroups of 512 threads that hold 32 149 (one
// workgroup, 8 wavefronts, per compute unit).  2000 rows of 128256 in bfloat16, gradient included, 242 us (1.03 GB, 4.2 TB/s).  2000 rows of 32003 in bfloat16 with 256 ids, the loss alone, 42 us (3.1 TB/s): bound by its
// instructions, 19 per logit, a third of them for the entries and the sums' ends; 256 threads that hold 16 vectors 43.
// 128 rows of 32000 in bfloat16 13 us: one chain of loads, four barriers and 64-bit exponentials.
constexpr int kFar = 4;           // vectors of a row that a thread asks for together where it does not hold them
constexpr int kEntryWaves = OT_MAX_TEACHER_TOP / 64;
// 1 - P that rounding can leave of log-probabilities that add up to 1: each is off by 2^-24 of itself, so P by 2^-24 of their entropy, at most
// ln 256, and what formed them had sums of its own to round.
constexpr double kNoRemainder = 0x1p-20;
constexpr float kImprobable = -600.f;
struct RowCoef {
  double q, p;              // a kept id's gradient: q exp((z - top) / T) - p (its probability with the teacher)
  float rest;               // of exp((z - mx) / T), mx the others' largest logit, in the others' gradients
  int32_t nothing;          // the row adds nothing
};
template <typename T, int kThreads, int kHeld, bool kGrad, bool kWhole>
__global__ __launch_bounds__(kThreads, kGrad || !kWhole ? 4 : 8) void top_distill_kernel(TopDistillArgs a) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kWaves = kThreads / 64;
  constexpr uint32_t kAll = (1u << kVec) - 1;
  extern __shared__ uint32_t s_keep[];                   // [V / 32 + 2]
  __shared__ volatile int s_id[OT_MAX_TEACHER_TOP];
  __shared__ volatile double s_p[OT_MAX_TEACHER_TOP];
  __shared__ double s_sum[kWaves], s_P[kEntryWaves], s_E[kEntryWaves], s_L[kEntryWaves];
  __shared__ float s_max[kWaves], s_top[kEntryWaves];
  __shared__ int s_twice;
  __shared__ RowCoef s_coef;
  const ot_top_distill_in& in = a.in;
  const int row = (int)blockIdx.x, tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, V = in.V;
  const T* z = static_cast<const T*>(in.logits) + (int64_t)row * in.ld;
  T* grad = kGrad ? static_cast<T*>(a.grad) + (int64_t)row * a.ld_grad : nullptr;
  const RowSplit<T> split(z, V);
  const Raw* zv = reinterpret_cast<const Raw*>(z + split.head);

  // the teacher's entries; the row's vectors behind them on their way
  const bool entries = wave < kEntryWaves && wave * 64 < in.n_top;   // (the same for a wavefront)
  int id = -1;
  float lp = -INFINITY;
  if (tid < in.n_top) {
    id = in.top_ids[(int64_t)row * in.n_top + tid];
    lp = in.top_logprobs[(int64_t)row * in.n_top + tid];
  }
  Raw raw[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int at = k * kThreads + tid;
    raw[k] = Raw{};
    if (at < split.vecs) raw[k] = __builtin_nontemporal_load(zv + at);
  }
  const bool has_edge = tid < split.head + split.tail;
  const int edge_id = has_edge ? split.edge(tid) : 0;
  float edge = has_edge ? Vec<T>::one(z + edge_id) : -INFINITY;
  const float temperature = row_temperature(in.temperature, in.row_off, in.B, row, lane), scale = kLog2e / temperature;
  const double temp = (double)temperature;
  for (int i = tid; i < V / 32 + 2; i += kThreads) s_keep[i] = 0;
  if (tid == 0) s_twice = 0;
  const bool inside = id >= -1 && id < (in.through_map ? a.V_t : V);
  if (in.through_map && inside && id >= 0) id = a.tmap[id];
  if (!inside || id >= V) id = -1;
  const bool wrong = !inside || (id >= 0 && (isnan(lp) || lp == INFINITY));
  float zk = -INFINITY;
  if (id >= 0) zk = Vec<T>::one(z + id);
  const bool broken = __syncthreads_or(wrong);           // (the bitmap is clear from here on)
  // Renormalised probabilities may all be below what 64 bits hold (a low temperature's, behind ids without a draft id): theirs are then taken
  // relative to the largest, whose logarithm is subtracted from all (exactly, from any within a factor of two of it; the others are below
  // exp(-600) of it).  What the row keeps is 0 in float32.
  const bool renormalise = in.rest == OT_REST_RENORMALISE;
  const bool some = __syncthreads_or(id >= 0 && (!renormalise || lp > kImprobable)) || broken;
  const bool improbable = renormalise && !some && __syncthreads_or(id >= 0);
  if (improbable) {
    if (tid < in.n_top) s_p[tid] = id >= 0 ? (double)lp : -INFINITY;
    __syncthreads();
    float largest = -INFINITY;
    for (int i = 0; i < in.n_top; ++i) largest = fmaxf(largest, (float)s_p[i]);
    __syncthreads();
    if (largest > -INFINITY) lp -= largest;
  } else if (!some) {                                    // no ids: the row's logits do not matter
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
  double p = 0.0;
  if (entries) {
    if (id >= 0) {
      const uint32_t bit = 1u << (id & 31);
      if (atomicOr(&s_keep[id >> 5], bit) & bit) s_twice = 1;
      p = exp((double)lp);
    }
    s_id[tid] = id;
    s_p[tid] = p;
    const double P = wave_sum(p);
    const float top = wave_max(zk);
    if (lane == 0) { s_P[wave] = P; s_top[wave] = top; }
  } else if (wave < kEntryWaves && lane == 0) {
    s_P[wave] = s_E[wave] = s_L[wave] = 0.0;
    s_top[wave] = -INFINITY;
  }
  __syncthreads();

  auto keep_at = [&](int v) { return __builtin_amdgcn_alignbit(s_keep[(v >> 5) + 1], s_keep[v >> 5], v & 31) & kAll; };
  const bool edge_kept = has_edge && (keep_at(edge_id) & 1);
  if (edge_kept) edge = -INFINITY;
  // of a vector from id v0 on: its values, -inf in the places of kept ids
  auto others = [&](Raw x, int v0, float* v) {
    if (const uint32_t keep = keep_at(v0)) mask_vector(&x, ~keep);
    Vec<T>::unpack(x, v);
  };
  float mx = edge;                                       // their largest
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    __builtin_amdgcn_sched_barrier(0);
    const int at = k * kThreads + tid;
    if (at >= split.vecs) continue;
    if (const uint32_t keep = keep_at(split.head + at * kVec)) mask_vector(&raw[k], ~keep);
    float v[kVec];
    Vec<T>::unpack(raw[k], v);
#pragma unroll
    for (int e = 0; e < kVec; ++e) mx = fmaxf(mx, v[e]);
  }
  // what is not held, in one pass: a sum of its own per lane, whose reference starts at the wavefront's largest that is held, and moves up with
  // the lane's largest (rarely: from -inf on, in every second vector of some lane, it cost 512 rows of 128256 ids 7 us)
  float far_ref = kWhole ? -INFINITY : wave_max(mx);
  double far_sum = 0.0;
  auto far_vectors = [&](auto take) {                    // each in turn, a few on their way together
    for (int at0 = kHeld * kThreads + tid; at0 < split.vecs; at0 += kFar * kThreads) {
      Raw x[kFar];
#pragma unroll
      for (int i = 0; i < kFar; ++i) x[i] = zv[min(at0 + i * kThreads, split.vecs - 1)];
#pragma unroll
      for (int i = 0; i < kFar; ++i) {
        const int at = at0 + i * kThreads;
        if (at >= split.vecs) continue;
        float v[kVec];
        others(x[i], split.head + at * kVec, v);
        take(v, split.head + at * kVec);
      }
    }
  };
  if constexpr (!kWhole)
    far_vectors([&](float* v, int) {
      float top_v = -INFINITY;
#pragma unroll
      for (int e = 0; e < kVec; ++e) top_v = fmaxf(top_v, v[e]);
      if (top_v > far_ref) {
        far_sum *= far_ref == -INFINITY ? 0.0 : exp(((double)far_ref - (double)top_v) / temp);
        far_ref = top_v;
      }
      const float r = far_ref == -INFINITY ? 0.f : far_ref;
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - r) * scale);
      far_sum += (double)tree_sum<kVec>(v);
    });
  if (!kWhole) mx = fmaxf(mx, far_ref);
  mx = wave_max(mx);
  if (lane == 0) s_max[wave] = mx;
  __syncthreads();
  mx = wave_max(lane < kWaves ? s_max[lane] : -INFINITY);
  const float top = fmaxf(mx, wave_max(lane < kEntryWaves ? s_top[lane] : -INFINITY));
  const float ref = mx == -INFINITY ? 0.f : mx;
  const double ref_top = top == -INFINITY ? 0.0 : (double)top;
  // and the sum of their exponentials
  double sum = (double)__builtin_amdgcn_exp2f((edge - ref) * scale);
  auto add = [&](float* v) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - ref) * scale);
    sum += (double)tree_sum<kVec>(v);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    __builtin_amdgcn_sched_barrier(0);                   // (one vector at a time: together they take twice the registers)
    if (k * kThreads + tid >= split.vecs) continue;
    float v[kVec];
    Vec<T>::unpack(raw[k], v);
    add(v);
  }
  if (!kWhole && far_ref != -INFINITY) sum += far_sum * (far_ref == mx ? 1.0 : exp(((double)far_ref - (double)mx) / temp));
  else if (!kWhole) sum += far_sum;                                   // (0, or NaN)
  sum = wave_sum(sum);
  if (lane == 0) s_sum[wave] = sum;
  // entries of the same id: the first of them has the id's part in Q and its gradient
  bool first = id >= 0;
  double p_id = p, e = 0.0;
  if (entries) {
    if (s_twice) {
      for (int i = 0; i < in.n_top; ++i) {
        if (id < 0 || s_id[i] != id) continue;
        if (i < tid) first = false;
        if (i > tid) p_id += s_p[i];
      }
    }
    const double x = ((double)zk - ref_top) / temp;
    if (id >= 0) e = exp(x);
    const double E = wave_sum(first ? e : 0.0), L = wave_sum(p != 0.0 ? p * ((double)lp - x) : 0.0);
    if (lane == 0) { s_E[wave] = E; s_L[wave] = L; }
  }
  __syncthreads();

  const double P = (s_P[0] + s_P[1]) + (s_P[2] + s_P[3]);
  const double norm = in.rest == OT_REST_RENORMALISE ? P : 1.0;
  if (wave == 0) {
    const double S_rest = wave_sum(lane < kWaves ? s_sum[lane] : 0.0);
    const double shift = ((double)mx - ref_top) / temp;  // (-inf: there are no others)
    const double down = mx == -INFINITY && !isnan(S_rest) ? 0.0 : exp(shift);
    const double S_others = S_rest * down, S = ((s_E[0] + s_E[1]) + (s_E[2] + s_E[3])) + S_others;
    // Where the others have no probability at all, what the sum of rounded probabilities lacks of 1 has no place to go, and is none.
    double left = in.rest == OT_REST_BUCKET && P < 1.0 ? 1.0 - P : 0.0;
    if (S_others == 0.0 && left <= kNoRemainder) left = 0.0;
    const bool nothing = S == 0.0 && top == -INFINITY && !broken;       // masked whole
    const double lnS = log(S);
    double loss = norm > 0.0 ? ((s_L[0] + s_L[1]) + (s_L[2] + s_L[3]) + P * (lnS - log(norm))) / norm : 0.0;
    if (left > 0.0) loss += left * (log(left) - (S_rest == 0.0 ? -INFINITY : log(S_rest) + shift - lnS));
    if (nothing) loss = 0.0;
    if (lane == 0) {
      a.loss[row] = broken || isnan(S) ? kNan : (float)loss;   // (S: also where no p is above 0)
      if (a.kept) a.kept[row] = broken ? kNan : improbable ? 0.f : (float)P;
      if (kGrad) {
        const double scaled = (a.grad_loss ? (double)a.grad_loss[row] : 1.0) / temp;
        // in front of q_v: what the terms of the loss add up to, in OT_REST_BUCKET more than 1 where P is
        const double mass = in.rest == OT_REST_RENORMALISE ? (P > 0.0 ? 1.0 : 0.0) : left > 0.0 ? 1.0 : P;
        double factor = down == 0.0 ? 0.0 : scaled * mass * down / S;
        if (left > 0.0 && S_rest > 0.0) factor -= scaled * left / S_rest;
        s_coef.rest = nothing ? 0.f : broken || isnan(S) ? kNan : (float)factor;
        s_coef.nothing = nothing;
        s_coef.q = scaled * mass / S;
        s_coef.p = norm > 0.0 ? scaled / norm : 0.0;
      }
    }
  }
  if (!kGrad) return;
  __syncthreads();
  const float c = s_coef.rest;
  if (first) {
    double g = s_coef.q * e - s_coef.p * p_id;
    if (s_coef.nothing || (zk == -INFINITY && !isnan(s_coef.q))) g = 0.0;
    store_one(grad + id, broken ? kNan : (float)g);
  }
  const float none = isnan(c) ? c : 0.f;                 // where the exponential is 0, also beside an infinite factor
  const bool vectors = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0;
  auto gradient = [&](float x) {
    const float y = __builtin_amdgcn_exp2f((x - ref) * scale);
    return y == 0.f ? none : c * y;
  };
  auto put = [&](float* v, int v0) {
    const uint32_t keep = keep_at(v0);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = gradient(v[e]);
    if (vectors && keep == 0) {
      store_vec(grad + v0, v);
    } else {                                             // the kept ids' are the entries' business
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (!(keep >> e & 1)) store_one(grad + v0 + e, v[e]);
    }
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    __builtin_amdgcn_sched_barrier(0);
    const int at = k * kThreads + tid;
    if (at >= split.vecs) continue;
    float v[kVec];
    Vec<T>::unpack(raw[k], v);
    put(v, split.head + at * kVec);
  }
  if constexpr (!kWhole) far_vectors(put);
  if (has_edge && !edge_kept) store_one(grad + edge_id, gradient(edge));
}

template <typename T, bool kGrad>
hipError_t launch(const TopDistillArgs& a, int n_cu, hipStream_t stream) {
  constexpr int kVec = Vec<T>::kElems;
  const size_t lds = sizeof(uint32_t) * ((size_t)a.in.V / 32 + 2);
  auto go = [&](auto kernel, int threads) {
    if (lds > (56 << 10)) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.in.M), dim3(threads), lds, stream, a);
    return hipGetLastError();
  };
  // The smallest workgroup that holds the row.  Beyond 512 threads that is for a row per compute unit (256 rows of 32000 in float32 16.4 us, by
  // 512 threads 18.8).  More rows: two workgroups of 512 per compute unit wait at barriers in turn, and a row's second reading is a cache's
  // (2000 of 33706 in bfloat16 74 us, held by 1024 threads 110; of 32000 in float32 99 and 123).  Longer rows too (2000 of 128256 in bfloat16
  // 242 us, by 1024 threads 336), but for float32 that the caches no longer keep (128256: 479 and 433; 72971: 269 and 267), and where the bitmap leaves
  // a compute unit one workgroup (512 of 1000000 in bfloat16 639 and 583).  The loss alone takes the same, so that it has the same bits.
  if (a.in.V <= 256 * 4 * kVec) return go(top_distill_kernel<T, 256, 4, kGrad, true>, 256);
  if (a.in.V <= 512 * 8 * kVec) return go(top_distill_kernel<T, 512, 8, kGrad, true>, 512);
  if (a.in.V <= 1024 * 8 * kVec && a.in.M <= n_cu) return go(top_distill_kernel<T, 1024, 8, kGrad, true>, 1024);
  // Few rows have no second workgroup to wait beside, and take 1024 threads that hold more of the row: in float32 up to a row for two compute units
  // (1, 64, 128 rows of 72971 17.7, 21.0, 23.9 us, by 512 threads 22.1, 25.4, 29.1; of 33003 12.7, 14.2, 14.9 and 13.4, 15.0, 16.7, but their
  // loss alone 9.7, 11.0, 11.3 and 9.8, 10.0, 10.5; for 256 rows 36.8 and 37.3, their loss alone 20.2 and 18.2); in bfloat16 up to a row each
  // where it is long (300000 ids: 51, 59, 90 us for 1, 64, 256 rows and 57, 67, 93; but 152064: 30, 35, 51 and 33, 36, 44).
  const bool few = sizeof(T) == 4 ? a.in.M <= n_cu / 2 : a.in.M <= n_cu && a.in.V > 192 << 10;
  if (!few && a.in.V <= (sizeof(T) == 4 ? 80 << 10 : 512 << 10)) return go(top_distill_kernel<T, 512, 8, kGrad, false>, 512);
  return go(top_distill_kernel<T, 1024, 12, kGrad, false>, 1024);
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
  const hipError_t e = in->dtype == OT_BF16 ? (with_grad ? launch<uint16_t, true>(a, ctx->n_cu, ctx->stream) : launch<uint16_t, false>(a, ctx->n_cu, ctx->stream))
                                            : (with_grad ? launch<float, true>(a, ctx->n_cu, ctx->stream) : launch<float, false>(a, ctx->n_cu, ctx->stream));
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
