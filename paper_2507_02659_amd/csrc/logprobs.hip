// Log-probabilities of given tokens with entropy and the most likely alternatives, and their gradient with respect to the logits.
//
// With mx the row's largest logit, e_v = exp((z_v - mx)/T), S = sum e and E = sum e (mx - z)/T:
//   ln p_v = (z_v - mx)/T - ln S,   entropy = ln S + E / S,
//   dz_v = (1/T) [ sum over tokens of v of g - p_v (G + gH (ln p_v + entropy)) ],   G = sum of the row's g.
#include <math.h>

#include <algorithm>

#include "device_math.h"
#include "otv_host.h"

namespace otv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNan = __builtin_nanf("");

struct LogprobArgs {
  ot_logprob_in in;
  ot_logprob_out out;
};

__device__ inline float logit(const void* row, int dtype, int64_t v) {
  return dtype == OT_BF16 ? bf16_to_f32(static_cast<const uint16_t*>(row)[v]) : static_cast<const float*>(row)[v];
}
__device__ inline const void* row_of(const ot_logprob_in& in, int64_t row) {
  return static_cast<const char*>(in.logits) + row * in.ld * (in.dtype == OT_BF16 ? 2 : 4);
}
// Temperature of a row, of which log2(e) / T is finite; by a whole wavefront.
__device__ inline float row_temperature(const ot_logprob_in& in, int row, int lane) {
  if (!in.temperature) return 1.f;
  const float T = in.temperature[in.row_off ? find_sequence(in.row_off, in.B, row, 0, lane) : row];
  return T > 0.f ? fmaxf(T, 0x1p-126f) : 1.f;
}
__device__ inline bool any_given(const ot_logprob_in& in, int64_t row) {
  for (int i = 0; i < in.n_tok; ++i)
    if (in.tokens[row * in.n_tok + i] != -1) return true;
  return false;
}

// ------------------------------------------------------------------------------------------------ alternatives
// Order of alternatives as one number: by descending logit (-0 and 0 alike), of equal ones the lowest id first; 0 is none.
typedef unsigned long long key_t;
__device__ inline key_t order_key(float z, int v) {
  const uint32_t u = __float_as_uint(z + 0.f), up = u & 0x80000000u ? ~u : u | 0x80000000u;
  return z > -INFINITY ? (key_t)up << 32 | (0xFFFFFFFFu - (uint32_t)v) : 0ull;
}
__device__ inline int key_id(key_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }
__device__ inline float key_logit(key_t k) {
  const uint32_t up = (uint32_t)(k >> 32);
  return k ? __uint_as_float(up & 0x80000000u ? up ^ 0x80000000u : ~up) : -INFINITY;
}
__device__ inline key_t lane_key(key_t k, int l) {
  return (key_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, l);
}
// The partner's key, lanes apart by exclusive or with kMask: data-parallel moves within a row of 16 lanes, else through the LDS network.
template <int kCtrl>
__device__ inline key_t dpp_key(key_t k) {
  const int hi = (int)(k >> 32), lo = (int)k;
  return (key_t)(uint32_t)__builtin_amdgcn_update_dpp(hi, hi, kCtrl, 0xF, 0xF, false) << 32 |
         (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, kCtrl, 0xF, 0xF, false);
}
template <int kMask>
__device__ inline key_t partner(key_t k) {
  if constexpr (kMask == 1) return dpp_key<0xB1>(k);
  else if constexpr (kMask == 2) return dpp_key<0x4E>(k);
  else if constexpr (kMask == 3) return dpp_key<0x1B>(k);
  else if constexpr (kMask == 4) return dpp_key<0x1B>(dpp_key<0x141>(k));
  else if constexpr (kMask == 7) return dpp_key<0x141>(k);
  else if constexpr (kMask == 8) return dpp_key<0x128>(k);
  else if constexpr (kMask == 15) return dpp_key<0x140>(k);
  else return __shfl_xor(k, kMask);
}
// The larger of the two partners' keys into the lower lane.
template <int kMask>
__device__ inline key_t exchange(key_t k, int lane) {
  const key_t other = partner<kMask>(k);
  constexpr int kHighest = kMask >= 32 ? 32 : kMask >= 16 ? 16 : kMask >= 8 ? 8 : kMask >= 4 ? 4 : kMask >= 2 ? 2 : 1;
  return (other > k) != ((lane & kHighest) != 0) ? other : k;
}
// Sorts 64 keys over the lanes, the largest into lane 0: merges of 2, 4, ... lanes whose first step meets the mirrored lane, so that every
// step has the same direction.
__device__ inline key_t sort_keys(key_t k, int lane) {
  k = exchange<1>(k, lane);
  k = exchange<3>(k, lane); k = exchange<1>(k, lane);
  k = exchange<7>(k, lane); k = exchange<2>(k, lane); k = exchange<1>(k, lane);
  k = exchange<15>(k, lane); k = exchange<4>(k, lane); k = exchange<2>(k, lane); k = exchange<1>(k, lane);
  k = exchange<31>(k, lane); k = exchange<8>(k, lane); k = exchange<4>(k, lane); k = exchange<2>(k, lane); k = exchange<1>(k, lane);
  k = exchange<63>(k, lane); k = exchange<16>(k, lane); k = exchange<8>(k, lane); k = exchange<4>(k, lane); k = exchange<2>(k, lane);
  return exchange<1>(k, lane);
}
// The 64 largest of a sorted list and of one whose lane i holds the (63 - i)-th.
__device__ inline key_t merge_keys(key_t k, key_t mirrored, int lane) {
  k = mirrored > k ? mirrored : k;
  k = exchange<32>(k, lane); k = exchange<16>(k, lane); k = exchange<8>(k, lane); k = exchange<4>(k, lane); k = exchange<2>(k, lane);
  return exchange<1>(k, lane);
}
// Puts a key (the same in every lane) into a sorted list.
__device__ inline key_t insert_key(key_t list, key_t k, int lane) {
  const int at = __popcll(__ballot(list > k));
  const key_t below = __shfl_up(list, 1);
  return lane < at ? list : lane == at ? k : below;
}

// ------------------------------------------------------------------------------------------------ a row's sums
// Per lane: maximum, sum of 2^t and of 2^t |t|, t = (z - mx) * scale.
struct Sums {
  float mx;
  double S, E;
};
__device__ inline float reference(float mx) { return mx == -INFINITY ? 0.f : mx; }
__device__ inline Sums rescaled(Sums a, float mx, float scale) {      // to a maximum that is no smaller
  const double d = fmax((double)((reference(a.mx) - reference(mx)) * scale), -2000.0);
  if (a.mx == -INFINITY || a.mx == mx) { a.mx = mx; return a; }
  const double f = exp_neg_fast(d * 0.6931471805599453);
  a.E = f * (a.E - d * a.S);
  a.S = f * a.S;
  a.mx = mx;
  return a;
}
__device__ inline Sums wave_sums(Sums a, float scale) {
  a = rescaled(a, wave_max(a.mx), scale);
  a.S = wave_sum(a.S);
  a.E = wave_sum(a.E);
  return a;
}

// What the workgroups of a row hand to the last of them.
struct Segment {
  double S, E;
  float mx, pad;
  key_t top[OT_MAX_TOP];
};

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int kElems = 4;
  typedef float Raw __attribute__((ext_vector_type(4)));
  __device__ static void unpack(const Raw& x, float* v) { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
  __device__ static float one(const float* p) { return *p; }
};
template <> struct Vec<uint16_t> {
  static constexpr int kElems = 8;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  __device__ static void unpack(const Raw& x, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(x[i] << 16);
      v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
  }
  __device__ static float one(const uint16_t* p) { return bf16_to_f32(*p); }
};

// Sum of n values, the deepest of them log2 n additions deep.
template <int n>
__device__ inline float tree_sum(const float* x) {
  if constexpr (n == 1) return x[0];
  else return tree_sum<n / 2>(x) + tree_sum<n - n / 2>(x + n / 2);
}

// kPer logits per lane into the running sums and the sorted list of the best.  id0 + id_of(e): the id of the lane's element e, ascending in e.
// masked: elements may be -inf because they are past the row's end.
template <int kPer, bool kTop, typename IdFn>
__device__ __forceinline__ void take(const float* v, float scale, int n_top, int lane, int lowest_id, IdFn id_of, Sums* a, key_t* list) {
  float mx = v[0];
#pragma unroll
  for (int e = 1; e < kPer; ++e) mx = fmaxf(mx, v[e]);
  if (__any(mx > a->mx)) *a = rescaled(*a, fmaxf(mx, a->mx), scale);
  const float ref = reference(a->mx);
  constexpr int kBatch = kPer < 16 ? kPer : 16;
#pragma unroll
  for (int e0 = 0; e0 < kPer; e0 += kBatch) {
    float ex[kBatch], en[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const float t = (v[e0 + e] - ref) * scale;
      ex[e] = __builtin_amdgcn_exp2f(t);
      en[e & 3] = fmaf(ex[e], fmaxf(t, -200.f), en[e & 3]);
    }
    a->S += (double)tree_sum<kBatch>(ex);
    a->E -= (double)((en[0] + en[1]) + (en[2] + en[3]));
  }
  if constexpr (kTop) {
    key_t last = lane_key(*list, n_top - 1);
    float bar = key_logit(last);
    // Ids in front of the last of the list win where the logits are equal.
    const bool earlier = last != 0 && lowest_id < key_id(last);
    const unsigned long long hit = __ballot(earlier ? mx >= bar : mx > bar);
    if (hit == 0) return;
    int taken = -1;
    if (__popcll(hit) > 6) {                             // many: every lane's best at once
      int at = 0;
#pragma unroll
      for (int e = kPer - 1; e >= 0; --e) at = v[e] == mx ? e : at;
      taken = at;
      *list = merge_keys(*list, __shfl(sort_keys(order_key(mx, id_of(at)), lane), 63 - lane), lane);
      last = lane_key(*list, n_top - 1);
      bar = key_logit(last);
    }
    const float least = earlier || taken >= 0 ? bar : nextafterf(bar, INFINITY);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {                     // and what else is above the bar, one by one
      unsigned long long more = __ballot(v[e] >= least && v[e] > -INFINITY && e != taken);
      while (more) {
        const int l = (int)__builtin_ctzll(more);
        more &= more - 1;
        const key_t k = lane_key(order_key(v[e], id_of(e)), l);
        if (k > last) {
          *list = insert_key(*list, k, lane);
          last = lane_key(*list, n_top - 1);
        }
      }
    }
  }
}

// Grid = segments x rows; a wavefront takes whole tiles of 64 * kPer logits of its segment, one after the other.  Rows start at any element:
// the tiles are laid out from the first 16-byte boundary on, and the elements in front of it and behind the last whole vector go, one a
// lane, with the first wavefront of the first segment.
template <typename T, int kPer, bool kTop>
__global__ __launch_bounds__(256) void logprob_kernel(LogprobArgs a, int segments, int tiles_per_wave, Segment* part, int32_t* count) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kLoads = kPer / kVec;
  const ot_logprob_in& in = a.in;
  const int row = (int)(blockIdx.x / (unsigned)segments), seg = (int)(blockIdx.x % (unsigned)segments);
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  __shared__ Sums s_sums[4];
  __shared__ key_t s_list[3][64];
  const T* z = static_cast<const T*>(row_of(in, row));
  const bool skip = in.given_rows_only && !any_given(in, row);
  if (skip && seg > 0) return;                           // such a row's first workgroup writes what is left
  const int V = skip ? 0 : in.V;
  const int head = min(V, (int)((kVec - ((reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (kVec - 1))) & (kVec - 1)));
  const int vecs = (V - head) / kVec, tail = V - head - vecs * kVec;
  const Raw* zv = reinterpret_cast<const Raw*>(z + head);
  Sums own{-INFINITY, 0.0, 0.0};
  key_t list = 0;
  const float scale = kLog2e / row_temperature(in, row, lane);
  int tile = (seg * 4 + wave) * tiles_per_wave;
  const int end = min(tile + tiles_per_wave, (vecs + 64 * kLoads - 1) / (64 * kLoads));
  if (seg == 0 && wave == 0 && head + tail > 0) {
    const int id = lane < head ? lane : V - tail + lane - head;
    const float v = lane < head + tail ? Vec<T>::one(z + id) : -INFINITY;
    take<1, kTop>(&v, scale, in.n_top, lane, 0, [&](int) { return id; }, &own, &list);
  }
  for (; tile < end; ++tile) {
    const int first = tile * 64 * kLoads + lane;
    Raw raw[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) raw[i] = __builtin_nontemporal_load(zv + min(first + i * 64, vecs - 1));
    float v[kPer];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) Vec<T>::unpack(raw[i], v + i * kVec);
    if ((tile + 1) * 64 * kLoads > vecs) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[i * kVec + e] = first + i * 64 < vecs ? v[i * kVec + e] : -INFINITY;
    }
    take<kPer, kTop>(v, scale, in.n_top, lane, head + tile * 64 * kLoads * kVec,
                     [&](int e) { return head + (first + e / kVec * 64) * kVec + e % kVec; }, &own, &list);
  }
  own = wave_sums(own, scale);
  if (lane == 0) s_sums[wave] = own;
  if (kTop && wave > 0) s_list[wave - 1][63 - lane] = list;
  __syncthreads();
  if (wave != 0) return;
  Sums all = lane < 4 ? s_sums[lane] : Sums{-INFINITY, 0.0, 0.0};
  all = wave_sums(all, scale);
  if constexpr (kTop) {
#pragma unroll
    for (int w = 0; w < 3; ++w) list = merge_keys(list, s_list[w][lane], lane);
  }
  if (segments > 1 && !skip) {
    Segment* mine = part + (int64_t)row * segments + seg;
    if (lane == 0) {
      publish(&mine->S, all.S);
      publish(&mine->E, all.E);
      publish(reinterpret_cast<int32_t*>(&mine->mx), (int32_t)__float_as_int(all.mx));
    }
    if (kTop && lane < in.n_top) publish(reinterpret_cast<double*>(&mine->top[lane]), __longlong_as_double((long long)list));
    stores_done();
    int last = 0;
    if (lane == 0) last = arrive(count + row, segments);
    if (!uniform(last)) return;
    Segment* others = part + (int64_t)row * segments;
    all = Sums{-INFINITY, 0.0, 0.0};
    for (int s0 = 0; s0 < segments; s0 += 64) {
      Sums x{-INFINITY, 0.0, 0.0};
      if (s0 + lane < segments) {
        x.mx = __int_as_float(observe(reinterpret_cast<int32_t*>(&others[s0 + lane].mx)));
        x.S = observe(&others[s0 + lane].S);
        x.E = observe(&others[s0 + lane].E);
      }
      x = wave_sums(x, scale);
      const float mx = fmaxf(all.mx, x.mx);
      all = rescaled(all, mx, scale);
      x = rescaled(x, mx, scale);
      all.S += x.S;
      all.E += x.E;
    }
    if constexpr (kTop) {
      list = 0;
      const int mirrored = 63 - lane;
      for (int s = 0; s < segments; ++s) {
        key_t other = 0;
        if (mirrored < in.n_top) other = (key_t)__double_as_longlong(observe(reinterpret_cast<double*>(&others[s].top[mirrored])));
        list = merge_keys(list, other, lane);
      }
    }
  }
  // the row's results, by one wavefront
  const double S = all.S, lnS = log(S), mx = (double)all.mx, temp = (double)row_temperature(in, row, lane);
  const float invalid = S == 0.0 ? -INFINITY : kNan;      // of a row without a distribution
  const bool valid = S > 0.0 && S < 1e300;
  if (lane == 0) {
    if (a.out.entropy) a.out.entropy[row] = valid ? (float)(lnS + all.E / S * 0.6931471805599453) : S == 0.0 ? 0.f : kNan;
    if (a.out.row_max) { a.out.row_max[row] = all.mx; a.out.row_sumexp[row] = valid || S == 0.0 ? (float)S : kNan; }
  }
  for (int i = lane; i < in.n_tok; i += 64) {
    const int t = in.tokens[(int64_t)row * in.n_tok + i];
    float lp = 0.f;
    if (t < -1 || t >= in.V) lp = kNan;
    else if (t >= 0) lp = valid ? (float)(((double)Vec<T>::one(z + t) - mx) / temp - lnS) : invalid;
    a.out.logprob[(int64_t)row * in.n_tok + i] = lp;
  }
  if (kTop && lane < in.n_top) {
    const bool some = valid && list != 0;
    a.out.top_ids[(int64_t)row * in.n_top + lane] = some ? key_id(list) : -1;
    a.out.top_logprobs[(int64_t)row * in.n_top + lane] = some ? (float)(((double)key_logit(list) - mx) / temp - lnS) : -INFINITY;
  }
}

struct LogprobGradArgs {
  ot_logprob_in in;
  const float *row_max, *row_sumexp, *entropy, *grad_logprob, *grad_entropy;
  void* grad;
  int64_t ld_grad;
};

__device__ inline uint16_t f32_to_bf16(float x) {         // to nearest, ties to even; NaN stays one
  const uint32_t u = __float_as_uint(x);
  return x != x ? 0x7FC0 : (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}

// Grid = chunks x rows.
constexpr int kGradChunk = 2048;
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobGradArgs a, int chunks) {
  const ot_logprob_in& in = a.in;
  const int row = blockIdx.x / chunks, v0 = (int)(blockIdx.x % chunks) * kGradChunk, tid = threadIdx.x, lane = tid & 63;
  const void* z = row_of(in, row);
  const float T = row_temperature(in, row, lane), scale = kLog2e / T, invT = 1.f / T;
  const float mx = a.row_max[row], S = a.row_sumexp[row];
  const float lnS = logf(S), invS = 1.f / S, gH = a.grad_entropy ? a.grad_entropy[row] : 0.f, H = a.grad_entropy ? a.entropy[row] : 0.f;
  float G = 0.f;
  for (int i = 0; a.grad_logprob && i < in.n_tok; ++i) {
    const int t = in.tokens[(int64_t)row * in.n_tok + i];
    if (t >= 0 && t < in.V) G += a.grad_logprob[(int64_t)row * in.n_tok + i];
  }
  for (int v = v0 + tid; v < min(v0 + kGradChunk, in.V); v += 256) {
    float out = 0.f;
    if (S != 0.f) {
      const float x = logit(z, in.dtype, v), t = (x - mx) * scale, p = __builtin_amdgcn_exp2f(t) * invS;
      const float lp = fmaxf(t, -200.f) * 0.69314718f - lnS;
      out = -p * (G + gH * (lp + H));
      for (int i = 0; a.grad_logprob && i < in.n_tok; ++i)
        if (in.tokens[(int64_t)row * in.n_tok + i] == v && x > -INFINITY) out += a.grad_logprob[(int64_t)row * in.n_tok + i];
      out *= invT;
    }
    const int64_t at = (int64_t)row * a.ld_grad + v;
    if (in.dtype == OT_BF16) static_cast<uint16_t*>(a.grad)[at] = f32_to_bf16(out);
    else static_cast<float*>(a.grad)[at] = out;
  }
}

// Segments of a row: as many workgroups as the chip holds at a time, each wavefront of them with one tile at least; of the rows whose
// workgroups meet in memory there are at most kLogprobSegments segments.
template <typename T, int kPer>
hipError_t launch_logprobs(const ot_ctx* ctx, const LogprobArgs& a, hipStream_t stream) {
  const int tiles = std::max(1, ceil_div(a.in.V, 64 * kPer)), want = ceil_div(4 * ctx->n_cu, a.in.M);
  int segments = std::max(1, std::min({want, ceil_div(tiles, 4), kLogprobSegments / a.in.M}));
  const int tiles_per_wave = ceil_div(tiles, 4 * segments);
  segments = ceil_div(tiles, 4 * tiles_per_wave);
  const dim3 grid((unsigned)segments * (unsigned)a.in.M);
  if (a.in.n_top > 0)
    hipLaunchKernelGGL((logprob_kernel<T, kPer, true>), grid, dim3(256), 0, stream, a, segments, tiles_per_wave, static_cast<Segment*>(ctx->lp_part), ctx->lp_count);
  else
    hipLaunchKernelGGL((logprob_kernel<T, kPer, false>), grid, dim3(256), 0, stream, a, segments, tiles_per_wave, static_cast<Segment*>(ctx->lp_part), ctx->lp_count);
  return hipGetLastError();
}

int check_in(const ot_ctx* ctx, const ot_logprob_in* in, const char* who) {
  if (in->dtype != OT_BF16 && in->dtype != OT_F32) return ot_fail(OT_ERR_DTYPE, "%s: logits are OT_BF16 or OT_F32 (%d)", who, in->dtype);
  if (in->M < 0 || in->V < 1 || in->n_tok < 0 || in->ld < in->V)
    return ot_fail(OT_ERR_SHAPE, "%s: need M >= 0, V >= 1, n_tok >= 0 and ld >= V (M = %d, V = %d, n_tok = %d, ld = %lld)", who, in->M, in->V, in->n_tok, (long long)in->ld);
  if (in->n_top < 0 || in->n_top > OT_MAX_TOP) return ot_fail(OT_ERR_SHAPE, "%s: n_top must be in 0..%d (%d)", who, OT_MAX_TOP, in->n_top);
  if (in->reserved != 0) return ot_fail(OT_ERR_SHAPE, "%s: reserved must be 0", who);
  if (in->given_rows_only && in->n_tok == 0) return ot_fail(OT_ERR_SHAPE, "%s: given_rows_only needs tokens", who);
  if (in->row_off && (in->B < 1 || !in->temperature)) return ot_fail(OT_ERR_SHAPE, "%s: row_off needs B >= 1 sequences and their temperatures", who);
  if (in->M > 0 && (!in->logits || (in->n_tok > 0 && !in->tokens))) return ot_fail(OT_ERR_NULL, "%s: logits and tokens must not be NULL", who);
  if (reinterpret_cast<uintptr_t>(in->logits) % (in->dtype == OT_BF16 ? 2 : 4)) return ot_fail(OT_ERR_SHAPE, "%s: logits are not aligned to their type", who);
  return ot_check_device(ctx, who);
}

}  // namespace

size_t logprob_segment_bytes() { return sizeof(Segment); }

}  // namespace otv

using namespace otv;

#pragma GCC visibility push(default)
extern "C" {

int ot_token_logprobs(ot_ctx* ctx, const ot_logprob_in* in, ot_logprob_out* out) {
  if (!ctx || !in || !out) return ot_fail(OT_ERR_NULL, "ot_token_logprobs: ctx, in and out must not be NULL");
  if (const int bad = check_in(ctx, in, "ot_token_logprobs")) return bad;
  if (in->M == 0) return OT_OK;
  if ((in->n_tok > 0 && !out->logprob) || (in->n_top > 0 && (!out->top_ids || !out->top_logprobs)))
    return ot_fail(OT_ERR_NULL, "ot_token_logprobs: logprob, top_ids and top_logprobs are required where they have entries");
  if (!out->row_max != !out->row_sumexp) return ot_fail(OT_ERR_NULL, "ot_token_logprobs: row_max and row_sumexp come together");
  const LogprobArgs a{*in, *out};
  const bool few = (int64_t)in->M * in->V < (int64_t)ctx->n_cu * 8192;
  hipError_t e;
  if (in->dtype == OT_BF16) e = few ? launch_logprobs<uint16_t, 16>(ctx, a, ctx->stream) : launch_logprobs<uint16_t, 64>(ctx, a, ctx->stream);
  else e = few ? launch_logprobs<float, 16>(ctx, a, ctx->stream) : launch_logprobs<float, 64>(ctx, a, ctx->stream);
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_token_logprobs: launch");
}

int ot_token_logprobs_grad(ot_ctx* ctx, const ot_logprob_in* in, const ot_logprob_out* fwd, const float* grad_logprob, const float* grad_entropy,
                           void* grad, int64_t ld_grad) {
  if (!ctx || !in || !fwd) return ot_fail(OT_ERR_NULL, "ot_token_logprobs_grad: ctx, in and forward must not be NULL");
  if (const int bad = check_in(ctx, in, "ot_token_logprobs_grad")) return bad;
  if (ld_grad < in->V) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: ld_grad = %lld is below V = %d", (long long)ld_grad, in->V);
  if (in->M == 0) return OT_OK;
  if (!grad || !fwd->row_max || !fwd->row_sumexp || (grad_entropy && !fwd->entropy))
    return ot_fail(OT_ERR_NULL, "ot_token_logprobs_grad: grad, row_max, row_sumexp and (with grad_entropy) entropy must not be NULL");
  if (reinterpret_cast<uintptr_t>(grad) % (in->dtype == OT_BF16 ? 2 : 4))
    return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: grad is not aligned to its type");
  if (grad == in->logits && ld_grad != in->ld) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: in place, ld_grad must be ld");
  const int chunks = ceil_div(in->V, kGradChunk);
  if ((int64_t)chunks * in->M > 0x7FFFFFFF) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: %d rows of %d ids are too many for a launch", in->M, in->V);
  const LogprobGradArgs a{*in, fwd->row_max, fwd->row_sumexp, fwd->entropy, grad_logprob, grad_entropy, grad, ld_grad};
  hipLaunchKernelGGL(logprob_grad_kernel, dim3((unsigned)(chunks * in->M)), dim3(256), 0, ctx->stream, a, chunks);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_token_logprobs_grad: launch");
}

}  // extern "C"
#pragma GCC visibility pop
