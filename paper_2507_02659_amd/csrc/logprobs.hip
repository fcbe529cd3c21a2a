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
// Sums of 2^t and of -2^t t, t = (z - mx) * scale, with a reference mx near the largest logit (-inf: of none).
struct Sums {
  float mx;
  double S, E;
};
__device__ inline float reference(float mx) { return mx == -INFINITY ? 0.f : mx; }
__device__ inline Sums rescaled(Sums a, float mx, float scale) {      // to another reference
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

// kPer logits per lane into the lane's running sums (-inf: none); returns the largest.  The sums' reference is one for the wavefront and
// moves, in 64 bits, only when a logit is more than 4 above it in the exponent: with a lane's own maximum for it nearly every tile moved one
// (144 rows x 128256 ids 17.2 us, 2000 x 32003 in bf16 30.5).
template <int kPer>
__device__ __forceinline__ float add_logits(const float* v, float scale, Sums* a) {
  float mx = v[0];
#pragma unroll
  for (int e = 1; e < kPer; ++e) mx = fmaxf(mx, v[e]);
  if (__any((mx - a->mx) * scale > 4.f)) *a = rescaled(*a, fmaxf(wave_max(mx), a->mx), scale);
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
  return mx;
}

// kPer values per lane, by a whole wavefront, into the sorted list whose first n count (-inf: none).  id_of(e): the id of the lane's value e,
// ascending in e; ids of different lanes and calls come in any order.  n values of the row, at least, are known not to be below `least`.
template <int kPer, typename IdFn>
__device__ __forceinline__ void select(const float* v, int n, float least, int lane, IdFn id_of, key_t* list) {
  float mx = v[0];
#pragma unroll
  for (int e = 1; e < kPer; ++e) mx = fmaxf(mx, v[e]);
  key_t last = lane_key(*list, n - 1);
  least = fmaxf(least, -3.402823466e38f);
  float bar = fmaxf(key_logit(last), least);             // below it, or at it with a higher id, nothing changes the first n
  const unsigned long long hit = __ballot(mx >= bar);
  if (hit == 0) return;
  int taken = -1;
  if (__popcll(hit) > 6) {                               // many: every lane's best at once
    int at = 0;
#pragma unroll
    for (int e = kPer - 1; e >= 0; --e) at = v[e] == mx ? e : at;
    taken = at;
    const key_t best = sort_keys(order_key(mx, id_of(at)), lane);
    *list = last == 0 && lane_key(*list, 0) == 0 ? best : merge_keys(*list, __shfl(best, 63 - lane), lane);
    last = lane_key(*list, n - 1);
    bar = fmaxf(key_logit(last), least);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) {                       // and what else is not below the bar, one by one
    unsigned long long more = __ballot(v[e] >= bar && e != taken);
    while (more) {
      const int l = (int)__builtin_ctzll(more);
      more &= more - 1;
      const key_t k = lane_key(order_key(v[e], id_of(e)), l);
      if (k > last) {
        *list = insert_key(*list, k, lane);
        last = lane_key(*list, n - 1);
      }
    }
  }
}
// The lists of a workgroup's wavefronts joined, two by two, in the first one; all of them call it.
template <int kWaves>
__device__ inline key_t join_lists(key_t list, key_t (*s_list)[64], int wave, int lane) {
#pragma unroll
  for (int step = 1; step < kWaves; step *= 2) {
    if (wave % step == 0) s_list[wave][lane] = list;
    __syncthreads();
    if (wave % (2 * step) == 0) list = merge_keys(list, s_list[wave + step][63 - lane], lane);
  }
  return list;
}

// Grid = segments x rows; a wavefront takes whole tiles of 64 * kPer logits of its segment, one after the other.  Rows start at any element:
// the tiles are laid out from the first 16-byte boundary on, and the elements in front of it and behind the last whole vector go, one a
// lane, with the first wavefront of the first segment.  The workgroup of a row that ends last joins the sums.
//
// The alternatives cost the pass nothing but the largest logit of every lane, which it has for the sums.  The n best of these maxima are n
// logits of the segment, so its n best logits are not below the n-th of them, and only the lanes that reach it can hold any: the workgroup
// selects those and reads what they have read once more, from a cache.
template <typename T, int kPer, int kWaves, bool kTop>
__global__ __launch_bounds__(64 * kWaves) void logprob_kernel(LogprobArgs a, int segments, int tiles_per_wave, Segment* part, int32_t* count) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kLoads = kPer / kVec;
  const ot_logprob_in& in = a.in;
  const int row = (int)(blockIdx.x / (unsigned)segments), seg = (int)(blockIdx.x % (unsigned)segments);
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  __shared__ Sums s_sums[kWaves];
  __shared__ key_t s_list[kTop ? kWaves : 1][64];
  __shared__ int s_last;
  const T* z = static_cast<const T*>(row_of(in, row));
  const bool skip = in.given_rows_only && !any_given(in, row);
  if (skip && seg > 0) return;                           // such a row's first workgroup writes what is left
  const int V = skip ? 0 : in.V;
  const int head = min(V, (int)((kVec - ((reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (kVec - 1))) & (kVec - 1)));
  const int vecs = (V - head) / kVec, tail = V - head - vecs * kVec, tiles = (vecs + 64 * kLoads - 1) / (64 * kLoads);
  const Raw* zv = reinterpret_cast<const Raw*>(z + head);
  const int edge_id = lane < head ? lane : V - tail + lane - head;
  const float temperature = row_temperature(in, row, lane), scale = kLog2e / temperature;
  Sums own{-INFINITY, 0.0, 0.0};
  const int tile0 = seg * kWaves * tiles_per_wave;        // of the segment: wavefront w takes tile0 + w, tile0 + kWaves + w, ...
  int tile = tile0 + wave;
  const int end = min(tile0 + kWaves * tiles_per_wave, tiles);
  Raw raw[kLoads];
  auto load = [&](int t, int l) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) raw[i] = zv[min(t * 64 * kLoads + l + i * 64, vecs - 1)];
  };
  auto unpack = [&](int t, int l, float* v) {            // -inf past the end
#pragma unroll
    for (int i = 0; i < kLoads; ++i) Vec<T>::unpack(raw[i], v + i * kVec);
    if ((t + 1) * 64 * kLoads > vecs) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[i * kVec + e] = t * 64 * kLoads + l + i * 64 < vecs ? v[i * kVec + e] : -INFINITY;
    }
  };
  auto tile_id = [&](int t, int l, int e) { return head + (t * 64 * kLoads + l + e / kVec * 64) * kVec + e % kVec; };
  if (tile < end) load(tile, lane);
  // the given tokens' logits, which the last workgroup of the row needs at its end
  int token = -1;
  float token_logit = 0.f;
  if (wave == 0 && lane < in.n_tok && V > 0) {
    token = in.tokens[(int64_t)row * in.n_tok + lane];
    if (token >= 0 && token < V) token_logit = Vec<T>::one(z + token);
  }
  const bool edges = seg == 0 && wave == 0 && head + tail > 0;
  float edge = -INFINITY, lane_max = -INFINITY;
  if (edges) {
    if (lane < head + tail) edge = Vec<T>::one(z + edge_id);
    lane_max = add_logits<1>(&edge, scale, &own);
  }
  for (; tile < end; tile += kWaves) {
    float v[kPer];
    unpack(tile, lane, v);
    if (tile + kWaves < end) load(tile + kWaves, lane);  // on its way while this one is taken
    lane_max = fmaxf(lane_max, add_logits<kPer>(v, scale, &own));
  }
  Segment* parts = part + (int64_t)row * segments;
  const bool split = segments > 1 && !skip;
  own = wave_sums(rescaled(own, wave_max(lane_max), scale), scale);   // the true maximum from here on
  if (lane == 0) s_sums[wave] = own;
  key_t list = 0;
  if constexpr (kTop) {
    // the lanes with the largest maxima, lane l of wavefront w as 64 w + l
    list = join_lists<kWaves>(sort_keys(order_key(lane_max, tid), lane), s_list, wave, lane);
    if (wave == 0) s_list[0][lane] = list;
    __syncthreads();
    const key_t holder = s_list[0][lane];
    const float bar = key_logit(lane_key(holder, in.n_top - 1));
    const key_t worst = lane_key(holder, 63);
    __syncthreads();
    list = 0;
    // more lanes than the list holds reach the bar (equal logits): all of them.  (Of 64 alternatives the last holder is the bar.)
    bool all_lanes = worst != 0 && key_logit(worst) >= bar;
    if (all_lanes) all_lanes = __syncthreads_count(lane_max >= bar) > 64;
    if (all_lanes) {
      for (int t = tile0 + wave; t < end; t += kWaves) {
        float v[kPer];
        load(t, lane);
        unpack(t, lane, v);
        select<kPer>(v, in.n_top, bar, lane, [&](int e) { return tile_id(t, lane, e); }, &list);
      }
    } else {
      const int l = key_id(holder) & 63, w = key_id(holder) >> 6;
      const bool reaches = holder != 0 && key_logit(holder) >= bar;
      for (int j = wave; j < tiles_per_wave; j += kWaves) {
        const int t = tile0 + j * kWaves + w;
        float v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = -INFINITY;
        if (reaches && t < end) {
          load(t, l);
          unpack(t, l, v);
        }
        select<kPer>(v, in.n_top, bar, lane, [&](int e) { return tile_id(t, l, e); }, &list);
      }
    }
    if (edges) select<1>(&edge, in.n_top, bar, lane, [&](int) { return edge_id; }, &list);
    list = join_lists<kWaves>(list, s_list, wave, lane);
  }
  __syncthreads();
  Sums all = lane < kWaves ? s_sums[lane] : Sums{-INFINITY, 0.0, 0.0};
  all = wave_sums(all, scale);
  if (split) {
    if (wave == 0) {
      if (kTop && lane < in.n_top) publish(reinterpret_cast<double*>(&parts[seg].top[lane]), __longlong_as_double((long long)list));
      if (lane == 0) {
        publish(&parts[seg].S, all.S);
        publish(&parts[seg].E, all.E);
        publish(reinterpret_cast<int32_t*>(&parts[seg].mx), (int32_t)__float_as_int(all.mx));
      }
      stores_done();
      if (lane == 0) s_last = arrive(count + row, segments);
    }
    __syncthreads();
    if (!s_last) return;
    all = Sums{-INFINITY, 0.0, 0.0};
    for (int s0 = 0; s0 < segments && wave == 0; s0 += 64) {
      Sums x{-INFINITY, 0.0, 0.0};
      if (s0 + lane < segments) {
        x.mx = __int_as_float(observe(reinterpret_cast<int32_t*>(&parts[s0 + lane].mx)));
        x.S = observe(&parts[s0 + lane].S);
        x.E = observe(&parts[s0 + lane].E);
      }
      x = wave_sums(x, scale);
      const float mx = fmaxf(all.mx, x.mx);
      all = rescaled(all, mx, scale);
      x = rescaled(x, mx, scale);
      all.S += x.S;
      all.E += x.E;
    }
    if constexpr (kTop) {                                // wavefront w joins the lists of segments w, w + kWaves, ...
      list = 0;
      const int mirrored = 63 - lane;
      for (int s0 = wave; s0 < segments; s0 += 4 * kWaves) {
        key_t other[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          other[j] = s0 + j * kWaves < segments && mirrored < in.n_top
                         ? (key_t)__double_as_longlong(observe(reinterpret_cast<double*>(&parts[s0 + j * kWaves].top[mirrored]))) : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (s0 + j * kWaves < segments) list = merge_keys(list, other[j], lane);
      }
      list = join_lists<kWaves>(list, s_list, wave, lane);
    }
  }
  if (wave != 0) return;
  // the row's results, by one wavefront
  const double S = all.S, lnS = log(S), mx = (double)all.mx, temp = (double)temperature;
  const float invalid = S == 0.0 ? -INFINITY : kNan;      // of a row without a distribution
  const bool valid = S > 0.0 && S < 1e300;
  if (lane == 0) {
    if (a.out.entropy) a.out.entropy[row] = valid ? (float)(lnS + all.E / S * 0.6931471805599453) : S == 0.0 ? 0.f : kNan;
    if (a.out.row_max) { a.out.row_max[row] = all.mx; a.out.row_sumexp[row] = valid || S == 0.0 ? (float)S : kNan; }
  }
  for (int i = lane; i < in.n_tok; i += 64) {
    if (i >= 64) {
      token = in.tokens[(int64_t)row * in.n_tok + i];
      if (token >= 0 && token < in.V) token_logit = Vec<T>::one(z + token);
    }
    const int t = token;
    float lp = 0.f;
    if (t < -1 || t >= in.V) lp = kNan;
    else if (t >= 0) lp = valid ? (float)(((double)token_logit - mx) / temp - lnS) : invalid;
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

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ inline void store_one(float* p, float x) { *p = x; }
__device__ inline void store_one(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }   // to nearest
__device__ inline void store_vec(float* p, const float* x) {
  typedef float raw_t __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(raw_t{x[0], x[1], x[2], x[3]}, reinterpret_cast<raw_t*>(p));
}
__device__ inline void store_vec(uint16_t* p, const float* x) {
  typedef uint32_t raw_t __attribute__((ext_vector_type(4)));
  raw_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
  __builtin_nontemporal_store(r, reinterpret_cast<raw_t*>(p));
}

// Grid = chunks x rows: four vectors of logits per thread, all asked for at once, whole where the rows of the logits and of the gradient start
// at the same place of a 16-byte unit, else one by one.  Bound by memory: a logit is read once, a gradient written once (512 x 128256
// float32 91.7 us, 5.7 TB/s; a copy of the logits takes 98).  Two vectors per thread: bf16 66 us instead of 48; eight: float32 170.
constexpr int kGradLoads = 4;
template <typename T>
constexpr int kGradChunk = 256 * kGradLoads * Vec<T>::kElems;
// kGiven: given_rows_only, whose rows without a token are not read (as a choice at run time it cost the others 4 %: 512 x 128256 float32
// with the forward pass 133 us instead of 127).
template <typename T, bool kGiven>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobGradArgs a, int chunks) {
  constexpr int kVec = Vec<T>::kElems, kLoads = kGradLoads, kEach = kLoads * kVec, kChunk = kGradChunk<T>;
  const ot_logprob_in& in = a.in;
  const int row = (int)(blockIdx.x / (unsigned)chunks), tid = threadIdx.x, lane = tid & 63;
  const T* z = static_cast<const T*>(row_of(in, row));
  T* grad = static_cast<T*>(a.grad) + (int64_t)row * a.ld_grad;
  const int shift = (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (kVec - 1);
  const bool vectors = ((int)(reinterpret_cast<uintptr_t>(grad) / sizeof(T)) & (kVec - 1)) == shift;
  // thread's vector i holds ids v0 + 256 i kVec ..; of the row's first one the ids below 0, of its last one those past the end are nobody's
  const int c0 = (int)(blockIdx.x % (unsigned)chunks) * kChunk - shift, v0 = c0 + tid * kVec;
  auto whole = [&](int i) { const int at = v0 + i * 256 * kVec; return vectors && at >= 0 && at + kVec <= in.V; };
  if (kGiven && a.row_sumexp[row] == 0.f) {  // a row that is not read (or one without a distribution)
    const float zero[kVec] = {};
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (whole(i)) {
        store_vec(grad + v0 + i * 256 * kVec, zero);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (const int at = v0 + i * 256 * kVec + e; at >= 0 && at < in.V) store_one(grad + at, 0.f);
      }
    }
    return;
  }
  typename Vec<T>::Raw raw[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
    if (whole(i)) raw[i] = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::Raw*>(z + v0 + i * 256 * kVec));
  const float T_row = row_temperature(in, row, lane), scale = kLog2e / T_row, invT = 1.f / T_row;
  const float mx = a.row_max[row], S = a.row_sumexp[row];
  const float gH = a.grad_entropy ? a.grad_entropy[row] : 0.f, H = a.grad_entropy ? a.entropy[row] : 0.f;
  const float invS = S == 0.f ? 0.f : invT / S, HS = H - logf(S);
  float v[kEach];
  auto mine = [&](int i, int e) { return v0 + i * 256 * kVec + e; };
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    if (whole(i)) {
      Vec<T>::unpack(raw[i], v + i * kVec);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[i * kVec + e] = mine(i, e) >= 0 && mine(i, e) < in.V ? Vec<T>::one(z + mine(i, e)) : -INFINITY;
    }
  }
  const int n_tok = a.grad_logprob ? in.n_tok : 0;
  double sum = 0.0;
  for (int i = lane; i < n_tok; i += 64) {
    const int t = in.tokens[(int64_t)row * in.n_tok + i];
    if (t >= 0 && t < in.V) sum += a.grad_logprob[(int64_t)row * in.n_tok + i];
  }
  const float G = (float)wave_sum(sum);
  float out[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float t = (v[i] - mx) * scale, p = __builtin_amdgcn_exp2f(t) * invS;   // over T
    out[i] = -p * fmaf(gH, fmaf(fmaxf(t, -200.f), 0.69314718f, HS), G);
  }
  if (S != 0.f) {
    for (int i0 = 0; i0 < n_tok; i0 += 64) {
      int t = -1;
      float g = 0.f;
      if (i0 + lane < n_tok) {
        t = in.tokens[(int64_t)row * in.n_tok + i0 + lane];
        g = a.grad_logprob[(int64_t)row * in.n_tok + i0 + lane];
      }
      unsigned long long here = __ballot(t >= 0 && t >= c0 && t < min(c0 + kChunk, in.V));
      while (here) {
        const int l = (int)__builtin_ctzll(here);
        here &= here - 1;
        const int at = __builtin_amdgcn_readlane(t, l);
        const float add = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), l)) * invT;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (mine(i / kVec, i % kVec) == at && v[i] > -INFINITY) out[i] += add;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) out[i] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    if (whole(i)) {
      store_vec(grad + v0 + i * 256 * kVec, out + i * kVec);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (mine(i, e) >= 0 && mine(i, e) < in.V) store_one(grad + mine(i, e), out[i * kVec + e]);
    }
  }
}

// Workgroups of four wavefronts, two per compute unit where the rows are few enough to be split; a wavefront has one tile at least.  Of the
// rows whose workgroups meet in memory there are at most kLogprobSegments segments.
// Measured, us for 144 rows x 128256 ids with 20 alternatives / 2000 x 32003 in bf16 with 5: tiles of 16 logits per lane 24.3 / 39.5, of 32
// 27.3 / 38.4; workgroups of 8 wavefronts 27.2 / 42.7, of 16 38.8 / 92; four per compute unit 26.6 / 39.4.
constexpr int kPerLane = 16, kRowWaves = 4;
template <typename T>
hipError_t launch_logprobs(const ot_ctx* ctx, const LogprobArgs& a, hipStream_t stream) {
  const int tiles = std::max(1, ceil_div(a.in.V, 64 * kPerLane)), want = ceil_div(2 * ctx->n_cu, a.in.M);
  int segments = std::max(1, std::min({want, ceil_div(tiles, kRowWaves), kLogprobSegments / a.in.M}));
  const int tiles_per_wave = ceil_div(tiles, kRowWaves * segments);
  segments = ceil_div(tiles, kRowWaves * tiles_per_wave);
  const dim3 grid((unsigned)segments * (unsigned)a.in.M);
  const auto kernel = a.in.n_top > 0 ? logprob_kernel<T, kPerLane, kRowWaves, true> : logprob_kernel<T, kPerLane, kRowWaves, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * kRowWaves), 0, stream, a, segments, tiles_per_wave, static_cast<Segment*>(ctx->lp_part), ctx->lp_count);
  return hipGetLastError();
}

int check_in(const ot_ctx* ctx, const ot_logprob_in* in, const char* who) {
  if (in->dtype != OT_BF16 && in->dtype != OT_F32) return ot_fail(OT_ERR_DTYPE, "%s: logits are OT_BF16 or OT_F32 (%d)", who, in->dtype);
  if (in->M < 0 || in->V < 1 || in->V > (1 << 30) || in->n_tok < 0 || in->ld < in->V)
    return ot_fail(OT_ERR_SHAPE, "%s: need M >= 0, 1 <= V <= 2^30, n_tok >= 0 and ld >= V (M = %d, V = %d, n_tok = %d, ld = %lld)", who, in->M, in->V, in->n_tok, (long long)in->ld);
  if (in->n_top < 0 || in->n_top > OT_MAX_TOP) return ot_fail(OT_ERR_SHAPE, "%s: n_top must be in 0..%d (%d)", who, OT_MAX_TOP, in->n_top);
  if (in->reserved != 0) return ot_fail(OT_ERR_SHAPE, "%s: reserved must be 0", who);
  if (in->given_rows_only && in->n_tok == 0) return ot_fail(OT_ERR_SHAPE, "%s: given_rows_only needs tokens", who);
  if (in->row_off && (in->B < 1 || !in->temperature)) return ot_fail(OT_ERR_SHAPE, "%s: row_off needs B >= 1 sequences and their temperatures", who);
  if (in->M > 0 && (!in->logits || (in->n_tok > 0 && !in->tokens))) return ot_fail(OT_ERR_NULL, "%s: logits and tokens must not be NULL", who);
  if (reinterpret_cast<uintptr_t>(in->logits) % (in->dtype == OT_BF16 ? 2 : 4)) return ot_fail(OT_ERR_SHAPE, "%s: logits are not aligned to their type", who);
  return ot_check_device(ctx, who);
}

// Whether rows of the gradient share memory with rows of the logits and are not those rows themselves.
bool overlaps(const ot_logprob_in& in, const void* grad, int64_t ld_grad) {
  const int64_t size = in.dtype == OT_BF16 ? 2 : 4, row = in.V * size, step = in.ld * size;
  const uintptr_t from = reinterpret_cast<uintptr_t>(in.logits), to = reinterpret_cast<uintptr_t>(grad);
  if (to == from || to >= from + (uintptr_t)((in.M - 1) * step + row) || from >= to + (uintptr_t)((in.M - 1) * ld_grad * size + row)) return false;
  if (ld_grad != in.ld) return true;
  const int64_t apart = (int64_t)(to > from ? (to - from) % (uintptr_t)step : step - (int64_t)((from - to) % (uintptr_t)step));
  return apart < row || apart > step - row;              // (a row's end, and the next row's start)
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
  if (!grid_fits(in->M, 64 * kRowWaves)) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs: %d rows are too many for a launch", in->M);
  const LogprobArgs a{*in, *out};
  const hipError_t e = in->dtype == OT_BF16 ? launch_logprobs<uint16_t>(ctx, a, ctx->stream) : launch_logprobs<float>(ctx, a, ctx->stream);
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
  if (overlaps(*in, grad, ld_grad)) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: rows of grad overlap other places of the logits' rows");
  const int chunks = ceil_div((int64_t)in->V + 7, in->dtype == OT_BF16 ? kGradChunk<uint16_t> : kGradChunk<float>);   // a row starts up to 7 elements into its first vector
  if (!grid_fits((int64_t)chunks * in->M, 256)) return ot_fail(OT_ERR_SHAPE, "ot_token_logprobs_grad: %d rows of %d ids are too many for a launch", in->M, in->V);
  const LogprobGradArgs a{*in, fwd->row_max, fwd->row_sumexp, fwd->entropy, grad_logprob, grad_entropy, grad, ld_grad};
  const auto kernel = in->dtype == OT_BF16 ? (in->given_rows_only ? logprob_grad_kernel<uint16_t, true> : logprob_grad_kernel<uint16_t, false>)
                                           : (in->given_rows_only ? logprob_grad_kernel<float, true> : logprob_grad_kernel<float, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)chunks * (unsigned)in->M), dim3(256), 0, ctx->stream, a, chunks);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_token_logprobs_grad: launch");
}

}  // extern "C"
#pragma GCC visibility pop
