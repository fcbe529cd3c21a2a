// What requests ask of their logits: penalties for repeated tokens, biases, masks, on the rows of a batch of windows.
//
//   z' = z / rho if z > 0 else z rho   (ids of the history and of the window's tokens in front of the row)
//   z' = z' - f n - [n > 0] g          (n: how often an id occurs behind the prompt and in front of the row in the window)
//   z' = z' + bias,   z' = -inf where the mask's bit is clear.
#include <math.h>

#include <algorithm>

#include "otv_host.h"
#include "rows.h"

namespace otv {
namespace {

struct AdjustArgs {
  ot_adjust_in in;
  void* out;
  int64_t ld_out;
  int32_t slices, parts;
};

constexpr uint32_t kSeen = 0x80000000u;   // of a count: the id occurs in the prompt

// Grid = (parts x slices) x sequences: a workgroup has a slice of ids of some of a sequence's rows.  It counts the slice's ids in the history
// into a table in LDS, once for all of its rows (whole numbers: the order of the additions does not matter), and marks the ids that the table
// or the bias list names in a bitmap; a row then costs one pass over its logits, of which a vector without a marked id is only copied.  The
// window's tokens join the table row by row.
template <typename T, int kSlice>
__global__ __launch_bounds__(256) void adjust_kernel(AdjustArgs a) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kThreads = 256, kLoads = kSlice / (kThreads * kVec) > 0 ? kSlice / (kThreads * kVec) : 1;
  extern __shared__ uint32_t lds[];
  uint32_t* s_mark = lds;                                // [kSlice / 32 + 1]
  uint32_t* s_count = lds + kSlice / 32 + 4;             // [kSlice]
  int32_t* s_bias = reinterpret_cast<int32_t*>(s_count + kSlice);   // [kSlice], with a bias list: its last entry of the id, from 1
  const ot_adjust_in& in = a.in;
  const int tid = threadIdx.x;
  const int part = (int)(blockIdx.x % (unsigned)a.parts), t = (int)(blockIdx.x / (unsigned)a.parts);
  const int slice = t % a.slices, b = t / a.slices;
  const int row0 = in.row_off ? max(0, in.row_off[b]) : b, row1 = in.row_off ? min(in.M, in.row_off[b + 1]) : b + 1;
  const int each = (max(0, row1 - row0) + a.parts - 1) / a.parts, first = row0 + part * each, last = min(row1, first + each);
  if (first >= last) return;
  const int s0 = slice * kSlice, n_ids = min(kSlice, in.V - s0);
  const bool has_bias = in.n_bias > 0;

  for (int i = tid; i < kSlice / 32 + 1; i += kThreads) s_mark[i] = 0;
  for (int i = tid; i < kSlice; i += kThreads) s_count[i] = 0;
  if (has_bias)
    for (int i = tid; i < kSlice; i += kThreads) s_bias[i] = 0;
  __syncthreads();
  auto mark = [&](int o) { atomicOr(&s_mark[o >> 5], 1u << (o & 31)); };
  auto mine = [&](int id) { return id >= s0 && id - s0 < n_ids; };
  if (in.history) {
    const int n = (int)min((int64_t)max(0, in.n_history ? in.n_history[b] : (int)min(in.ld_history, (int64_t)0x7FFFFFFF)), in.ld_history);
    const int n_prompt = in.n_prompt ? in.n_prompt[b] : 0;
    const int32_t* ids = in.history + (int64_t)b * in.ld_history;
    for (int64_t i = tid; i < n; i += kThreads) {
      const int id = ids[i];
      if (!mine(id)) continue;
      if (i < n_prompt) atomicOr(&s_count[id - s0], kSeen);
      else atomicAdd(&s_count[id - s0], 1u);
      mark(id - s0);
    }
  }
  if (in.window)
    for (int r = row0 + tid; r < first; r += kThreads)
      if (const int id = in.window[r]; mine(id)) { atomicAdd(&s_count[id - s0], 1u); mark(id - s0); }
  for (int i = tid; i < in.n_bias; i += kThreads)
    if (const int id = in.bias_ids[(int64_t)b * in.n_bias + i]; mine(id)) { atomicMax(&s_bias[id - s0], i + 1); mark(id - s0); }
  __syncthreads();

  const double rho = in.repetition ? (double)in.repetition[b] : 1.0, inv_rho = 1.0 / rho;
  const double f = in.frequency ? (double)in.frequency[b] : 0.0, g = in.presence ? (double)in.presence[b] : 0.0;
  auto adjusted = [&](float z, int o) {
    if (z == -INFINITY) return z;
    const uint32_t c = s_count[o], n = c & ~kSeen;
    double x = (double)z;
    if (c) {
      x = x > 0.0 ? x * inv_rho : x * rho;
      if (n) x = x - f * (double)n - g;
    }
    if (has_bias)
      if (const int i = s_bias[o]) x += (double)in.bias[(int64_t)b * in.n_bias + i - 1];
    return (float)x;
  };

  for (int row = first; row < last; ++row) {
    const T* z = static_cast<const T*>(in.logits) + (int64_t)row * in.ld + s0;
    T* out = static_cast<T*>(a.out) + (int64_t)row * a.ld_out + s0;
    const bool in_place = z == out;
    const RowSplit<T> split(z, n_ids);
    const bool vectors = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int m = in.mask_of_row ? in.mask_of_row[row] : in.masks ? row : -1;
    const bool no_such = m < -1 || m >= in.n_masks;
    const uint32_t* mask = m >= 0 && !no_such ? in.masks + (int64_t)m * in.ld_mask : nullptr;
    // bits of `count` ids from the o-th of the slice on
    auto marks_at = [&](int o) { return (uint32_t)((((uint64_t)s_mark[(o >> 5) + 1] << 32) | s_mark[o >> 5]) >> (o & 31)); };
    auto allowed_at = [&](int o, int count) {
      if (!mask) return 0xFFFFFFFFu;
      const int v = s0 + o;
      return (uint32_t)((((uint64_t)mask[(v + count - 1) >> 5] << 32) | mask[v >> 5]) >> (v & 31));
    };
    auto one = [&](int o) {
      const float x = Vec<T>::one(z + o);
      if (no_such) store_one(out + o, kNan);
      else if (!(allowed_at(o, 1) & 1)) store_one(out + o, -INFINITY);
      else if (marks_at(o) & 1) store_one(out + o, adjusted(x, o));
      else if (!in_place) out[o] = z[o];
    };
    constexpr uint32_t kAll = (1u << kVec) - 1;
    const Raw* zv = reinterpret_cast<const Raw*>(z + split.head);
    if (vectors) {
      Raw raw[kLoads];
      uint32_t marked[kLoads], allowed[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int k = i * kThreads + tid, o = split.head + k * kVec;
        marked[i] = 0;
        allowed[i] = kAll;
        raw[i] = Raw{};
        if (k < split.vecs) {
          if (!in_place) raw[i] = __builtin_nontemporal_load(zv + k);
          marked[i] = marks_at(o) & kAll;
          allowed[i] = allowed_at(o, kVec) & kAll;
          if (in_place && allowed[i] != 0 && ((marked[i] | ~allowed[i]) & kAll) != 0) raw[i] = zv[k];
        }
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int k = i * kThreads + tid, o = split.head + k * kVec;
        if (k >= split.vecs) continue;
        Raw* to = reinterpret_cast<Raw*>(out + o);
        if (!no_such && marked[i] == 0 && allowed[i] == kAll) {
          if (!in_place) __builtin_nontemporal_store(raw[i], to);
          continue;
        }
        float v[kVec];
        if (no_such) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] = kNan;
        } else {
          Vec<T>::unpack(raw[i], v);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (marked[i] >> e & 1) v[e] = adjusted(v[e], o + e);
            if (!(allowed[i] >> e & 1)) v[e] = -INFINITY;
          }
        }
        store_vec(reinterpret_cast<T*>(to), v);
      }
      if (tid < split.head + split.tail) one(split.edge(tid));
    } else {
      for (int o = tid; o < n_ids; o += kThreads) one(o);
    }
    if (in.window && row + 1 < last)
      if (const int id = in.window[row]; mine(id)) {     // the same in every thread
        __syncthreads();
        if (tid == 0) { s_count[id - s0] += 1; s_mark[(id - s0) >> 5] |= 1u << ((id - s0) & 31); }
        __syncthreads();
      }
  }
}

template <typename T, int kSlice>
hipError_t launch(const AdjustArgs& a, dim3 grid, hipStream_t stream) {
  const size_t lds = sizeof(uint32_t) * (kSlice / 32 + 4 + (size_t)kSlice * (a.in.n_bias > 0 ? 2 : 1));
  hipLaunchKernelGGL((adjust_kernel<T, kSlice>), grid, dim3(256), lds, stream, a);
  return hipGetLastError();
}

constexpr int kSliceIds = 4096;

}  // namespace
}  // namespace otv

using namespace otv;

#pragma GCC visibility push(default)
extern "C" {

int ot_adjust_logits(ot_ctx* ctx, const ot_adjust_in* in, void* out, int64_t ld_out) {
  if (!ctx || !in) return ot_fail(OT_ERR_NULL, "ot_adjust_logits: ctx and in must not be NULL");
  if (in->dtype != OT_BF16 && in->dtype != OT_F32) return ot_fail(OT_ERR_DTYPE, "ot_adjust_logits: logits are OT_BF16 or OT_F32 (%d)", in->dtype);
  const int64_t size = in->dtype == OT_BF16 ? 2 : 4;
  if (in->M < 0 || in->V < 1 || in->V > (1 << 30) || in->ld < in->V || ld_out < in->V)
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: need M >= 0, 1 <= V <= 2^30, ld and ld_out >= V (M = %d, V = %d, ld = %lld, ld_out = %lld)", in->M, in->V,
                   (long long)in->ld, (long long)ld_out);
  if (in->reserved[0] != 0 || in->reserved[1] != 0) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: reserved must be 0");
  if (in->row_off ? in->B < 0 : in->B != in->M)
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: need B >= 0 sequences of row_off, or without it B = M (B = %d, M = %d)", in->B, in->M);
  if (in->n_bias < 0 || in->n_masks < 0 || in->ld_history < 0 || (in->masks && in->ld_mask < ceil_div(in->V, 32)))
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: need n_bias, n_masks and ld_history >= 0, ld_mask >= ceil(V / 32)");
  if (in->window && !in->row_off) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: a window needs row_off");
  if (in->masks && !in->mask_of_row && in->n_masks < in->M)
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: without mask_of_row every row has its own mask (n_masks = %d, M = %d)", in->n_masks, in->M);
  if (in->M == 0 || in->B == 0) return OT_OK;
  if (!in->logits || !out || (in->n_bias > 0 && (!in->bias_ids || !in->bias)) || (in->n_masks > 0 && !in->masks) || (in->ld_history > 0 && !in->history))
    return ot_fail(OT_ERR_NULL, "ot_adjust_logits: logits, out, bias_ids and bias, masks and history must not be NULL where they have entries");
  if (reinterpret_cast<uintptr_t>(in->logits) % size || reinterpret_cast<uintptr_t>(out) % size)
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: logits and out must be aligned to their type");
  if (out == in->logits && ld_out != in->ld) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: in place, ld_out must be ld");
  if (ot_rows_overlap(in->logits, in->ld, out, ld_out, in->M, in->V, size))
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: rows of out overlap other places of the logits' rows");
  AdjustArgs a{*in, out, ld_out, ceil_div(in->V, kSliceIds), 1};
  const int64_t groups = (int64_t)a.slices * in->B;
  // a sequence's rows in parts until there are a few workgroups per compute unit
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(in->M, in->B), 4 * ctx->n_cu / groups));
  if (!grid_fits(groups * a.parts, 256)) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: %d sequences of %d ids are too many for a launch", in->B, in->V);
  if (const int bad = ot_check_device(ctx, "ot_adjust_logits")) return bad;
  const dim3 grid((unsigned)(groups * a.parts));
  const hipError_t e = in->dtype == OT_BF16 ? launch<uint16_t, kSliceIds>(a, grid, ctx->stream) : launch<float, kSliceIds>(a, grid, ctx->stream);
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_adjust_logits: launch");
}

}  // extern "C"
#pragma GCC visibility pop
