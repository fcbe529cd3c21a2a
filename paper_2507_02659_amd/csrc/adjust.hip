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
  int32_t bias_slots;       // of the table of biases: a power of two, at least twice n_bias, or 0
};

// An id's word in a slice's table: how often it was said, and two flags.  A history of 2^29 ids and a window of 2^29 rows, of which the last has
// 2^29 - 1 tokens in front, stay below the flags.
constexpr uint32_t kSeen = 0x80000000u;     // it occurs in the prompt
constexpr uint32_t kBiased = 0x40000000u;   // the bias list names it
constexpr uint32_t kNoKey = 0xFFFFFFFFu;

typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// 32 bits of a bitmap from bit `at` on, of which its words at / 32 and the one behind are at hand.
__device__ inline uint32_t bits_at(uint32_t lo, uint32_t hi, int at) { return __builtin_amdgcn_alignbit(hi, lo, at & 31); }

// Grid = (parts x slices) x sequences: a workgroup has a slice of 16 ids per thread of some of a sequence's rows.  It counts the slice's ids in
// the history into a table in LDS, once for all of its rows (whole numbers: the order of the additions does not matter), puts the slice's biases
// into a small hash table and marks the ids of both in a bitmap; a row then costs one pass over its logits, of which a vector without a marked or
// masked id is only copied (in place: not even read).  The window's tokens join the table row by row.  The first row's logits are on their
// way while the table is built.
// Values are formed in 64 bits and rounded to float32 and the logits' type: only marked ids are, a few thousand of a row.
// Bound by memory where histories are short: 144 rows of 128256 float32 logits behind histories of 2000 ids 29 us (149 MB, 5.1 TB/s: a copy's rate).
// 64 rows of 152064 behind 24576 ids each 33 us (2.6 TB/s), without a history 18: every slice's workgroup reads the whole history, and 640
// workgroups of which 512 are there at once take a second round (131072 ids, 512 workgroups: 25 us).  With up to 64 registers eight wavefronts
// are on a SIMD (144 rows: 43 us with 98 registers and rows asked for ahead); slices of 16 ids per thread, since a smaller one reads the history more
// often and a larger table leaves room for one workgroup per compute unit.
template <typename T, int kThreads, bool kInPlace>
__global__ __launch_bounds__(kThreads, 8) void adjust_kernel(AdjustArgs a) {
  typedef typename Vec<T>::Raw Raw;
  constexpr int kVec = Vec<T>::kElems, kLoads = 16 / kVec, kSlice = kThreads * 16;
  constexpr uint32_t kAll = (1u << kVec) - 1;
  extern __shared__ uint32_t lds[];
  uint32_t* s_mark = lds;                                // [kSlice / 32 + 1]
  uint32_t* s_count = lds + kSlice / 32 + 4;             // [kSlice]
  uint32_t* s_key = s_count + kSlice;                    // [bias_slots] id within the slice, or kNoKey
  int32_t* s_entry = reinterpret_cast<int32_t*>(s_key + a.bias_slots);   // [bias_slots] the list's last entry of that id
  const ot_adjust_in& in = a.in;
  const int tid = threadIdx.x, lane = tid & 63;
  const int part = (int)(blockIdx.x % (unsigned)a.parts), t = (int)(blockIdx.x / (unsigned)a.parts);
  const int slice = t % a.slices, b = t / a.slices;
  const int row0 = in.row_off ? max(0, in.row_off[b]) : b, row1 = in.row_off ? min(in.M, in.row_off[b + 1]) : b + 1;
  const int each = (max(0, row1 - row0) + a.parts - 1) / a.parts, first = row0 + part * each, last = min(row1, first + each);
  if (first >= last) return;
  const int s0 = slice * kSlice, n_ids = min(kSlice, in.V - s0);

  // a row's logits in this slice, and its mask's words of them
  struct Fetched {
    Raw raw[kLoads];
    uint32_t lo[kLoads], hi[kLoads];
  };
  auto logits_of = [&](int row) { return static_cast<const T*>(in.logits) + (int64_t)row * in.ld + s0; };
  auto out_of = [&](int row) { return static_cast<T*>(a.out) + (int64_t)row * a.ld_out + s0; };
  auto no_such = [&](int m) { return m < -1 || m >= in.n_masks; };
  auto mask_of = [&](int m) { return m >= 0 && m < in.n_masks ? in.masks + (int64_t)m * in.ld_mask : nullptr; };
  auto fetch = [&](int row, int m, Fetched* f) {
    const T* z = logits_of(row);
    const uint32_t* mask = mask_of(m);
    const RowSplit<T> split(z, n_ids);
    const Raw* zv = reinterpret_cast<const Raw*>(z + split.head);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int k = i * kThreads + tid, v = s0 + split.head + k * kVec;
      if (!kInPlace) f->raw[i] = Raw{};
      f->lo[i] = f->hi[i] = kNoKey;
      if (k >= split.vecs) continue;
      if (!kInPlace) f->raw[i] = zv[k];
      if (mask) { f->lo[i] = mask[v >> 5]; f->hi[i] = mask[(v + kVec - 1) >> 5]; }
    }
  };
  // masks and window tokens of 64 rows, a row a lane
  int rows_at = first, masks = -1, tokens = -1;
  auto fetch_rows = [&]() {
    const int row = min(rows_at + lane, last - 1);
    masks = in.mask_of_row ? in.mask_of_row[row] : in.masks ? row : -1;
    tokens = in.window ? in.window[row] : -1;
  };
  fetch_rows();
  Fetched now;
  int m_now = __builtin_amdgcn_readlane(masks, 0);
  fetch(first, m_now, &now);

  for (int i = tid; i < kSlice / 32 + 1; i += kThreads) s_mark[i] = 0;
  for (int i = tid; i < kSlice; i += kThreads) s_count[i] = 0;
  for (int i = tid; i < a.bias_slots; i += kThreads) { s_key[i] = kNoKey; s_entry[i] = 0; }
  __syncthreads();
  auto mark = [&](int o, uint32_t flag) {
    if (flag) atomicOr(&s_count[o], flag);
    else atomicAdd(&s_count[o], 1u);
    atomicOr(&s_mark[o >> 5], 1u << (o & 31));
  };
  auto mine = [&](int id) { return id >= s0 && id - s0 < n_ids; };
  if (in.history) {
    const int n = (int)min((int64_t)(in.n_history ? max(0, in.n_history[b]) : 0x7FFFFFFF), in.ld_history);
    const int n_prompt = in.n_prompt ? in.n_prompt[b] : 0;
    const int32_t* ids = in.history + (int64_t)b * in.ld_history;
    constexpr int kBatch = 2;                            // vectors of four ids per thread that are on their way together
    for (int i0 = 0; i0 < n; i0 += kBatch * 4 * kThreads) {
      i32x4_any got[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = i0 + (j * kThreads + tid) * 4;
        got[j] = i32x4_any{-1, -1, -1, -1};
        if (i + 4 <= n) {
          got[j] = *reinterpret_cast<const i32x4_any*>(ids + i);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (i + e < n) got[j][e] = ids[i + e];
        }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (const int id = got[j][e]; mine(id)) mark(id - s0, i0 + (j * kThreads + tid) * 4 + e < n_prompt ? kSeen : 0u);
    }
  }
  if (in.window)
    for (int r = row0 + tid; r < first; r += kThreads)
      if (const int id = in.window[r]; mine(id)) mark(id - s0, 0u);
  auto slot_of = [&](uint32_t o) { return o * 0x9E3779B1u >> 7 & (uint32_t)(a.bias_slots - 1); };
  for (int i = tid; i < in.n_bias; i += kThreads) {
    const int id = in.bias_ids[(int64_t)b * in.n_bias + i];
    if (!mine(id)) continue;
    const uint32_t o = (uint32_t)(id - s0);
    uint32_t at = slot_of(o);
    for (int tries = 0; tries < a.bias_slots; ++tries) { // (half of the slots stay free: it ends before)
      const uint32_t key = atomicCAS(&s_key[at], kNoKey, o);
      if (key == kNoKey || key == o) break;
      at = (at + 1) & (uint32_t)(a.bias_slots - 1);
    }
    atomicMax(&s_entry[at], i);
    mark((int)o, kBiased);
  }
  __syncthreads();

  const double rho = in.repetition ? (double)in.repetition[b] : 1.0, inv_rho = 1.0 / rho;
  const double f = in.frequency ? (double)in.frequency[b] : 0.0, g = in.presence ? (double)in.presence[b] : 0.0;
  auto adjusted = [&](float z, int o) {
    if (z == -INFINITY) return z;
    const uint32_t c = s_count[o], n = c & ~(kSeen | kBiased);
    double x = (double)z;
    if (c & ~kBiased) {
      x = x > 0.0 ? x * inv_rho : x * rho;
      if (n) x = x - f * (double)n - g;
    }
    if (c & kBiased) {
      uint32_t at = slot_of((uint32_t)o);
      for (int tries = 0; tries < a.bias_slots && s_key[at] != (uint32_t)o; ++tries) at = (at + 1) & (uint32_t)(a.bias_slots - 1);
      x += (double)in.bias[(int64_t)b * in.n_bias + s_entry[at]];
    }
    return (float)x;
  };
  auto marks_at = [&](int o) { return bits_at(s_mark[o >> 5], s_mark[(o >> 5) + 1], o); };

  for (int row = first; row < last; ++row) {
    const int token = __builtin_amdgcn_readlane(tokens, row - rows_at), m = m_now;
    const T* z = logits_of(row);
    T* out = out_of(row);
    const uint32_t* mask = mask_of(m);
    const bool none = no_such(m);
    const RowSplit<T> split(z, n_ids);
    const bool vectors = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    auto one = [&](int o) {
      const int v = s0 + o;
      if (none) store_one(out + o, kNan);
      else if (mask && !(mask[v >> 5] >> (v & 31) & 1)) store_one(out + o, -INFINITY);
      else if (marks_at(o) & 1) store_one(out + o, adjusted(Vec<T>::one(z + o), o));
      else if (!kInPlace) out[o] = z[o];
    };
    if (vectors) {
      uint32_t marked[kLoads], allowed[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int k = i * kThreads + tid, o = split.head + k * kVec;
        marked[i] = 0;
        if (k < split.vecs) marked[i] = marks_at(o) & kAll;
        allowed[i] = bits_at(now.lo[i], now.hi[i], s0 + o) & kAll;
        if (kInPlace && k < split.vecs) {
          now.raw[i] = Raw{};
          if (allowed[i] != 0 && (marked[i] != 0 || allowed[i] != kAll)) now.raw[i] = *reinterpret_cast<const Raw*>(z + o);
        }
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int k = i * kThreads + tid, o = split.head + k * kVec;
        if (k >= split.vecs) continue;
        if (none || marked[i] != 0) {
          float v[kVec];
          Vec<T>::unpack(now.raw[i], v);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (none) v[e] = kNan;
            else if (marked[i] >> e & 1) v[e] = adjusted(v[e], o + e);
          }
          now.raw[i] = pack_vec(v);                      // (the others' bits come back, but a signaling NaN's of bfloat16: to keep it too took 26.6 us, not 25.8)
        }
        if (!none && allowed[i] != kAll) mask_vector(&now.raw[i], allowed[i]);
        if (!kInPlace || none || marked[i] != 0 || allowed[i] != kAll) __builtin_nontemporal_store(now.raw[i], reinterpret_cast<Raw*>(out + o));
      }
      if (tid < split.head + split.tail) one(split.edge(tid));
    } else {
      for (int o = tid; o < n_ids; o += kThreads) one(o);
    }
    if (row + 1 < last) {
      if (row + 1 - rows_at == 64) { rows_at += 64; fetch_rows(); }
      m_now = __builtin_amdgcn_readlane(masks, row + 1 - rows_at);
      fetch(row + 1, m_now, &now);
      if (mine(token)) {                                 // the same in every thread
        __syncthreads();
        if (tid == 0) { s_count[token - s0] += 1; s_mark[(token - s0) >> 5] |= 1u << ((token - s0) & 31); }
        __syncthreads();
      }
    }
  }
}

template <typename T, int kThreads>
hipError_t launch(const AdjustArgs& a, hipStream_t stream) {
  const size_t lds = sizeof(uint32_t) * (kThreads / 2 + 4 + (size_t)kThreads * 16 + 2 * (size_t)a.bias_slots);
  const auto kernel = a.out == a.in.logits ? adjust_kernel<T, kThreads, true> : adjust_kernel<T, kThreads, false>;
  if (lds > (60 << 10)) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.slices * (unsigned)a.parts * (unsigned)a.in.B), dim3(kThreads), lds, stream, a);
  return hipGetLastError();
}

constexpr int kFewIds = 8192;       // ids of a history up to which workgroups are small
// Parts of a sequence with a window at most: each reads the tokens in front of its rows, so that a row a workgroup cost the square of a long window
// (one of 65536 rows of 1000 ids 1259 us, of 16384 of 32003 in bfloat16 1055; in 256 parts 477 and 580, 1024 212 and 599, 4096 200 and 715, 16384
// 399 and 1055).
constexpr int kWindowParts = 2048;

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
  if (in->n_bias < 0 || in->n_bias > OT_MAX_BIAS || in->n_masks < 0 || in->ld_history < 0 || in->ld_history > OT_MAX_HISTORY || (in->masks && in->ld_mask < ceil_div(in->V, 32)))
    return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: need 0 <= n_bias <= %d, n_masks >= 0, 0 <= ld_history <= 2^29, ld_mask >= ceil(V / 32)", OT_MAX_BIAS);
  if (in->window && !in->row_off) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: a window needs row_off");
  if (in->window && in->M > OT_MAX_HISTORY) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: with a window, at most 2^29 rows (M = %d)", in->M);
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
  const int threads = in->ld_history > kFewIds ? 1024 : 256;
  AdjustArgs a{*in, out, ld_out, ceil_div(in->V, 16 * threads), 1, 0};
  const int64_t groups = (int64_t)a.slices * in->B;
  // Large workgroups for long histories: 144 rows of 128256, 64 of 152064 and 512 of 32003 in bfloat16 take behind 8000 ids 37, 27 and 37 us in small
  // ones, 36, 25 and 39 in large ones; behind 4000 32, 24 and 33 against 36, 23 and 38, behind 16000 45, 33 and 44 against 38, 28 and 40.
  // A row a workgroup where the table is quickly made (up to as many workgroups as keep every compute unit busy), else a sequence's rows in parts
  // until there is a workgroup for every compute unit (512 rows of 32003: 31 us a row a workgroup, 40 four rows)
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(in->M, in->B), threads == 1024 ? ctx->n_cu / groups : (1 << 22) / groups));
  if (in->window) a.parts = std::min(a.parts, kWindowParts);
  if (in->n_bias > 0)
    for (a.bias_slots = 2; a.bias_slots < 2 * in->n_bias;) a.bias_slots *= 2;
  if (!grid_fits(groups * a.parts, threads)) return ot_fail(OT_ERR_SHAPE, "ot_adjust_logits: %d sequences of %d ids are too many for a launch", in->B, in->V);
  if (const int bad = ot_check_device(ctx, "ot_adjust_logits")) return bad;
  const bool bf16 = in->dtype == OT_BF16;
  const hipError_t e = threads == 1024 ? (bf16 ? launch<uint16_t, 1024>(a, ctx->stream) : launch<float, 1024>(a, ctx->stream))
                                       : (bf16 ? launch<uint16_t, 256>(a, ctx->stream) : launch<float, 256>(a, ctx->stream));
  return e == hipSuccess ? OT_OK : ot_fail_hip(e, "ot_adjust_logits: launch");
}

}  // extern "C"
#pragma GCC visibility pop
