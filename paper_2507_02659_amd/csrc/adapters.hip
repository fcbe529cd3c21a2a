// Low-rank adapters of many requests beside the head: out = logits + scale (hidden down^T) up^T, every row through its own adapter's matrices.
//
// Rows are taken in blocks of 64: one row a lane, a wavefront finds the block's adapters and their rows by ballots, without a sort and
// without a launch of its own.  Rows of one adapter go 16 at a time (a tile) through the matrix instructions.  Two launches: hidden rows to
// u = scale (hidden down^T), a few numbers per row, then u to the logits.
#include <math.h>

#include <algorithm>

#include "otv_host.h"
#include "rows.h"

namespace otv {
namespace {

struct AdapterArgs {
  ot_adapter_in in;
  void* out;
  int64_t ld_out;
  uint8_t* u;              // OT_BF16: [3][rows][depth] bfloat16, else [rows][depth] float32, rows = those of the launch
  int32_t row0, rows;      // the launch's rows
  int32_t depth;           // rank in whole 32s
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
// four neighbouring logits, from any element on
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ inline f32x4 load4(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(p)); }
__device__ inline f32x4 load4(const uint16_t* p) {
  const u16x4_any x = __builtin_nontemporal_load(reinterpret_cast<const u16x4_any*>(p));
  return f32x4{bf16_to_f32(x.x), bf16_to_f32(x.y), bf16_to_f32(x.z), bf16_to_f32(x.w)};
}
__device__ inline void store4(float* p, f32x4 x) { __builtin_nontemporal_store(f32x4_any(x), reinterpret_cast<f32x4_any*>(p)); }
__device__ inline void store4(uint16_t* p, f32x4 x) {
  u16x4_any r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
  __builtin_nontemporal_store(r, reinterpret_cast<u16x4_any*>(p));
}

// Operands of the matrix instructions: of 16 rows (lane & 15) the kDepth products' indices from k0 on, those past K as 0.  Which of the block's
// indices a lane's element stands for is the same on both sides, so any order will do.
template <typename W> struct Operand;
template <> struct Operand<uint16_t> {
  static constexpr int kDepth = 32;
  typedef bf16x8 Frag;
  __device__ static Frag load(const uint16_t* row, int k0, int K, int lane) {
    const int k = k0 + (lane >> 4) * 8;
    return k < K ? *reinterpret_cast<const Frag*>(row + k) : Frag{};             // K is a multiple of 8
  }
  __device__ static f32x4 product(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<float> {
  static constexpr int kDepth = 16;
  typedef f32x4 Frag;
  __device__ static Frag load(const float* row, int k0, int K, int lane) {
    const int k = k0 + (lane >> 4) * 4;
    if (k + 4 <= K) return *reinterpret_cast<const f32x4_any*>(row + k);
    Frag f{};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k + i < K) f[i] = row[k + i];
    return f;
  }
  __device__ static f32x4 product(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

// The adapters of a block of 64 rows, one after the other.
struct Block {
  int lane, adapter;                 // the lane's row's: -1 none, -2 no such
  unsigned long long left;           // lanes whose rows are still to come
  int now;                           // the adapter at hand,
  int n;                             // its rows,
  int order;                         // lane i: the i-th of them
  __device__ Block(const AdapterArgs& a, int block, int lane_) : lane(lane_) {
    const int row = block * 64 + lane;
    const bool here = row < a.rows;
    adapter = here ? a.in.adapter[a.row0 + row] : -1;
    if (adapter < -1 || adapter >= a.in.n_adapters) adapter = -2;
    left = __ballot(here);
  }
  // the next adapter among the rows that are left
  __device__ bool next() {
    if (left == 0) return false;
    now = __builtin_amdgcn_readlane(adapter, (int)__builtin_ctzll(left));
    const unsigned long long mine = __ballot(adapter == now) & left;
    left &= ~mine;
    n = (int)__popcll(mine);
    const unsigned long long below = (1ull << lane) - 1;
    const int to = mine >> lane & 1 ? (int)__popcll(mine & below) : n + (int)__popcll(~mine & below);   // a permutation of the lanes
    order = __builtin_amdgcn_ds_permute(to * 4, lane);
    return true;
  }
  // row of the block of the i-th of the adapter's rows, those past the last as the first
  __device__ int row(int i) const { return __shfl(order, i < n ? i : 0); }
};

// Grid = blocks of 64 rows x 16s of the rank x kSlots.  A workgroup takes every kSlots-th tile of its block; its 16 wavefronts share the hidden
// indices and add their sums in LDS, in one order.
constexpr int kDownWaves = 16;
template <typename W>
__global__ __launch_bounds__(64 * kDownWaves) void adapter_down_kernel(AdapterArgs a, int slots) {
  typedef Operand<W> Op;
  const ot_adapter_in& in = a.in;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int slot = (int)(blockIdx.x % (unsigned)slots), t0 = (int)(blockIdx.x / (unsigned)slots);
  const int r0 = t0 % (a.depth / 16) * 16, block = t0 / (a.depth / 16);
  __shared__ float s_part[kDownWaves][256];
  Block rows(a, block, lane);
  int tile = 0;
  while (rows.next()) {
    if (rows.now < 0) continue;
    for (int q = 0; q < rows.n; q += 16, ++tile) {
      if (tile % slots != slot) continue;
      const int r = r0 + (lane & 15), m = block * 64 + rows.row(q + (lane & 15));
      const W* down = static_cast<const W*>(in.down) + ((int64_t)rows.now * in.rank + min(r, in.rank - 1)) * in.d;
      const W* hidden = static_cast<const W*>(in.hidden) + (int64_t)(a.row0 + m) * in.d;
      const int K = r < in.rank ? in.d : 0;
      f32x4 sum{};
      for (int k0 = wave * Op::kDepth; k0 < in.d; k0 += kDownWaves * Op::kDepth)
        sum = Op::product(Op::load(down, k0, K, lane), Op::load(hidden, k0, in.d, lane), sum);
      // lane: of row (lane & 15) the ranks (lane >> 4) * 4 ..
#pragma unroll
      for (int i = 0; i < 4; ++i) s_part[wave][lane * 4 + i] = sum[i];
      __syncthreads();
      if (tid < 256) {
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kDownWaves; ++w) all += (double)s_part[w][tid];
        const float scale = in.scale ? in.scale[rows.now] : 1.f;
        const float u = (float)(all * (double)scale);
        const int l = tid >> 2, rank = r0 + (l >> 4) * 4 + (tid & 3), i = q + (l & 15);
        const int at = block * 64 + rows.row(i);         // (whole wavefronts come here)
        if (i < rows.n) {
          if constexpr (sizeof(W) == 2) {                // three parts, whose sum is u
            uint16_t* to = reinterpret_cast<uint16_t*>(a.u) + (int64_t)at * a.depth + rank;
            const int64_t part = (int64_t)a.rows * a.depth;
            const float hi = (float)(__bf16)u, mid = (float)(__bf16)(u - hi);
            store_one(to, hi);
            store_one(to + part, mid);
            store_one(to + 2 * part, u - hi - mid);
          } else {
            reinterpret_cast<float*>(a.u)[(int64_t)at * a.depth + rank] = u;
          }
        }
      }
      __syncthreads();
    }
  }
}

// Grid = strips of 256 ids x blocks of 64 rows; a wavefront has 64 ids of all of the block's rows.  The matrix of the ids is the first operand, so
// that a lane ends up with four neighbouring ids of one row.
template <typename W, typename T, int kBlocks>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs a, int strips) {
  typedef Operand<W> Op;
  typedef typename Op::Frag Frag;
  constexpr int kParts = sizeof(W) == 2 ? 3 : 1;
  const ot_adapter_in& in = a.in;
  const int wave = uniform((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int strip = (int)(blockIdx.x % (unsigned)strips), block = (int)(blockIdx.x / (unsigned)strips);
  const int v0 = strip * 256 + wave * 64;
  if (v0 >= in.V) return;
  Block rows(a, block, lane);
  while (rows.next()) {
    if (rows.now == -1 && a.out == in.logits) continue;
    Frag up[kBlocks][4];
    if (rows.now >= 0) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const W* row = static_cast<const W*>(in.up) + ((int64_t)rows.now * in.V + min(v0 + c * 16 + (lane & 15), in.V - 1)) * in.rank;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) up[kb][c] = Op::load(row, kb * Op::kDepth, in.rank, lane);
      }
    }
    for (int q = 0; q < rows.n; q += 16) {
      const int m = block * 64 + rows.row(q + (lane & 15));
      const bool mine = q + (lane & 15) < rows.n;
      const int64_t row = a.row0 + m;
      const T* z = static_cast<const T*>(in.logits) + row * in.ld;
      T* out = static_cast<T*>(a.out) + row * a.ld_out;
      f32x4 base[4], sum[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int v = v0 + c * 16 + (lane >> 4) * 4;
        base[c] = f32x4{};
        sum[c] = f32x4{};
        if (!in.logits || !mine) continue;
        if (v + 4 <= in.V) {
          base[c] = load4(z + v);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (v + i < in.V) base[c][i] = Vec<T>::one(z + v + i);
        }
      }
      if (rows.now >= 0) {
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
#pragma unroll
          for (int part = kParts - 1; part >= 0; --part) {
            const W* u = reinterpret_cast<const W*>(a.u) + ((int64_t)part * a.rows + m) * a.depth;
            const Frag x = Op::load(u, kb * Op::kDepth, a.depth, lane);
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] = Op::product(up[kb][c], x, sum[c]);
          }
        }
      } else if (rows.now == -2) {
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] = f32x4{kNan, kNan, kNan, kNan};
      }
      if (!mine) continue;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int v = v0 + c * 16 + (lane >> 4) * 4;
        const f32x4 x = base[c] + sum[c];
        if (v + 4 <= in.V) {
          store4(out + v, x);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (v + i < in.V) store_one(out + v + i, x[i]);
        }
      }
    }
  }
}

template <typename W, typename T>
hipError_t launch_up(const AdapterArgs& a, dim3 grid, int strips, hipStream_t stream) {
  const int blocks = ceil_div(a.in.rank, Operand<W>::kDepth);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, strips); return hipGetLastError(); };
  if (blocks <= 1) return go(adapter_up_kernel<W, T, 1>);
  if (blocks <= 2) return go(adapter_up_kernel<W, T, 2>);
  if (blocks <= 4) return go(adapter_up_kernel<W, T, 4>);
  if constexpr (sizeof(W) == 4)
    if (blocks > 8) return go(adapter_up_kernel<W, T, 16>);
  return go(adapter_up_kernel<W, T, 8>);
}

template <typename W>
hipError_t launch_adapters(const AdapterArgs& a, hipStream_t stream) {
  const int blocks = ceil_div(a.rows, 64), strips = ceil_div(a.in.V, 256);
  const int slots = std::min({a.rows, 16, std::min(a.in.n_adapters, 64) + 3});
  hipLaunchKernelGGL(adapter_down_kernel<W>, dim3((unsigned)(blocks * (a.depth / 16) * slots)), dim3(64 * kDownWaves), 0, stream, a, slots);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)strips * (unsigned)blocks);
  return a.in.logits_dtype == OT_BF16 ? launch_up<W, uint16_t>(a, grid, strips, stream) : launch_up<W, float>(a, grid, strips, stream);
}

}  // namespace
}  // namespace otv

using namespace otv;

#pragma GCC visibility push(default)
extern "C" {

int ot_adapter_logits(ot_ctx* ctx, const ot_adapter_in* in, void* out, int64_t ld_out) {
  if (!ctx || !in) return ot_fail(OT_ERR_NULL, "ot_adapter_logits: ctx and in must not be NULL");
  if ((in->dtype != OT_BF16 && in->dtype != OT_F32) || (in->logits_dtype != OT_BF16 && in->logits_dtype != OT_F32))
    return ot_fail(OT_ERR_DTYPE, "ot_adapter_logits: types are OT_BF16 or OT_F32 (%d, %d)", in->dtype, in->logits_dtype);
  const int64_t size = in->logits_dtype == OT_BF16 ? 2 : 4;
  const int unit = in->dtype == OT_BF16 ? 8 : 4;
  if (in->M < 0 || in->d < 1 || in->V < 1 || in->V > (1 << 30) || in->n_adapters < 1 || (in->logits && in->ld < in->V) || ld_out < in->V)
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: need M >= 0, d >= 1, 1 <= V <= 2^30, n_adapters >= 1, ld and ld_out >= V (M = %d, d = %d, V = %d, n_adapters = %d)",
                   in->M, in->d, in->V, in->n_adapters);
  if (in->rank < 1 || in->rank > OT_MAX_ADAPTER_RANK || in->rank % unit != 0 || (in->dtype == OT_BF16 && in->d % 8 != 0))
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: the rank is a multiple of %d up to %d, d of bf16 a multiple of 8 (rank = %d, d = %d)", unit, OT_MAX_ADAPTER_RANK,
                   in->rank, in->d);
  if (in->reserved != 0) return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: reserved must be 0");
  if (in->M == 0) return OT_OK;
  if (!in->hidden || !in->down || !in->up || !in->adapter || !out)
    return ot_fail(OT_ERR_NULL, "ot_adapter_logits: hidden, down, up, adapter and out must not be NULL");
  if ((reinterpret_cast<uintptr_t>(in->hidden) | reinterpret_cast<uintptr_t>(in->down) | reinterpret_cast<uintptr_t>(in->up)) % 16)
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: hidden, down and up start at a multiple of 16 bytes");
  if (reinterpret_cast<uintptr_t>(in->logits) % size || reinterpret_cast<uintptr_t>(out) % size)
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: logits and out must be aligned to their type");
  if (out == in->logits && ld_out != in->ld) return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: in place, ld_out must be ld");
  if (in->logits && ot_rows_overlap(in->logits, in->ld, out, ld_out, in->M, in->V, size))
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: rows of out overlap other places of the logits' rows");
  const int most = std::min(in->M, kAdapterRows);
  if (!grid_fits((int64_t)ceil_div(in->V, 256) * ceil_div(most, 64), 256))
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: %d ids are too many for a launch of %d rows", in->V, most);
  if (const int bad = ot_check_device(ctx, "ot_adapter_logits")) return bad;
  for (int row0 = 0; row0 < in->M; row0 += kAdapterRows) {
    const AdapterArgs a{*in, out, ld_out, ctx->adapter_u, row0, std::min(in->M - row0, kAdapterRows), ceil_div(in->rank, 32) * 32};
    const hipError_t e = in->dtype == OT_BF16 ? launch_adapters<uint16_t>(a, ctx->stream) : launch_adapters<float>(a, ctx->stream);
    if (e != hipSuccess) return ot_fail_hip(e, "ot_adapter_logits: launch");
  }
  return OT_OK;
}

}  // extern "C"
#pragma GCC visibility pop
