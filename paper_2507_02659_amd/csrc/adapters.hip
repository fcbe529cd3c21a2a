// Low-rank adapters of many requests beside the head: out = logits + scale (hidden down^T) up^T, every row through its own adapter's matrices.
//
// Rows are taken in blocks of 64: one row a lane, a wavefront finds the block's adapters and their rows by ballots, without a sort and
// without a launch of its own.  Rows of one adapter go 16 at a time (a tile) through the matrix instructions.  Two launches: hidden rows to
// u = scale (hidden down^T), a few numbers per row, then u to the logits, which is where the bytes are: every logit is read and written once.
//
// Rounding: products of bfloat16 are exact, sums fp32.  u is rounded to float32 and, as an operand of bfloat16 instructions, split into three
// parts that hold all of its 24 bits; with the nearest bfloat16 alone the sums would be off by 2^-9, a thousand times their own rounding.  The
// two parts more cost nothing where the logits' bytes do not wait for instructions (144 rows of 128256 ids, rank 16: 38 us, with one part alone
// 37.5) and a quarter where they do (2000 rows of 32003 in bfloat16, rank 64: 95 us and 72).
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
  uint8_t* u;              // OT_BF16: [rows][3][depth] bfloat16, else [rows][depth] float32, rows = those of the launch
  int32_t row0, rows;      // the launch's rows
  int32_t depth;           // rank in whole 32s
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));   // from any element on

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

// Grid = slots x 16s of the rank x blocks of 64 rows.  A workgroup takes every slots-th tile of its block; its 16 wavefronts share the hidden
// indices and add their sums in LDS, in one order.  3.5 us with one row of 1024 indices, 11.4 with 144 of 4096 (rank 16), 13.4 with 2000 of 2056 (rank
// 64), as long with nothing in front of it (3.4, 11.2 and 13.6 in a row of such launches alone) and with every load from a cached line: it is bound
// by its own chain, the adapters' numbers, the loads behind them, the sums through LDS.  Float32 matrices 19.5 instead of 11.4.  Indices split over
// four workgroups, whose sums the last one adds, took 10.0 and 16.4; eight steps of loads ahead instead of four changed nothing.
constexpr int kDownWaves = 16, kDownSteps = 4;
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
      const int K = r < in.rank ? in.d : 0, end = r0 < in.rank ? in.d : 0;   // (behind the rank: zeros)
      f32x4 sum{};
      for (int k0 = wave * Op::kDepth; k0 < end; k0 += kDownSteps * kDownWaves * Op::kDepth) {
        typename Op::Frag x[kDownSteps], y[kDownSteps];
#pragma unroll
        for (int i = 0; i < kDownSteps; ++i) {
          const int k = k0 + i * kDownWaves * Op::kDepth;
          x[i] = Op::load(down, k, K, lane);
          y[i] = Op::load(hidden, k, in.d, lane);
        }
#pragma unroll
        for (int i = 0; i < kDownSteps; ++i) sum = Op::product(x[i], y[i], sum);
      }
      // lane: of row (lane & 15) the ranks (lane >> 4) * 4 ..
#pragma unroll
      for (int i = 0; i < 4; ++i) s_part[wave][lane * 4 + i] = sum[i];
      __syncthreads();
      if (tid < 256) {
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kDownWaves; ++w) all += (double)s_part[w][tid];
        const float scale = in.scale ? in.scale[rows.now] : 1.f;
        float u = (float)(all * (double)scale);
        if (!isfinite(u)) u = kNan;                      // (else 0 * inf or a sign would decide what becomes of the row)
        const int l = tid >> 2, rank = r0 + (l >> 4) * 4 + (tid & 3), i = q + (l & 15);
        const int at = block * 64 + rows.row(i);         // (whole wavefronts come here)
        if (i < rows.n) {
          if constexpr (sizeof(W) == 2) {                // three parts, whose sum is u
            uint16_t* to = reinterpret_cast<uint16_t*>(a.u) + (int64_t)at * 3 * a.depth + rank;
            float hi = (float)(__bf16)u;                 // (from 255.5 2^120 on the nearest is infinite: the largest, and the rest in the others)
            if (isinf(hi)) hi = copysignf(0x1.fep127f, hi);
            const float mid = (float)(__bf16)(u - hi);
            store_one(to, hi);
            store_one(to + a.depth, mid);
            store_one(to + 2 * a.depth, u - hi - mid);
          } else {
            reinterpret_cast<float*>(a.u)[(int64_t)at * a.depth + rank] = u;
          }
        }
      }
      __syncthreads();
    }
  }
}

// Grid = strips of ids x slots x blocks of 64 rows; a workgroup takes every slots-th tile of its block.  A tile's sums are formed 64 ids a wavefront and go
// through LDS to the logits, which a wavefront reads and writes row by row in whole 16-byte vectors, wherever the row starts: a strip has the
// vectors that begin in its kStride ids, and computes the kVec - 1 ids more that the last of them may reach.  In LDS a row is shifted so that
// its vectors are whole there too.  The next tile's logits are on their way while one is taken.
// 144 rows of 128256 ids, rank 16, 38 us (208 MB: 5.5 TB/s, a copy's rate); 2000 rows of 32003 in bfloat16, rank 64, 95 us (2.7 TB/s): there a tile's
// instructions come on top of its bytes: with one of the three parts 72 us, with rows that all start at 16 bytes (32256 ids) 91.  Ranks 33 to 64
// of bfloat16 matrices spill 4 to 12 registers, those above 64 leave a compute unit one workgroup: 144 rows of 128256, rank 16, 64, 128 and 256,
// 38, 89, 128 and 231 us (208, 386, 623 and 1098 MB: 5.5, 4.3, 4.9, 4.8 TB/s); float32 matrices of rank 16, 64, 128 51, 127, 235.  Each lane
// storing its own four ids without LDS took 48 and 216 us, strips of 64 ids per wavefront 62 and 134, of 256 per workgroup 50 and 127.  Strips follow
// each other in memory: with the blocks of a strip on one XCD after the other 68 us instead of 50.
constexpr int kUpWaves = 8, kStrip = 64 * kUpWaves, kFront = 8;
constexpr int kPitch = kStrip + kFront + 4;              // four rows on another quarter of the 64 banks than the next four
template <typename T>
constexpr int kStride = kStrip - Vec<T>::kElems;
template <typename W, typename T, int kBlocks>
__global__ __launch_bounds__(64 * kUpWaves, kBlocks <= 2 ? 4 : 2) void adapter_up_kernel(AdapterArgs a, int strips, int slots) {
  typedef Operand<W> Op;
  typedef typename Op::Frag Frag;
  typedef typename Vec<T>::Raw Raw;
  constexpr int kParts = sizeof(W) == 2 ? 3 : 1, kVec = Vec<T>::kElems, kTurns = kStrip / (64 * kVec), kRows = 16 / kUpWaves;
  constexpr bool kLargest = kBlocks == 4;
  const ot_adapter_in& in = a.in;
  const int wave = uniform((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int strip = (int)(blockIdx.x % (unsigned)strips), t0 = (int)(blockIdx.x / (unsigned)strips), slot = t0 % slots, block = t0 / slots;
  __shared__ alignas(16) float s_sum[2][16][kPitch];
  const int v0 = strip * kStride<T>, own = wave * 64;
  const bool edges = strip == 0 || v0 + kStrip >= in.V;
  const int row_at = a.row0 + block * 64;                // first row of the block
  auto out_of = [&](int row) { return static_cast<T*>(a.out) + (row_at + (int64_t)row) * a.ld_out; };
  auto logits_of = [&](int row) { return in.logits ? static_cast<const T*>(in.logits) + (row_at + (int64_t)row) * in.ld : nullptr; };
  // ids of the strip in front of a row's first vector: modulo kVec, so 32 bits will do
  const uint32_t at_v0 = (uint32_t)(reinterpret_cast<uintptr_t>(a.out) / sizeof(T)) + (uint32_t)v0 + (uint32_t)row_at * (uint32_t)a.ld_out;
  auto first_of = [&](int row) { return (int)(0u - (at_v0 + (uint32_t)row * (uint32_t)a.ld_out) & (uint32_t)(kVec - 1)); };
  // whether the logits' rows have their vectors where the output's do
  const bool vectors = ((reinterpret_cast<uintptr_t>(in.logits) ^ reinterpret_cast<uintptr_t>(a.out)) & 15) == 0 && (((uint32_t)in.ld - (uint32_t)a.ld_out) & (kVec - 1)) == 0;
  // first id of the lane's t-th vector, or -1
  auto id_of = [&](int first, int t) {
    const int at = first + (t * 64 + lane) * kVec;
    return at < kStride<T> && v0 + at + kVec <= in.V ? v0 + at : -1;
  };
  Block rows(a, block, lane);
  // A tile: its adapter (-3: none is left), the adapter's rows in the block, which they are, the tile's first.
  struct Tile { int adapter, n, order, q; };
  auto behind = [&](const Tile& t) {
    if (t.q + 16 < t.n) return Tile{t.adapter, t.n, t.order, t.q + 16};
    do {
      if (!rows.next()) return Tile{-3, 0, 0, 0};
    } while (rows.now == -1 && a.out == in.logits);      // in place there is nothing to do for rows without an adapter
    return Tile{rows.now, rows.n, rows.order, 0};
  };
  int seen = 0;
  auto after = [&](Tile t) {                             // the next that is this workgroup's
    do t = behind(t);
    while (t.adapter != -3 && seen++ % slots != slot);
    return t;
  };
  auto load_base = [&](const Tile& of, Raw (&base)[kRows][kTurns]) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int i = of.q + wave + kUpWaves * j;
#pragma unroll
      for (int t = 0; t < kTurns; ++t) base[j][t] = Raw{};
      if (i >= of.n || !in.logits) continue;
      const int row = __builtin_amdgcn_readlane(of.order, i);
      const T* z = logits_of(row);
      const int first = first_of(row);
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int id = id_of(first, t);
        if (id < 0) continue;
        if (vectors) {
          base[j][t] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(z + id));
        } else {
          float x[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[e] = Vec<T>::one(z + id + e);
          base[j][t] = pack_vec(x);
        }
      }
    }
  };
  constexpr int kChunk = kBlocks * Op::kDepth;            // of the rank: so much of the operands is held; a larger rank reads them in turn for every tile
  Frag up[kBlocks][4], u[kBlocks][kParts];
  constexpr int kAhead = kTurns == 1 ? 2 : 1;            // tiles whose logits are on their way while one is taken
  Raw base[kAhead + 1][kRows][kTurns];
  Tile tile[kAhead + 1];
  int loaded = -1, turn = 0;
  auto load_operands = [&](const Tile& of, int k0) {
    if (of.adapter < 0) return;
    const int i = of.q + (lane & 15);
    // (depth: whole 32s, zeros behind the rank; of up to two blocks of 32 a constant, so that the loads share an address)
    const int depth = kParts == 3 && kBlocks <= 2 ? kBlocks * 32 : a.depth;
    const W* of_row = reinterpret_cast<const W*>(a.u) + (size_t)(uint32_t)((block * 64 + __shfl(of.order, i < of.n ? i : 0)) * kParts * depth + (lane >> 4) * (Op::kDepth / 4));
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
      for (int part = 0; part < kParts; ++part)
        if (kBlocks <= 2 || k0 + kb * Op::kDepth < depth)
          u[kb][part] = *reinterpret_cast<const Frag*>(of_row + part * depth + k0 + kb * Op::kDepth);
        else
          u[kb][part] = Frag{};
    if (of.adapter == loaded && in.rank <= kChunk) return;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const W* row = static_cast<const W*>(in.up) + ((int64_t)of.adapter * in.V + min(v0 + own + c * 16 + (lane & 15), in.V - 1)) * in.rank;
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) up[kb][c] = Op::load(row, k0 + kb * Op::kDepth, in.rank, lane);
    }
    loaded = of.adapter;
  };
  tile[0] = after(Tile{-3, 0, 0, 0});
  load_operands(tile[0], 0);
  load_base(tile[0], base[0]);
#pragma unroll
  for (int i = 1; i < kAhead; ++i) {
    tile[i] = after(tile[i - 1]);
    load_base(tile[i], base[i]);
  }
  while (tile[0].adapter != -3) {
    const int now = tile[0].adapter, now_n = tile[0].n, now_order = tile[0].order, now_q = tile[0].q;
    tile[kAhead] = after(tile[kAhead - 1]);
    load_base(tile[kAhead], base[kAhead]);
    float (*sums)[kPitch] = s_sum[turn];
    f32x4 sum[4] = {};
    auto add_products = [&]() {
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
        for (int part = kParts - 1; part >= 0; --part)
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[c] = Op::product(u[kb][part], up[kb][c], sum[c]);
    };
    if (now >= 0) {
      add_products();
      if constexpr (kLargest)
        for (int k0 = kChunk; k0 < in.rank; k0 += kChunk) {
          load_operands(tile[0], k0);
          add_products();
        }
    }
    // asked for in front of this tile's stores, which a wait for what was asked for behind them would wait for too
    load_operands(tile[1], 0);
    if (now >= 0) {
      // lane: of the rows (lane >> 4) * 4 .. the id (lane & 15) of each 16
      const int i = now_q + (lane & 15), shift = kFront - first_of(__shfl(now_order, i < now_n ? i : 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = (lane >> 4) * 4 + e;
        float* to = &sums[row][own + (lane & 15) + __shfl(shift, row)];
#pragma unroll
        for (int c = 0; c < 4; ++c) to[c * 16] = sum[c][e];
      }
      __syncthreads();
      turn ^= 1;                                         // (the other half is written next: one barrier per tile)
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int i = wave + kUpWaves * j;
      if (now_q + i >= now_n) break;
      const int row = __builtin_amdgcn_readlane(now_order, now_q + i);
      T* out = out_of(row);
      const int first = first_of(row);
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int id = id_of(first, t);
        if (id < 0) continue;
        if (now != -1) {
          float x[kVec];
          Vec<T>::unpack(base[0][j][t], x);
#pragma unroll
          for (int e = 0; e < kVec; e += 4) {
            const f32x4 y = now >= 0 ? *reinterpret_cast<const f32x4*>(&sums[i][kFront + (t * 64 + lane) * kVec + e]) : f32x4{kNan, kNan, kNan, kNan};
            x[e] += y.x; x[e + 1] += y.y; x[e + 2] += y.z; x[e + 3] += y.w;
          }
          base[0][j][t] = pack_vec(x);
        }
        __builtin_nontemporal_store(base[0][j][t], reinterpret_cast<Raw*>(out + id));
      }
      if (edges) {                                       // in front of the row's first vector, behind its last one: one id a lane
        const T* z = logits_of(row);
        const RowSplit<T> split(out, in.V);
        const int tail = split.head + split.vecs * kVec, v = lane < kVec ? lane : tail + lane - kVec;
        if (lane < kVec ? strip == 0 && v < split.head : lane < 2 * kVec && v < in.V && tail >= v0 && tail < v0 + kStride<T>) {
          if (now == -1) out[v] = z ? z[v] : T{};
          else store_one(out + v, (z ? Vec<T>::one(z + v) : 0.f) + (now >= 0 ? sums[i][kFront + v - v0 - first] : kNan));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      tile[i] = tile[i + 1];
#pragma unroll
      for (int j = 0; j < kRows; ++j)
#pragma unroll
        for (int t = 0; t < kTurns; ++t) base[i][j][t] = base[i + 1][j][t];
    }
  }
}

template <typename W, typename T>
hipError_t launch_up(const AdapterArgs& a, int n_cu, hipStream_t stream) {
  const int blocks = ceil_div(a.in.rank, Operand<W>::kDepth), strips = ceil_div(a.in.V, kStride<T>), of_rows = ceil_div(a.rows, 64);
  // a block's tiles one after the other, unless that leaves compute units without a workgroup (56 rows of five adapters and 2251 ids, five strips: 24
  // us in one slot, 9 in 16; shared out with enough strips, the adapter's matrix would be read by every slot: 152064 ids 6.2 us, in two slots 6.7)
  const int slots = std::max(1, std::min({a.rows, 16, (int)(n_cu / ((int64_t)strips * of_rows))}));
  const dim3 grid((unsigned)strips * (unsigned)slots * (unsigned)of_rows);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * kUpWaves), 0, stream, a, strips, slots); return hipGetLastError(); };
  if (blocks <= 1) return go(adapter_up_kernel<W, T, 1>);
  if (blocks <= 2) return go(adapter_up_kernel<W, T, 2>);
  return go(adapter_up_kernel<W, T, 4>);                 // also of more
}

template <typename W>
hipError_t launch_adapters(const AdapterArgs& a, int n_cu, hipStream_t stream) {
  const int blocks = ceil_div(a.rows, 64);
  const int slots = std::min({a.rows, 16, std::min(a.in.n_adapters, 64) + 3});
  hipLaunchKernelGGL(adapter_down_kernel<W>, dim3((unsigned)(blocks * (a.depth / 16) * slots)), dim3(64 * kDownWaves), 0, stream, a, slots);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return a.in.logits_dtype == OT_BF16 ? launch_up<W, uint16_t>(a, n_cu, stream) : launch_up<W, float>(a, n_cu, stream);
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
  if (in->M < 0 || in->d < 1 || in->d > (1 << 24) || in->V < 1 || in->V > (1 << 30) || in->n_adapters < 1 || (in->logits && in->ld < in->V) || ld_out < in->V)
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: need M >= 0, 1 <= d <= 2^24, 1 <= V <= 2^30, n_adapters >= 1, ld and ld_out >= V (M = %d, d = %d, V = %d, n_adapters = %d)",
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
  if (!grid_fits((int64_t)ceil_div(in->V, kStride<uint16_t>) * ceil_div(most, 64), 64 * kUpWaves))
    return ot_fail(OT_ERR_SHAPE, "ot_adapter_logits: %d ids are too many for a launch of %d rows", in->V, most);
  if (const int bad = ot_check_device(ctx, "ot_adapter_logits")) return bad;
  for (int row0 = 0; row0 < in->M; row0 += kAdapterRows) {
    const AdapterArgs a{*in, out, ld_out, ctx->adapter_u, row0, std::min(in->M - row0, kAdapterRows), ceil_div(in->rank, 32) * 32};
    const hipError_t e = in->dtype == OT_BF16 ? launch_adapters<uint16_t>(a, ctx->n_cu, ctx->stream) : launch_adapters<float>(a, ctx->n_cu, ctx->stream);
    if (e != hipSuccess) return ot_fail_hip(e, "ot_adapter_logits: launch");
  }
  return OT_OK;
}

}  // extern "C"
#pragma GCC visibility pop
