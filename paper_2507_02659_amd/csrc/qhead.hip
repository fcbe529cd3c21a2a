// A target head of 4-bit weights with group scales: z[m][v] = sum over groups g of s[g][v] * sum_{k in g} h[m][k] (c[k][v] - zp[g][v]).
//
// The codes c (0..15) become bf16 operands c - 7.5 of v_mfma_f32_16x16x32_bf16: centred, so that what
// a group's product sums is of the size of the weights.  (With 16 + c, by as many instructions, the sums were 24 times the hidden states
// and their rounding 2 to 5 times as large in the logits, without end where c = zp.)  A group's product is sum h (c - 7.5), and the sum of the
// group's hidden states, the same for every column, takes (zp - 7.5) times itself off it; then the group's scale multiplies 16 rows x 16 columns
// in four instructions.  Products of a bf16 number and c - 7.5 are exact in fp32, so what is rounded is the sums alone, 2^-24 of each: a group's
// at most once per hidden index, partial sums of h (c - 7.5) and of h (these times zp - 7.5), and the running total of scaled groups once per
// group, above 16 rows with the offsets of up to four groups in it.  The roundings add up as a random walk.
//
// What bounds it, groups of 128, weights from memory: up to 16 rows the weight stream (6 rows x 3584 x 152064 53 us, 5.4 TB/s, what a
// large copy moves; a bf16 head 163); above, the trips through LDS and registers between the products: 144 x 4096 x 128256 166-176 us, 0.9
// PFLOP/s, where the products alone take 95 and the weights 55; a bf16 head takes 172 there and 900 for 1017 rows, this one 1217.  With parts
// of the work left out (timing only): LDS reads 35 us less, staging 24, dequantisation 4, scaling 0.  Wavefronts of 64 columns, one per SIMD,
// with 32 x 32 x 16 products took 314 us, two blocks of 128 per barrier at nine row tiles 185.  Other ways to c - 7.5 of the same accuracy:
// sizes looked up as fp8 numbers by byte permutations 59 us for the 6 rows, bf16 halves looked up and put together 62.
#include <algorithm>

#include "device_math.h"
#include "otv_internal.h"

namespace otv {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight codes of one packed word as bf16 numbers c - 7.5, in ascending hidden index.  With c - 7.5 = +-(2 m + 1)/2 the fp8 number (e4m3) of sign,
// exponent 0 or 1 and low bits 2 m + 1 is +-(2 m + 1) 2^-9: below 16 of these steps fp8 is a fixed-point format.  Codes 0 .. 3 have sign and m in
// bits 7 and 3 .. 1 of the word's four bytes, and so have codes 4 .. 7 in the word read backwards; a mask and the low one away from that are
// four fp8 numbers, of which a conversion with a factor of 2^8 makes two bf16 numbers at a time.
// Mask, ones and factor come in registers (Bits): the instructions that use them take no literals.  The compiler has to choose these
// instructions itself: one written as inline asm is outside its bookkeeping of the waits between vector and matrix instructions, and
// a matrix product still in flight overwrote such results.
struct Bits {
  uint32_t mask, ones;
  float factor;
};
__device__ inline Bits code_bits() {                     // the empty statements keep the compiler from folding the constants back in
  Bits k{0x8E8E8E8Eu, 0x01010101u, 256.f};
  asm("" : "+s"(k.mask));
  asm("" : "+v"(k.ones));
  asm("" : "+s"(k.factor));
  return k;
}
template <bool kHigh>
__device__ inline uint32_t fp8_to_bf16(uint32_t w, Bits k) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, k.factor, kHigh));
}
__device__ inline u32x4 codes_to_bf16(uint32_t w, Bits k) {
  const uint32_t a = (w & k.mask) | k.ones, b = (__builtin_bitreverse32(w) & k.mask) | k.ones;
  return u32x4{fp8_to_bf16<false>(a, k), fp8_to_bf16<true>(a, k), fp8_to_bf16<false>(b, k), fp8_to_bf16<true>(b, k)};
}
// A group's scale and zero point less 7.5 of one column: the scale's fp32 bits, of which a bf16 or fp16 scale leaves the low 13 free.
__device__ inline float rec_scale(uint32_t r) { return __uint_as_float(r & 0xFFFFE000u); }
__device__ inline float rec_zero(uint32_t r) { return (float)(r & 0xFFu) - 7.5f; }
// What a hidden state that is infinite or NaN has left of a row's logits: no code makes 0 of it, so they are infinite or NaN, and become NaN.
__device__ inline float nan_if_infinite(float z) { return fmaf(z, 0.f, z); }

// One thread per lane's uint4 of codes: tile of 16 columns, block of 128 hidden indices, lane = 16 * (k / 8 % 4) + column.
__global__ void pack_codes_kernel(const uint8_t* __restrict__ codes, int d, int V_t, int blocks, int64_t n, u32x4* __restrict__ packed) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int lane = (int)(i & 63), b = (int)((i >> 6) % blocks);
  const int64_t v = (i >> 6) / blocks * 16 + (lane & 15);
  u32x4 w = {};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int k = b * 128 + ks * 32 + (lane >> 4) * 8 + j;
      const uint32_t c = k < d && v < V_t ? codes[(int64_t)(k >> 1) * V_t + v] >> (4 * (k & 1)) & 15u : 8u;
      const uint32_t m = c & 8u ? c & 7u : ~c & 7u, bits = (c < 8u ? 0x80u : 0u) | m << 1;
      x |= j < 4 ? bits << (8 * j) : __builtin_bitreverse32(bits << (8 * (j - 4)));
    }
    w[ks] = x;
  }
  packed[i] = w;
}

// One thread per scale: [tile][block][16 columns][groups of the block]
__global__ void pack_scales_kernel(const void* __restrict__ scales, int f16, const uint8_t* __restrict__ zeros, int groups, int V_t, int blocks,
                                   int per_block, int64_t n, uint32_t* __restrict__ recs) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const int64_t cell = i / per_block, tb = cell >> 4;
  const int g = (int)(tb % blocks) * per_block + (int)(i % per_block);
  const int64_t v = tb / blocks * 16 + (cell & 15);
  uint32_t r = 0;
  if (g < groups && v < V_t) {
    const int64_t at = (int64_t)g * V_t + v;
    const float s = f16 ? (float)static_cast<const _Float16*>(scales)[at] : bf16_to_f32(static_cast<const uint16_t*>(scales)[at]);
    r = (__float_as_uint(s) & 0xFFFFE000u) | (zeros ? zeros[at] & 15u : 8u);
  }
  recs[i] = r;
}

// What a wavefront reads of the weights: the codes of S tiles of 16 columns and a block of 128 hidden indices, with the scales.
// Addresses are a base that the wavefront shares and 32 bits of the lane's own.
template <int S, int kGroups>
struct Weights {
  u32x4 w[S];
  uint32_t rec[S][kGroups];
};
template <typename T>
__device__ inline T load_at(const void* base, uint32_t bytes) { return *reinterpret_cast<const T*>(static_cast<const char*>(base) + bytes); }
template <int S, int kGroups, bool kOnce>
__device__ inline void load_weights(const QuantHead& q, const int* tile, int b, int lane, Weights<S, kGroups>* out) {
  typedef uint32_t recs_t __attribute__((ext_vector_type(kGroups == 1 ? 2 : kGroups)));
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int64_t at = (int64_t)tile[s] * q.blocks + b;
    const char* codes = reinterpret_cast<const char*>(q.codes) + at * 1024;
    if (kOnce) out->w[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + (uint32_t)lane * 16));
    else out->w[s] = load_at<u32x4>(codes, (uint32_t)lane * 16);
    const char* recs = reinterpret_cast<const char*>(q.recs) + at * (64 * kGroups);
    if constexpr (kGroups == 1) {
      out->rec[s][0] = load_at<uint32_t>(recs, (uint32_t)(lane & 15) * 4);
    } else {
      const recs_t r = load_at<recs_t>(recs, (uint32_t)(lane & 15) * (4 * kGroups));
#pragma unroll
      for (int g = 0; g < kGroups; ++g) out->rec[s][g] = r[g];
    }
  }
}
// The operands of block b of 16 hidden rows; h: the rows' first element, row_at: the lane's row, in bytes.  Indices past d are read from the
// row's end, without a branch (which would make the compiler wait for whatever else is on its way), and zeroed by clear_tail.
__device__ inline void load_hidden(const uint16_t* h, uint32_t row_at, int b, int d, int lane, u32x4* x) {
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) x[ks] = load_at<u32x4>(h, row_at + 2u * min(b * 128 + ks * 32 + (lane >> 4) * 8, d - 8));
}
__device__ inline void clear_tail(int b, int d, int lane, u32x4* x) {
  if ((b + 1) * 128 <= d) return;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    if (b * 128 + ks * 32 + (lane >> 4) * 8 >= d) x[ks] = u32x4{};
}

// Up to 16 rows.  The hidden rows lie in LDS in the order of the matrix instruction's operand, [32-deep step][lane], all of the hidden
// dimension where it fits (chunk_steps steps); behind that every wavefront goes its own way: S tiles of 16 columns and one of `parts`
// parts of the hidden dimension, its weights asked for kAhead blocks ahead.  No barrier until the parts are joined.
template <int S, int kSteps, int kAhead>
__global__ __launch_bounds__(1024) void qhead_rows16_kernel(const uint16_t* __restrict__ H, int M, int d, QuantHead q, float* __restrict__ Z, int V_t,
                                                            int64_t ldz, int chunk_blocks, int parts) {
  constexpr int kGroups = 4 / kSteps;
  extern __shared__ u32x4 s_x[];
  const Bits bits = code_bits();
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n_waves = blockDim.x >> 6;
  const int part = wave % parts, first = ((int)blockIdx.x * (n_waves / parts) + wave / parts) * S;
  int tile[S];
#pragma unroll
  for (int s = 0; s < S; ++s) tile[s] = min(first + s, q.tiles - 1);
  const uint32_t h_at = 2u * (uint32_t)(min(lane & 15, M - 1) * d);
  f32x4 total[S] = {};
  for (int c0 = 0; c0 < q.blocks; c0 += chunk_blocks) {
    const int c1 = min(c0 + chunk_blocks, q.blocks), len = (c1 - c0 + parts - 1) / parts;
    const int b0 = min(c0 + part * len, c1), b1 = min(b0 + len, c1);
    Weights<S, kGroups> ring[kAhead];
    if (b0 < b1) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) load_weights<S, kGroups, true>(q, tile, min(b0 + i, b1 - 1), lane, &ring[i]);
    }
    if (c0 > 0) __syncthreads();
    for (int b = c0 + wave; b < c1; b += n_waves) {
      u32x4 x[4];
      load_hidden(H, h_at, b, d, lane, x);
      clear_tail(b, d, lane, x);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) s_x[((b - c0) * 4 + ks) * 64 + lane] = x[ks];
    }
    __syncthreads();
    for (int b = b0; b < b1; b += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (b + i < b1) {
          const u32x4* x = s_x + (b + i - c0) * 256 + lane;
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            f32x4 acc[S] = {}, sum = {};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
              const int ks = g * kSteps + t;
              const u32x4 xf = x[ks * 64];
              sum = mfma(xf, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, sum);
#pragma unroll
              for (int s = 0; s < S; ++s) acc[s] = mfma(xf, codes_to_bf16(ring[i].w[s][ks], bits), acc[s]);
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
              const float scale = rec_scale(ring[i].rec[s][g]), zero = rec_zero(ring[i].rec[s][g]);
#pragma unroll
              for (int e = 0; e < 4; ++e) total[s][e] = fmaf(scale, fmaf(-zero, sum[e], acc[s][e]), total[s][e]);
            }
          }
          load_weights<S, kGroups, true>(q, tile, min(b + i + kAhead, b1 - 1), lane, &ring[i]);
        }
      }
    }
  }
  if (parts > 1) {                                       // joined in ascending order by the wavefront of part 0
    __syncthreads();
    f32x4* red = reinterpret_cast<f32x4*>(s_x);
    if (part > 0) {
#pragma unroll
      for (int s = 0; s < S; ++s) red[(wave * S + s) * 64 + lane] = total[s];
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 1; p < parts; ++p) {
#pragma unroll
      for (int s = 0; s < S; ++s) total[s] += red[((wave + p) * S + s) * 64 + lane];
    }
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int v = (first + s) * 16 + (lane & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 4 * (lane >> 4) + e;
      if (row < M && v < V_t) Z[(int64_t)row * ldz + v] = nan_if_infinite(total[s][e]);
    }
  }
}

// More than 16 rows: blocks of RT tiles of 16 rows, so that weights are read and dequantised once for up to 144 rows.  A wavefront owns S tiles
// of 16 columns over the whole hidden dimension; the block's hidden rows come through LDS in chunks of kBlocks * 128 hidden indices, two buffers,
// one barrier per chunk.  A wavefront stages whole (row tile, block) units, in the order of the matrix instruction's operand, and forms their
// groups' sums on the way (a product with ones).
constexpr int kTallWaves = 8;
// Blocks per chunk: as many as registers and LDS hold (36 rows x 128256 with two instead of one 78.5 us instead of 82.2).
constexpr int tall_blocks(int RT, int S) { return S > 2 ? (RT <= 4 ? 2 : 1) : RT <= 2 ? 4 : RT <= 4 ? 2 : 1; }
template <int RT, int S, int kSteps, int kAhead>
__global__ __launch_bounds__(64 * kTallWaves) void qhead_tall_kernel(const uint16_t* __restrict__ H, int M, int d, QuantHead q, float* __restrict__ Z,
                                                                     int V_t, int64_t ldz, int m_blocks) {
  constexpr int kGroups = 4 / kSteps, kBlocks = tall_blocks(RT, S), kUnits = kBlocks * RT;
  constexpr int kStage = (kUnits + kTallWaves - 3) / (kTallWaves - 2);   // units per wavefront of six at least
  const Bits bits = code_bits();
  __shared__ u32x4 s_x[2][kUnits][4][64];
  // sums of the hidden states of a row over a group, in rings of blocks: four groups' worth is used at a time, a chunk is staged ahead
  constexpr int kRing = 2 * (kSteps > kBlocks ? kSteps : kBlocks);
  __shared__ float s_sum[kRing][RT][kGroups][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n_waves = blockDim.x >> 6;
  const int slot = (int)blockIdx.x >> 3, row0 = slot % m_blocks * (RT * 16), ct = slot / m_blocks * 8 + ((int)blockIdx.x & 7);
  const int first = (ct * n_waves + wave) * S;
  if (ct * n_waves * S >= q.tiles) return;               // padding of the id space
  int tile[S];
#pragma unroll
  for (int s = 0; s < S; ++s) tile[s] = min(first + s, q.tiles - 1);
  u32x4 stage[kStage][4];
  auto fetch = [&](int c) {                              // this wavefront's units of chunk c
#pragma unroll
    for (int j = 0; j < kStage; ++j) {
      const int u = wave + j * n_waves;
      if (j == 0 || u < kUnits) {
        const int row = min(min(u, kUnits - 1) % RT * 16 + (lane & 15), M - 1 - row0);
        load_hidden(H + (int64_t)row0 * d, 2u * (uint32_t)(row * d), c * kBlocks + min(u, kUnits - 1) / RT, d, lane, stage[j]);
      }
    }
  };
  auto put = [&](int c, int buf) {
#pragma unroll
    for (int j = 0; j < kStage; ++j) {
      const int u = wave + j * n_waves;
      if (u < kUnits) {
        clear_tail(c * kBlocks + u / RT, d, lane, stage[j]);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          f32x4 sum = {};
#pragma unroll
          for (int t = 0; t < kSteps; ++t) {
            const u32x4 x = stage[j][g * kSteps + t];
            s_x[buf][u][g * kSteps + t][lane] = x;
            sum = mfma(x, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, sum);
          }
          if ((lane & 15) == 0) *reinterpret_cast<f32x4*>(&s_sum[(c * kBlocks + u / RT) & (kRing - 1)][u % RT][g][4 * (lane >> 4)]) = sum;
        }
      }
    }
  };
  Weights<S, kGroups> ring[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load_weights<S, kGroups, false>(q, tile, min(i, q.blocks - 1), lane, &ring[i]);
  fetch(0);
  put(0, 0);
  f32x4 total[RT][S] = {};
  const int padded = (q.blocks + kSteps - 1) / kSteps * kSteps, chunks = (padded + kBlocks - 1) / kBlocks;   // whole fours of groups
  uint32_t rec4[S] = {};                                 // of four groups, a quarter of the lanes each
  auto block = [&](int buf, int j, int b, Weights<S, kGroups>& W) {
    u32x4 w[S][4];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) w[s][ks] = codes_to_bf16(W.w[s][ks], bits);
    float scale[S][kGroups];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        scale[s][g] = rec_scale(W.rec[s][g]);
        rec4[s] = (lane >> 4) == ((b * kGroups + g) & 3) ? W.rec[s][g] : rec4[s];
      }
    // a row tile's operands are read while the tile in front of it is multiplied; the fence keeps the compiler from sinking each read to
    // its use, which leaves the latency of LDS open in front of every product
    u32x4 x[2][4];
    auto read = [&](int rt) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) x[rt & 1][ks] = s_x[buf][j * RT + rt][ks][lane];
    };
    read(0);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (rt + 1 < RT) read(rt + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        f32x4 acc[S] = {};
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
#pragma unroll
          for (int s = 0; s < S; ++s) acc[s] = mfma(x[rt & 1][g * kSteps + t], w[s][g * kSteps + t], acc[s]);
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e) total[rt][s][e] = fmaf(scale[s][g], acc[s][e], total[rt][s][e]);
      }
      // a row tile's sums are formed before the tile after the next one is read: left to itself the compiler reads first and multiplies
      // last, and spills
#pragma unroll
      for (int s = 0; s < S; ++s) asm volatile("" : "+v"(total[rt][s]));
    }
  };
  // The offsets of the last four groups, of block b and those in front of it, as one fp32 product with four terms per row tile and column tile.
  auto offsets = [&](int b) {
    float off[S];
#pragma unroll
    for (int s = 0; s < S; ++s) off[s] = -rec_scale(rec4[s]) * rec_zero(rec4[s]);
    const int from = b * kGroups + kGroups - 4 + (lane >> 4);   // the lane's group
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float sum = s_sum[from / kGroups & (kRing - 1)][rt][from % kGroups][lane & 15];
#pragma unroll
      for (int s = 0; s < S; ++s) total[rt][s] = __builtin_amdgcn_mfma_f32_16x16x4f32(sum, off[s], total[rt][s], 0, 0, 0);
    }
  };
  constexpr int kTurn = kAhead / kBlocks;                // chunks per trip: the ring's places and, if even, the buffers are constants
  static_assert(kAhead % kBlocks == 0 && (kAhead % kSteps == 0 || kSteps % kAhead == 0), "a chunk's blocks have places of their own in the ring");
  // chunks are padded to whole trips: past the last block the hidden rows are staged as zeros
  for (int c0 = 0; c0 < chunks; c0 += kTurn) {
#pragma unroll
    for (int cc = 0; cc < kTurn; ++cc) {
      const int c = c0 + cc, buf = kTurn % 2 == 0 ? cc & 1 : c & 1;
      __syncthreads();
      fetch(c + 1);
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        const int b = c * kBlocks + j;
        if (b < q.blocks) block(buf, j, b, ring[cc * kBlocks + j]);
        // loaded without a condition (a repeat past the end): the count of loads in flight is then known where the staged rows are waited for
        load_weights<S, kGroups, false>(q, tile, min(b + kAhead, q.blocks - 1), lane, &ring[cc * kBlocks + j]);
        if ((b + 1) % kSteps == 0) offsets(b);           // (past the last block the sums are 0)
      }
      put(c + 1, buf ^ 1);
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int v = (first + s) * 16 + (lane & 15);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = row0 + rt * 16 + 4 * (lane >> 4) + e;
        if (row < M && v < V_t) Z[(int64_t)row * ldz + v] = nan_if_infinite(total[rt][s][e]);
      }
    }
}

}  // namespace

hipError_t launch_pack_quant(const uint8_t* codes, const void* scales, int scale_f16, const uint8_t* zeros, int group, int d, int V_t, const QuantHead& q,
                             uint4* packed, uint32_t* recs, hipStream_t stream) {
  const int64_t n_codes = (int64_t)q.tiles * q.blocks * 64, n_recs = (int64_t)q.tiles * q.blocks * 16 * (4 / q.steps);
  hipLaunchKernelGGL(pack_codes_kernel, dim3((unsigned)((n_codes + 255) / 256)), dim3(256), 0, stream, codes, d, V_t, q.blocks, n_codes,
                     reinterpret_cast<u32x4*>(packed));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pack_scales_kernel, dim3((unsigned)((n_recs + 255) / 256)), dim3(256), 0, stream, scales, scale_f16, zeros, ceil_div(d, group), V_t,
                     q.blocks, 4 / q.steps, n_recs, recs);
  return hipGetLastError();
}

namespace {

constexpr int kChunkBlocks = 38;      // blocks of 16 hidden rows in LDS at most: 4 KB each

template <int S, int kSteps>
hipError_t launch_rows16(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int columns, int parts, hipStream_t stream) {
  constexpr int kAhead = S == 1 ? 8 : S == 2 ? 4 : S == 3 ? 3 : 2;
  const int chunks = ceil_div(q.blocks, kChunkBlocks), chunk_blocks = ceil_div(q.blocks, chunks), waves = columns * parts;
  const size_t lds = (size_t)1024 * std::max(4 * chunk_blocks, parts > 1 ? waves * S : 0);
  hipLaunchKernelGGL((qhead_rows16_kernel<S, kSteps, kAhead>), dim3((unsigned)ceil_div(q.tiles, columns * S)), dim3(64 * waves), lds, stream, H, M, d, q, Z,
                     V_t, ldz, chunk_blocks, parts);
  return hipGetLastError();
}

// One workgroup per compute unit and round, of 16 wavefronts: its column tiles, up to four per wavefront, side by side, and where they are
// fewer than the wavefronts, as many parts of the hidden dimension as there are wavefronts for.  Without the parts 6 rows x 152064 take 55.9
// us instead of 54.3, the rest is the same within 2 % (with 8 wavefronts of twice the tiles 57.3): the loads in flight are enough.
template <int kSteps>
hipError_t launch_up_to_16(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int n_cu, hipStream_t stream) {
  const int rounds = ceil_div(q.tiles, 64 * n_cu), per_cu = ceil_div(q.tiles, rounds * n_cu);
  const int S = ceil_div(per_cu, 16), columns = ceil_div(per_cu, S), parts = std::max(1, std::min(16 / columns, q.blocks));
  switch (S) {
    case 1: return launch_rows16<1, kSteps>(H, M, d, q, Z, V_t, ldz, columns, parts, stream);
    case 2: return launch_rows16<2, kSteps>(H, M, d, q, Z, V_t, ldz, columns, parts, stream);
    case 3: return launch_rows16<3, kSteps>(H, M, d, q, Z, V_t, ldz, columns, parts, stream);
    default: return launch_rows16<4, kSteps>(H, M, d, q, Z, V_t, ldz, columns, parts, stream);
  }
}

// Weights four blocks ahead, two where the registers do not hold four.
template <int RT, int S, int kSteps>
hipError_t launch_tall(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int m_blocks, int waves, hipStream_t stream) {
  constexpr int kAhead = S <= 2 && (kSteps == 4 || RT <= 4) ? 4 : 2;
  const int64_t grid = (int64_t)ceil_div(ceil_div(q.tiles, waves * S), 8) * 8 * m_blocks;
  if (!grid_fits(grid, 64 * waves)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((qhead_tall_kernel<RT, S, kSteps, kAhead>), dim3((unsigned)grid), dim3(64 * waves), 0, stream, H, M, d, q, Z, V_t, ldz, m_blocks);
  return hipGetLastError();
}

// Blocks of at most nine row tiles (a tenth would not fit the registers beside two column tiles).  Of the column tiles S per wavefront and the
// 8 to 6 wavefronts per workgroup, those whose rounds of the chip take least: a round lasts as long as a workgroup has column tiles, and a
// column tile costs 6 : 7 : 8 at four, two and one per wavefront, which share what is read from LDS.  Measured, us, groups of 128:
//   rows x 128256, d = 4096   4 tiles  2      1              rows x 152064, d = 4096   chosen        least rounds alone   8 wavefronts alone
//   24                        62.7     74.6   74.9           24                        86.1 (2 x 7)  88.4                 90.0
//   48                        75.4     86.9   98.0           80                        155           175                  175
//   80                        100.8    118.8  145.8          144                       224           267                  267
//   144 (nine row tiles)      -        172    219
// and 24 rows x 32003, d = 2056: one tile 14.5, two 18.2 (half of the compute units idle).  Four tiles fit the registers with one scale
// per block of 128 and up to five row tiles.
template <int kSteps>
hipError_t launch_above_16(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int n_cu, hipStream_t stream) {
  const int m_blocks = ceil_div(M, 9 * 16), RT = ceil_div(M, 16 * m_blocks);
  const int most = kSteps == 4 && RT <= 5 ? 4 : 2;
  int S = 1, waves = 8;
  int64_t best = INT64_MAX;
  for (int s = 1; s <= most; s *= 2)
    for (int w = 8; w >= 6; --w) {
      const int64_t cost = (int64_t)ceil_div((int64_t)ceil_div(q.tiles, s * w) * m_blocks, n_cu) * s * w * (s == 4 ? 6 : s == 2 ? 7 : 8);
      if (cost < best || (cost == best && s > S)) { best = cost; S = s; waves = w; }
    }
#define OT_TALL(rt, s) if (RT == rt && S == s) return launch_tall<rt, s, kSteps>(H, M, d, q, Z, V_t, ldz, m_blocks, waves, stream)
  if constexpr (kSteps == 4) { OT_TALL(2, 4); OT_TALL(3, 4); OT_TALL(4, 4); OT_TALL(5, 4); }
  OT_TALL(2, 1); OT_TALL(2, 2); OT_TALL(3, 1); OT_TALL(3, 2); OT_TALL(4, 1); OT_TALL(4, 2); OT_TALL(5, 1); OT_TALL(5, 2);
  OT_TALL(6, 1); OT_TALL(6, 2); OT_TALL(7, 1); OT_TALL(7, 2); OT_TALL(8, 1); OT_TALL(8, 2); OT_TALL(9, 1); OT_TALL(9, 2);
#undef OT_TALL
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_qhead(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int n_cu, hipStream_t stream) {
  if (M == 0) return hipSuccess;
  if (q.steps == 4) return M <= 16 ? launch_up_to_16<4>(H, M, d, q, Z, V_t, ldz, n_cu, stream) : launch_above_16<4>(H, M, d, q, Z, V_t, ldz, n_cu, stream);
  if (q.steps == 2) return M <= 16 ? launch_up_to_16<2>(H, M, d, q, Z, V_t, ldz, n_cu, stream) : launch_above_16<2>(H, M, d, q, Z, V_t, ldz, n_cu, stream);
  return M <= 16 ? launch_up_to_16<1>(H, M, d, q, Z, V_t, ldz, n_cu, stream) : launch_above_16<1>(H, M, d, q, Z, V_t, ldz, n_cu, stream);
}

}  // namespace otv
