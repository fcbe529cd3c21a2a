// A target head of 4-bit weights with group scales: z[m][v] = sum over groups g of s[g][v] * sum_{k in g} h[m][k] (c[k][v] - zp[g][v]).
//
// The codes c (0..15) become bf16 operands of v_mfma_f32_16x16x32_bf16 in two instructions per pair and none of them a
// conversion: the bits 0x4180 | c << 3 are the bf16 number 16 + c, exactly.  So a group's product comes out as
// sum h (16 + c), and the sum of the group's hidden states, the same for every column, takes (16 + zp) times itself off it;
// then the group's scale multiplies 16 rows x 16 columns in four instructions.  Products of a bf16 number and 16 + c are exact in
// fp32, so what is rounded is the sums alone; they are at most 31 / |c - zp| times as large as with the centred codes, which
// costs less than the fp32 rounding of a group's scaled sum in the total over the groups.
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

// Eight codes of one packed word as bf16 numbers 16 + c, in ascending hidden index.  The word is the one whose nibble j holds code 2 j
// and whose nibble j + 4 code 2 j + 1 (j < 4), rotated left by 3: a pair's mantissa bits are then a shift and a mask away.
__device__ inline u32x4 codes_to_bf16(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
  return u32x4{(w & kMask) | kSixteen, (w >> 4 & kMask) | kSixteen, (w >> 8 & kMask) | kSixteen,
               (__builtin_amdgcn_alignbit(w, w, 12) & kMask) | kSixteen};
}
// A group's scale and 16 + zero point of one column: the scale's fp32 bits, of which a bf16 or fp16 scale leaves the low 13 free.
__device__ inline float rec_scale(uint32_t r) { return __uint_as_float(r & 0xFFFFE000u); }
__device__ inline float rec_zero(uint32_t r) { return (float)(r & 0xFFu); }

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
    for (int j = 0; j < 4; ++j) {
      const int k = b * 128 + ks * 32 + (lane >> 4) * 8 + 2 * j;         // even, as is d
      const uint32_t both = k < d && v < V_t ? codes[(int64_t)(k >> 1) * V_t + v] : 0u;
      x |= (both & 15u) << (4 * j) | (both >> 4) << (4 * j + 16);
    }
    w[ks] = x << 3 | x >> 29;
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
  uint32_t r = 16;
  if (g < groups && v < V_t) {
    const int64_t at = (int64_t)g * V_t + v;
    const float s = f16 ? (float)static_cast<const _Float16*>(scales)[at] : bf16_to_f32(static_cast<const uint16_t*>(scales)[at]);
    r = (__float_as_uint(s) & 0xFFFFE000u) | (16u + (zeros ? zeros[at] & 15u : 8u));
  }
  recs[i] = r;
}

// One wavefront per 16 columns and 16 rows.
template <int kSteps>
__global__ __launch_bounds__(256) void qhead_kernel(const uint16_t* __restrict__ H, int M, int d, QuantHead q, float* __restrict__ Z, int V_t, int64_t ldz) {
  constexpr int kGroups = 4 / kSteps;
  const int lane = threadIdx.x & 63, tile = blockIdx.x * 4 + uniform((int)threadIdx.x >> 6), row0 = blockIdx.y * 16;
  if (tile >= q.tiles) return;
  const uint16_t* h = H + (int64_t)min(row0 + (lane & 15), M - 1) * d;
  const u32x4* codes = reinterpret_cast<const u32x4*>(q.codes) + (int64_t)tile * q.blocks * 64 + lane;
  const uint32_t* recs = q.recs + (int64_t)tile * q.blocks * 16 * kGroups + (lane & 15) * kGroups;
  f32x4 total = {};
  for (int b = 0; b < q.blocks; ++b) {
    const u32x4 w = codes[(int64_t)b * 64];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint32_t rec = recs[(int64_t)b * 16 * kGroups + g];
      f32x4 acc = {}, sum = {};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int ks = g * kSteps + s, k = b * 128 + ks * 32 + (lane >> 4) * 8;
        const u32x4 x = k < d ? *reinterpret_cast<const u32x4*>(h + k) : u32x4{};
        acc = mfma(x, codes_to_bf16(w[ks]), acc);
        sum = mfma(x, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, sum);
      }
      const float s = rec_scale(rec), zero = rec_zero(rec);
#pragma unroll
      for (int i = 0; i < 4; ++i) total[i] = fmaf(s, fmaf(-zero, sum[i], acc[i]), total[i]);
    }
  }
  const int v = tile * 16 + (lane & 15);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 4 * (lane >> 4) + i;
    if (row < M && v < V_t) Z[(int64_t)row * ldz + v] = total[i];
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

hipError_t launch_qhead(const uint16_t* H, int M, int d, const QuantHead& q, float* Z, int V_t, int64_t ldz, int n_cu, hipStream_t stream) {
  (void)n_cu;
  if (M == 0) return hipSuccess;
  const dim3 grid((unsigned)ceil_div(q.tiles, 4), (unsigned)ceil_div(M, 16)), block(256);
  if (grid.y > 65535) return hipErrorInvalidValue;
  const auto kernel = q.steps == 4 ? qhead_kernel<4> : q.steps == 2 ? qhead_kernel<2> : qhead_kernel<1>;
  hipLaunchKernelGGL(kernel, grid, block, 0, stream, H, M, d, q, Z, V_t, ldz);
  return hipGetLastError();
}

}  // namespace otv
