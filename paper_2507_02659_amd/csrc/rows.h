// Rows of logits as the kernels beside the step read and write them: bfloat16 or float32, from any element on, in 16-byte vectors.
#pragma once

#include "device_math.h"

namespace otv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNan = __builtin_nanf("");

// Temperature of a row, of which log2(e) / T is finite and above 0 (else a masked id's distance of -inf gave NaN): one per row, or per sequence
// of row_off.  By a whole wavefront.
__device__ inline float row_temperature(const float* temperature, const int32_t* row_off, int B, int row, int lane) {
  if (!temperature) return 1.f;
  const float T = temperature[row_off ? find_sequence(row_off, B, row, 0, lane) : row];
  return T > 0.f ? fminf(fmaxf(T, 0x1p-126f), 0x1.fffffep127f) : 1.f;
}

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

// A vector of these values, as the row's type rounds them.
__device__ inline Vec<float>::Raw pack_vec(const float (&v)[4]) { return {v[0], v[1], v[2], v[3]}; }
__device__ inline Vec<uint16_t>::Raw pack_vec(const float (&v)[8]) {
  Vec<uint16_t>::Raw r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * i], v[2 * i + 1]}, bf16x2));
  return r;
}

// The elements of a vector whose bit is clear become -inf.
__device__ inline void mask_vector(Vec<float>::Raw* x, uint32_t allowed) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)allowed, e, 1);
    (*x)[e] = __uint_as_float((__float_as_uint((*x)[e]) & keep) | (0xFF800000u & ~keep));
  }
}
__device__ inline void mask_vector(Vec<uint16_t>::Raw* x, uint32_t allowed) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t low = (uint32_t)__builtin_amdgcn_sbfe((int)allowed, 2 * e, 1), high = (uint32_t)__builtin_amdgcn_sbfe((int)allowed, 2 * e + 1, 1);
    const uint32_t keep = (low & 0xFFFFu) | (high & 0xFFFF0000u);
    (*x)[e] = ((*x)[e] & keep) | (0xFF80FF80u & ~keep);
  }
}

// A row's elements as whole vectors from the first 16-byte boundary on, and those in front of it and behind the last whole one (fewer than
// two vectors' worth), which go one by one.
template <typename T>
struct RowSplit {
  int head, vecs, tail;
  __device__ RowSplit(const T* row, int n) {
    constexpr int kVec = Vec<T>::kElems;
    head = min(n, (int)((kVec - ((reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (kVec - 1))) & (kVec - 1)));
    vecs = (n - head) / kVec;
    tail = n - head - vecs * kVec;
  }
  __device__ int edge(int i) const { return i < head ? i : head + vecs * Vec<T>::kElems + i - head; }   // element of the i-th single one
};

}  // namespace otv
