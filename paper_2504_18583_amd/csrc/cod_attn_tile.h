// Tiles of attention over packed COD rows: MFMA operands of the stored types,
// and 16-row blocks in LDS.
//
// A block of 16 rows x HD elements lies in LDS as HD/16 squares of 16 rows x 16
// elements, 512 bytes each, row by row.  From it come both operand forms of the
// 16x16x32 MFMAs without bank conflicts:
//   rows    lane l holds row l % 16, elements 32 s + 8 (l / 16) .. + 7: one
//           16-byte read, the wavefront's lanes covering two squares
//   columns lane l holds column 16 b + l % 16 of rows 4 (l / 16) .. + 3 of one
//           block and of the next: two transposing reads, lane-linear
// The accumulator of a product with rows as A operand (lane l: column l % 16,
// rows 4 (l / 16) .. + 3) is, packed to 16 bits, the B operand of a product
// with columns as A: scores turn into probabilities in place.
#pragma once

#include "train.h"

namespace pard {
namespace cod {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct MmaBF16 {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, v2));
  }
  static __device__ __forceinline__ f32x2 unpack(uint32_t v) {
    return f32x2{__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)};
  }
};
struct MmaF16 {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, v2));
  }
  static __device__ __forceinline__ f32x2 unpack(uint32_t v) {
    const v2 h = __builtin_bit_cast(v2, v);
    return f32x2{(float)h[0], (float)h[1]};
  }
};

// LDS of one block of 16 rows, in 16-byte units.
template <int HD>
constexpr int kBlockUnits = HD / 16 * 32;

// A lane's part of a block: its row, and its byte offset in every 64 bytes of
// the row.
__device__ __forceinline__ int block_row(int lane) { return (lane & 31) >> 1; }
__device__ __forceinline__ int block_byte(int lane) { return (lane >> 5) * 32 + (lane & 1) * 16; }

// One block into LDS (LDS-DMA loads: complete at vmcnt 0); src: this lane's
// row + block_byte.
template <int HD>
__device__ __forceinline__ void load_block(const char* src, u32x4* block) {
#pragma unroll
  for (int j = 0; j < HD / 32; ++j)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + j * 64),
                                     (__attribute__((address_space(3))) void*)(block + j * 64), 16, 0, 0);
}

// Rows operand, elements 32 s ..
__device__ __forceinline__ u32x4 rows_frag(const u32x4* block, int s, int lane) {
  const int c16 = lane & 15, g4 = lane >> 4;
  return block[(2 * s + (g4 >> 1)) * 32 + c16 * 2 + (g4 & 1)];
}

// Columns operand 16 b .. of the rows of two blocks.
template <int HD>
__device__ __forceinline__ u32x4 cols_frag(const u32x4* blocks, int b, int lane) {
  typedef __attribute__((address_space(3))) s16x4* lds4;
  const u32x2* p = reinterpret_cast<const u32x2*>(blocks + b * 32) + lane;
  const u32x2* q = reinterpret_cast<const u32x2*>(blocks + kBlockUnits<HD> + b * 32) + lane;
  const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p));
  const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q));
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// Across the lanes l, l ^ 16, l ^ 32, l ^ 48 (lane swaps in the VALU).
__device__ __forceinline__ f32x2 swap16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ f32x2 swap32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float max4g(float x) {
  f32x2 r = swap16(x);
  x = fmaxf(r[0], r[1]);
  r = swap32(x);
  return fmaxf(r[0], r[1]);
}
__device__ __forceinline__ float sum4g(float x) {
  f32x2 r = swap16(x);
  x = r[0] + r[1];
  r = swap32(x);
  return r[0] + r[1];
}

// Scale of scores in base 2, and the sign bits that queries take over from a
// negative scale (an exact negation).  A zero scale becomes one that scores
// vanish under, so that hidden scores can be -infinity before the product.
__device__ __forceinline__ float base2_scale(float scale) { return fmaxf(fabsf(scale) * kLog2e, 1e-30f); }
__device__ __forceinline__ uint32_t scale_sign(float scale) { return scale < 0.f ? 0x80008000u : 0u; }

__device__ __forceinline__ char* at(const Heads16& h, uint32_t row, uint32_t head) {
  return h.data + (uint64_t)head * h.hs + (uint64_t)row * h.rs;
}
__device__ __forceinline__ int quotient(int x, const FastDiv& f) { return (int)(__umulhi((uint32_t)x << 2, f.m) >> f.l); }
__device__ __forceinline__ int remainder(int x, int q, const FastDiv& f) { return x - q * (int)f.d; }

// Everything this wavefront loaded is in LDS and its LDS reads are done; then
// everyone's.
__device__ __forceinline__ void wait_all() {
  __builtin_amdgcn_s_waitcnt(0x0070);              // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_and_meet() {
  wait_all();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace cod
}  // namespace pard
