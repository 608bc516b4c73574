// Rows of keys and values into a paged cache and out of it.
//
// A lane holds 8 elements of a head (16 bytes of a 16-bit type), so a block of
// 32, which shares a scale, is four neighbouring lanes: its largest magnitude
// takes two exchanges within quads of lanes.  A wavefront takes one row, or
// several where a row's keys have fewer than 64 such units; keys and values of
// a head go together.
//
// Bound: memory, each element read once and written once (30 778 rows of 8 heads x
// 128: into e2m1 34 us, back to bf16 30, 4.7 and 5.3 TB/s; 66 246 rows out of e4m3
// 83 us, 4.9; the VALU busy 58, 58 and 36 % of the time).  With an address of its own
// for every unit, not a step from head to head, it was issue: 40, 34 and 98 us.
#include "serve.h"

#include <algorithm>

namespace pard {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int kSeqsInLds = 1024;

struct Row8 { float v[8]; };

template <class E, bool VEC>
__device__ __forceinline__ Row8 load8(const char* row, int64_t at) {
  const typename E::T* p = reinterpret_cast<const typename E::T*>(row) + at;
  Row8 r;
  if constexpr (VEC) {
    if constexpr (sizeof(typename E::T) == 4) {
      const u32x4 a = reinterpret_cast<const u32x4*>(p)[0], b = reinterpret_cast<const u32x4*>(p)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[i] = __uint_as_float(a[i]), r.v[4 + i] = __uint_as_float(b[i]);
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) r.v[i] = E::load((uint16_t)(a[i >> 1] >> (16 * (i & 1))));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = E::load(p[i]);
  }
  return r;
}

template <class E>
__device__ __forceinline__ u32x4 pack8(const Row8& r) {
  u32x4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = (uint32_t)E::store(r.v[2 * i]) | (uint32_t)E::store(r.v[2 * i + 1]) << 16;
  return a;
}

template <class E, bool VEC>
__device__ __forceinline__ void store8(char* row, int64_t at, const Row8& r) {
  typename E::T* p = reinterpret_cast<typename E::T*>(row) + at;
  if constexpr (VEC) {
    if constexpr (sizeof(typename E::T) == 4) {
      u32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(r.v[i]), b[i] = __float_as_uint(r.v[4 + i]);
      reinterpret_cast<u32x4*>(p)[0] = a;
      reinterpret_cast<u32x4*>(p)[1] = b;
    } else {
      *reinterpret_cast<u32x4*>(p) = pack8<E>(r);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = E::store(r.v[i]);
  }
}

// The scale byte of a block with this largest magnitude (as bits, which are in
// the order of the floats): e + 127 of the smallest 2^e, e >= -126, that brings
// it within the type's range, 1.75 2^8 or 1.5 2^2.  A fraction above .75 or .5
// carries into the exponent.  255: the block is NaN.
template <int DT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
  constexpr uint32_t kCarry = DT == PARD_E4M3 ? 0x1fffffu : 0x3fffffu;
  constexpr int kTop = DT == PARD_E4M3 ? 8 : 2;
  if (largest >= 0x7f800000u) return 255;
  return (uint32_t)max((int)((largest + kCarry) >> 23) - kTop, 1);
}

// 8 elements into the cache; the four lanes of a block hold it together.
template <int DT>
__device__ __forceinline__ void put(Row8 r, char* held, uint8_t* scale, bool first) {
  if constexpr (DT == PARD_BF16) {
    *reinterpret_cast<u32x4*>(held) = pack8<ElemBF16>(r);
  } else if constexpr (DT == PARD_F16) {
    *reinterpret_cast<u32x4*>(held) = pack8<ElemF16>(r);
  } else {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(r.v[i]) & 0x7fffffffu);
    big = max(big, (uint32_t)__builtin_amdgcn_mov_dpp((int)big, 0xB1, 0xF, 0xF, false));   // quad_perm 1 0 3 2
    big = max(big, (uint32_t)__builtin_amdgcn_mov_dpp((int)big, 0x4E, 0xF, 0xF, false));   // quad_perm 2 3 0 1
    const uint32_t byte = scale_byte<DT>(big);
    if (first) *scale = (uint8_t)byte;
    if constexpr (DT == PARD_E4M3) {
      const float inv = __uint_as_float((254 - min(byte, 253u)) << 23);    // 2^-e: products with it are exact
      u32x2 w = {0, 0};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(r.v[4 * i] * inv, r.v[4 * i + 1] * inv, 0, false);
        x = __builtin_amdgcn_cvt_pk_fp8_f32(r.v[4 * i + 2] * inv, r.v[4 * i + 3] * inv, x, true);
        w[i] = (uint32_t)x;
      }
      *reinterpret_cast<u32x2*>(held) = w;
    } else {
      const float f = __uint_as_float(byte << 23);                         // (the conversion divides by it)
      uint32_t w = 0;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r.v[0], r.v[1], f, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r.v[2], r.v[3], f, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r.v[4], r.v[5], f, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, r.v[6], r.v[7], f, 3);
      *reinterpret_cast<uint32_t*>(held) = w;
    }
  }
}

// 8 elements of the cache as floats (a scale byte of 0 is 2^-127, 255 NaN: the
// conversions know both).
template <int DT>
__device__ __forceinline__ Row8 get(const char* held, const uint8_t* scale) {
  Row8 r;
  if constexpr (DT == PARD_E4M3) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(held);
    const float f = __uint_as_float((uint32_t)*scale << 23);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], f, true);
      r.v[4 * i] = lo[0], r.v[4 * i + 1] = lo[1], r.v[4 * i + 2] = hi[0], r.v[4 * i + 3] = hi[1];
    }
  } else if constexpr (DT == PARD_E2M1) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(held);
    const float f = __uint_as_float((uint32_t)*scale << 23);
    const f32x2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 1);
    const f32x2 x2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 3);
    r = Row8{{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]}};
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4*>(held);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint16_t h = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
      r.v[i] = DT == PARD_BF16 ? ElemBF16::load(h) : ElemF16::load(h);
    }
  }
  return r;
}

template <int HD, class E, int DT, bool VEC, bool WRITE>
__global__ __launch_bounds__(256) void k_kv_copy(const KvCopyArgs a) {
  constexpr int HU = HD / 8;                          // units of a head
  constexpr int RB = kv_row_bytes(DT, HD), SB = kv_scale_bytes(DT, HD);
  __shared__ int starts[kSeqsInLds + 1];
  const KvBatchView& b = a.batch;
  const bool in_lds = b.n_seqs <= kSeqsInLds;
  if (in_lds) {
    for (int i = threadIdx.x; i <= b.n_seqs; i += 256) starts[i] = b.row_start[i];
    __syncthreads();
  }
  // lanes of a row (of whole heads), rows of a wavefront; a lane keeps to its
  // place in a head, and goes from head to head
  const int lane = threadIdx.x & 63, units = a.cache.n_kv * HU;
  const int per_row = min(units, 64), per_wave = 64 / per_row;
  const int wave = blockIdx.x * 4 + (threadIdx.x >> 6), n_waves = gridDim.x * 4;
  const int sub = lane / per_row, u0 = lane - sub * per_row;
  if (sub >= per_wave) return;
  const int unit = u0 % HU, head0 = u0 / HU, heads = per_row / HU;
  const int64_t next = (int64_t)heads << a.cache.page_log2;               // slots
  for (int64_t r64 = (int64_t)wave * per_wave + sub; r64 < b.rows; r64 += (int64_t)n_waves * per_wave) {
    const int row = (int)r64;
    const int s = in_lds ? kv_seq_of(starts, b.n_seqs, row) : kv_seq_of(b.row_start, b.n_seqs, row);
    if (s >= b.n_seqs) continue;                      // (a row of no sequence)
    const int first = in_lds ? starts[s] : b.row_start[s], end = in_lds ? starts[s + 1] : b.row_start[s + 1];
    if (row < first) continue;
    const int pos = b.kv_len[s] - end + row;
    const int page = pos < 0 ? -1 : kv_page(a.cache, b, s, pos);
    if (WRITE && page < 0) continue;
    const int64_t slot = (((int64_t)max(page, 0) * a.cache.n_kv + head0) << a.cache.page_log2) + (pos & ((1 << a.cache.page_log2) - 1));
    char *kh = a.cache.k + slot * RB + unit * (RB / HU), *vh = a.cache.v + slot * RB + unit * (RB / HU);
    uint8_t *ks = SB ? a.cache.k_scale + slot * SB + unit / 4 : nullptr, *vs = SB ? a.cache.v_scale + slot * SB + unit / 4 : nullptr;
    int64_t ka = row * a.k.rs + head0 * a.k.hs + unit * 8, va = row * a.v.rs + head0 * a.v.hs + unit * 8;
    for (int u = u0; u < units; u += per_row) {
      if constexpr (WRITE) {
        const Row8 k = load8<E, VEC>(a.k.data, ka), v = load8<E, VEC>(a.v.data, va);
        put<DT>(k, kh, ks, unit % 4 == 0);
        put<DT>(v, vh, vs, unit % 4 == 0);
      } else {
        Row8 k, v;
        if (page >= 0) {
          k = get<DT>(kh, ks);
          v = get<DT>(vh, vs);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) k.v[i] = v.v[i] = __uint_as_float(0x7fc00000u);
        }
        store8<E, VEC>(a.k.data, ka, k);
        store8<E, VEC>(a.v.data, va, v);
      }
      kh += next * RB;
      vh += next * RB;
      if (SB) ks += next * SB, vs += next * SB;
      ka += heads * a.k.hs;
      va += heads * a.v.hs;
    }
  }
}

template <int HD, class E, int DT, bool VEC>
hipError_t launch_dir(bool write, const KvCopyArgs& a, hipStream_t st) {
  const int units = a.cache.n_kv * (HD / 8), per_wave = 64 / std::min(units, 64);
  const int64_t waves = ((int64_t)a.batch.rows + per_wave - 1) / per_wave;
  const unsigned grid = (unsigned)std::min<int64_t>((waves + 3) / 4, 1 << 16);
  if (write) k_kv_copy<HD, E, DT, VEC, true><<<grid, 256, 0, st>>>(a);
  else k_kv_copy<HD, E, DT, VEC, false><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int HD, class E, bool VEC>
hipError_t launch_type(bool write, int cache_dtype, const KvCopyArgs& a, hipStream_t st) {
  switch (cache_dtype) {
    case PARD_BF16: return launch_dir<HD, E, PARD_BF16, VEC>(write, a, st);
    case PARD_F16: return launch_dir<HD, E, PARD_F16, VEC>(write, a, st);
    case PARD_E4M3: return launch_dir<HD, E, PARD_E4M3, VEC>(write, a, st);
    default: return launch_dir<HD, E, PARD_E2M1, VEC>(write, a, st);
  }
}

template <int HD, bool VEC>
hipError_t launch_rows(bool write, int dtype, int cache_dtype, const KvCopyArgs& a, hipStream_t st) {
  if (dtype == PARD_F32) return launch_type<HD, ElemF32, VEC>(write, cache_dtype, a, st);
  if (dtype == PARD_BF16) return launch_type<HD, ElemBF16, VEC>(write, cache_dtype, a, st);
  return launch_type<HD, ElemF16, VEC>(write, cache_dtype, a, st);
}

}  // namespace

hipError_t launch_kv_copy(bool write, int head_dim, int dtype, int cache_dtype, bool vec, const KvCopyArgs& a,
                          hipStream_t st) {
  if (head_dim == 64)
    return vec ? launch_rows<64, true>(write, dtype, cache_dtype, a, st) : launch_rows<64, false>(write, dtype, cache_dtype, a, st);
  return vec ? launch_rows<128, true>(write, dtype, cache_dtype, a, st) : launch_rows<128, false>(write, dtype, cache_dtype, a, st);
}

}  // namespace pard
