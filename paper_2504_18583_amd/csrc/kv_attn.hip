// Attention of a batch's new rows over a paged cache.
//
// One wavefront per (row, query head): a lane holds HD / 64 elements, keys
// follow one another, the softmax is one pass with a running maximum.
#include "serve.h"

namespace pard {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <class E, int DT>
__device__ __forceinline__ float element(const char* head, const uint8_t* scale, int i) {
  if constexpr (DT == PARD_E4M3 || DT == PARD_E2M1) {
    const uint32_t byte = scale[i / kKvBlock];
    const float f = __uint_as_float(byte == 0 ? 0x400000u : byte == 255 ? 0x7fc00000u : byte << 23);
    float x;
    if constexpr (DT == PARD_E4M3) {
      x = __builtin_amdgcn_cvt_f32_fp8((uint8_t)head[i], 0);
    } else {
      const uint32_t w = (uint8_t)head[i / 2];
      x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0)[i & 1];
    }
    return E::load(E::store(x * f));
  } else {
    return E::load(reinterpret_cast<const uint16_t*>(head)[i]);
  }
}

template <int HD, class E, int DT>
__global__ __launch_bounds__(256) void k_kv_attn(const KvAttnArgs a) {
  constexpr int PER = HD / 64, RB = kv_row_bytes(DT, HD), SB = kv_scale_bytes(DT, HD);
  const KvBatchView& b = a.batch;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(w / a.n_heads), head = (int)(w % a.n_heads), kvh = head / a.group;
  if (row >= b.rows) return;
  const int s = kv_seq_of(b.row_start, b.n_seqs, row);
  if (s >= b.n_seqs || row < b.row_start[s]) return;
  const int pos = b.kv_len[s] - b.row_start[s + 1] + row;
  const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q.data + (uint64_t)row * a.q.rs + (uint64_t)head * a.q.hs);
  float x[PER], o[PER] = {}, m = -1e30f, l = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = E::load(q[lane * PER + i]);
  bool bad = pos >= b.cap;
  const int low = a.window ? max(pos - a.window + 1, 0) : 0, last = min(pos, b.cap - 1);
  for (int j = 0; j <= last; ++j) {
    if (j < low && j >= a.sinks) j = low;
    const int page = kv_page(a.cache, b, s, j);
    if (page < 0) {
      bad = true;
      continue;
    }
    const int64_t slot = (((int64_t)page * a.cache.n_kv + kvh) << a.cache.page_log2) + (j & ((1 << a.cache.page_log2) - 1));
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) dot += x[i] * element<E, DT>(a.cache.k + slot * RB, a.cache.k_scale + slot * SB, lane * PER + i);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) dot += __shfl_xor(dot, d);
    const float sc = dot * a.scale * kLog2e, m_new = fmaxf(m, sc);
    const float corr = __builtin_amdgcn_exp2f(m - m_new), p = __builtin_amdgcn_exp2f(sc - m_new);
    m = m_new;
    l = l * corr + p;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      o[i] = o[i] * corr + p * element<E, DT>(a.cache.v + slot * RB, a.cache.v_scale + slot * SB, lane * PER + i);
  }
  uint16_t* out = reinterpret_cast<uint16_t*>(a.out.data + (uint64_t)row * a.out.rs + (uint64_t)head * a.out.hs);
  const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int i = 0; i < PER; ++i) out[lane * PER + i] = E::store(bad ? nan : l == 0.f ? 0.f : o[i] / l);
  if (a.lse && lane == 0) a.lse[(int64_t)head * b.rows + row] = bad ? nan : l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int HD, class E, int DT>
hipError_t launch_cache(const KvAttnArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.batch.rows * a.n_heads;
  k_kv_attn<HD, E, DT><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int HD, class E, int SAME>
hipError_t launch_hd(int cache_dtype, const KvAttnArgs& a, hipStream_t st) {
  if (cache_dtype == PARD_E4M3) return launch_cache<HD, E, PARD_E4M3>(a, st);
  if (cache_dtype == PARD_E2M1) return launch_cache<HD, E, PARD_E2M1>(a, st);
  return launch_cache<HD, E, SAME>(a, st);
}

}  // namespace

size_t kv_attn_workspace(const KvAttnArgs&, int) { return 256; }

hipError_t launch_kv_attn(int head_dim, int dtype, int cache_dtype, const KvAttnArgs& a, int, hipStream_t st) {
  if (head_dim == 64)
    return dtype == PARD_BF16 ? launch_hd<64, ElemBF16, PARD_BF16>(cache_dtype, a, st) : launch_hd<64, ElemF16, PARD_F16>(cache_dtype, a, st);
  return dtype == PARD_BF16 ? launch_hd<128, ElemBF16, PARD_BF16>(cache_dtype, a, st) : launch_hd<128, ElemF16, PARD_F16>(cache_dtype, a, st);
}

}  // namespace pard
