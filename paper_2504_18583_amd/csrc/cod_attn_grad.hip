// Gradient of attention over packed COD rows.
#include "train.h"

namespace pard {
namespace {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

template <class E>
__device__ __forceinline__ const typename E::T* at(const Heads& h, int64_t row, int head) {
  return reinterpret_cast<const typename E::T*>(h.data) + row * h.rs + head * h.hs;
}
template <class E>
__device__ __forceinline__ typename E::T* at_out(const Heads& h, int64_t row, int head) {
  return reinterpret_cast<typename E::T*>(h.data) + row * h.rs + head * h.hs;
}

template <int HD, class E>
__device__ __forceinline__ float dot(const typename E::T* a, const typename E::T* b) {
  float s = 0.f;
  for (int d = 0; d < HD; ++d) s += E::load(a[d]) * E::load(b[d]);
  return s;
}

// Calls f(row) for this lane's share of the rows that order entry m (at
// position p) attends to.
template <class F>
__device__ __forceinline__ void keys_of(const CodPlanView& v, int off, int4 m, int p, F&& f) {
  const int lane = threadIdx.x;
  for (int t = lane; t < m.y; t += 64) f(t);
  for (int b = m.z + lane; b <= p && b < m.w; b += 64) f(v.order[off + b].x);
}

template <int HD, class E>
__global__ __launch_bounds__(64) void k_dq(const CodAttnArgs a) {
  const int2 tile = a.plan.tiles[blockIdx.x / kCodTile];
  const CodSampleInfo s = a.plan.samples[tile.x];
  const int p = tile.y * kCodTile + blockIdx.x % kCodTile, h = blockIdx.y;
  if (p >= s.cap) return;
  const int4 m = a.plan.order[s.off + p];
  const int64_t row = s.off + m.x;
  const int kvh = h / a.group;
  float acc[HD];
  for (int d = 0; d < HD; ++d) acc[d] = 0.f;
  if (p < s.len) {
    const auto* q = at<E>(a.q, row, h);
    const auto* go = at<E>(a.d_out, row, h);
    const float delta = dot<HD, E>(go, at<E>(a.out, row, h)), lse = a.lse[h * a.rows + row];
    if (threadIdx.x == 0) a.delta[h * a.rows + row] = delta;
    keys_of(a.plan, s.off, m, p, [&](int key) {
      const auto* k = at<E>(a.k, s.off + key, kvh);
      const float w = expf(a.scale * dot<HD, E>(q, k) - lse);
      const float ds = w * (dot<HD, E>(go, at<E>(a.v, s.off + key, kvh)) - delta) * a.scale;
      for (int d = 0; d < HD; ++d) acc[d] += ds * E::load(k[d]);
    });
  }
  for (int d = 0; d < HD; ++d) {
    const float o = wave_sum(acc[d]);
    if (threadIdx.x == 0) at_out<E>(a.dq, row, h)[d] = E::store(o);
  }
}

// One wavefront per (order position, key head): its key's queries are the
// later positions (real token) or those of its chain (mask row).
template <int HD, class E>
__global__ __launch_bounds__(64) void k_dkv(const CodAttnArgs a) {
  const int2 tile = a.plan.tiles[blockIdx.x / kCodTile];
  const CodSampleInfo s = a.plan.samples[tile.x];
  const int p = tile.y * kCodTile + blockIdx.x % kCodTile, kvh = blockIdx.y;
  if (p >= s.cap) return;
  const int4 m = a.plan.order[s.off + p];
  const int64_t row = s.off + m.x;
  float dk[HD], dv[HD];
  for (int d = 0; d < HD; ++d) dk[d] = dv[d] = 0.f;
  if (p < s.len) {
    const auto* k = at<E>(a.k, row, kvh);
    const auto* v = at<E>(a.v, row, kvh);
    const int end = m.x < s.n_real ? s.len : m.w;
    for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h)
      for (int i = p + threadIdx.x; i < end; i += 64) {
        const int64_t qr = s.off + a.plan.order[s.off + i].x;
        const auto* q = at<E>(a.q, qr, h);
        const auto* go = at<E>(a.d_out, qr, h);
        const float w = expf(a.scale * dot<HD, E>(q, k) - a.lse[h * a.rows + qr]);
        const float ds = w * (dot<HD, E>(go, v) - a.delta[h * a.rows + qr]) * a.scale;
        for (int d = 0; d < HD; ++d) {
          dv[d] += w * E::load(go[d]);
          dk[d] += ds * E::load(q[d]);
        }
      }
  }
  for (int d = 0; d < HD; ++d) {
    const float x = wave_sum(dk[d]), y = wave_sum(dv[d]);
    if (threadIdx.x == 0) {
      at_out<E>(a.dk, row, kvh)[d] = E::store(x);
      at_out<E>(a.dv, row, kvh)[d] = E::store(y);
    }
  }
}

template <int HD, class E>
hipError_t launch_grad(const CodAttnArgs& a, hipStream_t st) {
  k_dq<HD, E><<<dim3(a.n_tiles * kCodTile, a.n_heads), 64, 0, st>>>(a);
  k_dkv<HD, E><<<dim3(a.n_tiles * kCodTile, a.n_kv), 64, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cod_attn_grad(int head_dim, int dtype, const CodAttnArgs& a, hipStream_t st) {
  if (head_dim == 64) return dtype == PARD_BF16 ? launch_grad<64, ElemBF16>(a, st) : launch_grad<64, ElemF16>(a, st);
  return dtype == PARD_BF16 ? launch_grad<128, ElemBF16>(a, st) : launch_grad<128, ElemF16>(a, st);
}

}  // namespace pard
