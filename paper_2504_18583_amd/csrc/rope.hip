// Rotary positions of queries and keys, with an optional RMSNorm of every head
// in the same pass, and the gradient.
//
//   forward   n = x r g,  r = 1 / sqrt(mean(x^2) + eps)   (or n = x)
//             y = R n, R turning pair i of the head by the row's angle
//   gradient  dn = R^T dy;  dg += dn x r;  dx = r (t - x^ mean(t x^)), t = g dn, x^ = x r
//
// Bound: memory (x in, y out; dy, x in, dx out).
#include "train.h"

#include <algorithm>

namespace pard {
namespace {

constexpr int kRopeThreads = 256;

__global__ void k_rope_spec_table(pard_rope_spec s, int n_pos, float2* tab) {
  const int half = s.rot_dim / 2;
  const size_t total = (size_t)n_pos * half;
  const double two_pi = 6.283185307179586, theta = s.theta, factor = s.factor, low = s.low, high = s.high;
  const double orig = s.original_max_pos;
  for (size_t t = (size_t)blockIdx.x * blockDim.x + threadIdx.x; t < total; t += (size_t)gridDim.x * blockDim.x) {
    const int pos = (int)(t / half), i = (int)(t % half);
    double w = pow(theta, -(2.0 * i) / s.rot_dim), m = 1.0;
    if (s.scaling == PARD_ROPE_LINEAR) {
      w /= factor;
    } else if (s.scaling == PARD_ROPE_LLAMA3) {
      const double u = fmin(fmax((orig * w / two_pi - low) / (high - low), 0.0), 1.0);
      w = (1.0 - u) * w / factor + u * w;
    } else if (s.scaling == PARD_ROPE_YARN) {
      const double per = s.rot_dim / (2.0 * log(theta));     // dim(t) = per ln(orig / (2 pi t))
      const double a = fmax(floor(per * log(orig / (two_pi * high))), 0.0);
      const double b = fmin(ceil(per * log(orig / (two_pi * low))), s.rot_dim - 1.0);
      const double ramp = fmin(fmax((i - a) / fmax(b - a, 1e-3), 0.0), 1.0);
      w = w / factor * ramp + w * (1.0 - ramp);
      m = 0.1 * log(factor) + 1.0;
    }
    const double ang = (double)pos * w;
    tab[t] = make_float2((float)(cos(ang) * m), (float)(sin(ang) * m));
  }
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// Sum over groups of W consecutive lanes (W a power of two), in every lane.
template <int W>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int off = W / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, W);
  return x;
}

// Any shape: one wavefront per (row, head), a lane's elements 64 apart.
// Element e's partner in its pair and which half of the pair it is.
template <class E, int LAYOUT, bool GRAD>
__global__ __launch_bounds__(kRopeThreads) void k_rope_any(const RopeArgs a) {
  using T = typename E::T;
  const int lane = threadIdx.x & 63, heads = a.n_q + a.n_k;
  const int64_t units = (int64_t)a.rows * heads, waves = (int64_t)gridDim.x * (kRopeThreads / 64);
  const bool norm = a.q_gain != nullptr;
  for (int64_t u = (int64_t)blockIdx.x * (kRopeThreads / 64) + threadIdx.x / 64; u < units; u += waves) {
    const int row = (int)(u / heads), hh = (int)(u % heads);
    const bool is_q = hh < a.n_q;
    const int head = is_q ? hh : hh - a.n_q;
    const Heads& hi = is_q ? a.q_in : a.k_in;
    const Heads& hx = is_q ? a.q_x : a.k_x;
    const Heads& ho = is_q ? a.q_out : a.k_out;
    const float* gain = is_q ? a.q_gain : a.k_gain;
    const T* in = reinterpret_cast<const T*>(hi.data) + row * hi.rs + head * hi.hs;
    const T* x = reinterpret_cast<const T*>(hx.data) + row * hx.rs + head * hx.hs;
    T* out = reinterpret_cast<T*>(ho.data) + row * ho.rs + head * ho.hs;
    const int pos = a.pos[row];
    const bool ok = pos >= 0 && pos < a.n_pos;
    const float2* cs = a.table + (size_t)(ok ? pos : 0) * (a.rot / 2);
    const float bad = ok ? 0.f : __builtin_nanf("");
    float r = 1.f, mean = 0.f;
    // rotated element e of the input (the gradient turns the other way)
    auto turned = [&](int e) {
      const float v = E::load(in[e]) * (GRAD || !norm ? 1.f : r * gain[e]);
      if (e >= a.rot) return v;
      const bool second = LAYOUT == PARD_ROPE_HALF ? e >= a.rot / 2 : e & 1;
      const int i = LAYOUT == PARD_ROPE_HALF ? (second ? e - a.rot / 2 : e) : e / 2;
      const int p = LAYOUT == PARD_ROPE_HALF ? (second ? e - a.rot / 2 : e + a.rot / 2) : e ^ 1;
      const float w = E::load(in[p]) * (GRAD || !norm ? 1.f : r * gain[p]);
      const float sn = (second != GRAD) ? cs[i].y : -cs[i].y;
      return v * cs[i].x + w * sn;
    };
    if (norm) {
      float ss = 0.f;
      for (int e = lane; e < a.hd; e += 64) {
        const float v = E::load((GRAD ? x : in)[e]);
        ss += v * v;
      }
      r = 1.0f / sqrtf(wave_sum(ss) / a.hd + a.eps);
      if (GRAD) {
        float dot = 0.f;
        for (int e = lane; e < a.hd; e += 64) dot += turned(e) * gain[e] * E::load(x[e]) * r;
        mean = wave_sum(dot) / a.hd;
      }
    }
    // the head is written once it is read (out may be in)
    constexpr int kMost = 16;
    float y[kMost];
#pragma unroll
    for (int q = 0; q < kMost; ++q) {
      const int e = lane + 64 * q;
      y[q] = 0.f;
      if (e < a.hd) {
        y[q] = turned(e) + bad;
        if (GRAD && norm) y[q] = r * (y[q] * gain[e] - E::load(x[e]) * r * mean);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < kMost; ++q)
      if (lane + 64 * q < a.hd) out[lane + 64 * q] = E::store(y[q]);
  }
}

// Gain gradients of any shape: workgroup b sums the rows b, b + blocks, ..., a
// thread one element of the head (of queries, then of keys).
template <class E, int LAYOUT>
__global__ __launch_bounds__(kRopeThreads) void k_rope_gain_any(const RopeArgs a) {
  using T = typename E::T;
  __shared__ float red[kRopeThreads / 64];
  for (int kind = 0; kind < 2; ++kind) {
    const int heads = kind ? a.n_k : a.n_q;
    const Heads& hi = kind ? a.k_in : a.q_in;
    const Heads& hx = kind ? a.k_x : a.q_x;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};             // hd <= 1024
    for (int64_t u = blockIdx.x; u < (int64_t)a.rows * heads; u += gridDim.x) {
      const int row = (int)(u / heads), head = (int)(u % heads);
      const T* in = reinterpret_cast<const T*>(hi.data) + row * hi.rs + head * hi.hs;
      const T* x = reinterpret_cast<const T*>(hx.data) + row * hx.rs + head * hx.hs;
      const int pos = a.pos[row];
      const bool ok = pos >= 0 && pos < a.n_pos;
      const float2* cs = a.table + (size_t)(ok ? pos : 0) * (a.rot / 2);
      float ss = 0.f;
      for (int e = threadIdx.x; e < a.hd; e += kRopeThreads) {
        const float v = E::load(x[e]);
        ss += v * v;
      }
      ss = wave_sum(ss);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
      __syncthreads();
      ss = 0.f;
      for (int w = 0; w < kRopeThreads / 64; ++w) ss += red[w];
      const float r = 1.0f / sqrtf(ss / a.hd + a.eps);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = threadIdx.x + q * kRopeThreads;
        if (e >= a.hd) continue;
        float v = E::load(in[e]);
        if (e < a.rot) {
          const bool second = LAYOUT == PARD_ROPE_HALF ? e >= a.rot / 2 : e & 1;
          const int i = LAYOUT == PARD_ROPE_HALF ? (second ? e - a.rot / 2 : e) : e / 2;
          const int p = LAYOUT == PARD_ROPE_HALF ? (second ? e - a.rot / 2 : e + a.rot / 2) : e ^ 1;
          v = v * cs[i].x + E::load(in[p]) * (second ? -cs[i].y : cs[i].y);
        }
        acc[q] += ok ? v * E::load(x[e]) * r : __builtin_nanf("");
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int e = threadIdx.x + q * kRopeThreads;
      if (e < a.hd) a.part[((size_t)blockIdx.x * 2 + kind) * a.hd + e] = acc[q];
    }
  }
}

// Sums the workgroups' partial gain gradients in a fixed order: one wavefront
// per element.
__global__ __launch_bounds__(64) void k_rope_gain_sum(const float* part, int blocks, int hd, int n_k, float* qg,
                                                      float* kg) {
  const int e = blockIdx.x % hd, kind = blockIdx.x / hd;
  float s = 0.f;
  for (int b = threadIdx.x; b < blocks; b += 64) s += part[((size_t)b * 2 + kind) * hd + e];
  s = wave_sum(s);
  if (threadIdx.x == 0) {
    if (kind == 0) qg[e] = s;
    else if (n_k > 0) kg[e] = s;
  }
}

template <class E, int LAYOUT>
hipError_t launch_layout(bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain, hipStream_t st) {
  const int64_t units = (int64_t)a.rows * (a.n_q + a.n_k);
  const int blocks = (int)std::min<int64_t>((units + 3) / 4, 4096);
  if (grad && a.q_gain) {
    // (before the rotation: dx may overwrite dy)
    k_rope_gain_any<E, LAYOUT><<<rope_grad_blocks(a), kRopeThreads, 0, st>>>(a);
    k_rope_gain_sum<<<2 * a.hd, 64, 0, st>>>(a.part, rope_grad_blocks(a), a.hd, a.n_k, q_dgain, k_dgain);
  }
  if (blocks == 0) return hipGetLastError();
  if (grad) k_rope_any<E, LAYOUT, true><<<blocks, kRopeThreads, 0, st>>>(a);
  else k_rope_any<E, LAYOUT, false><<<blocks, kRopeThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <class E>
hipError_t launch_elem(int layout, bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain, hipStream_t st) {
  return layout == PARD_ROPE_HALF ? launch_layout<E, PARD_ROPE_HALF>(grad, a, q_dgain, k_dgain, st)
                                  : launch_layout<E, PARD_ROPE_INTERLEAVED>(grad, a, q_dgain, k_dgain, st);
}

}  // namespace

int rope_grad_blocks(const RopeArgs& a) {
  return (int)std::min<int64_t>(std::max<int64_t>(1, (int64_t)a.rows * (a.n_q + a.n_k) / 16), 1024);
}

hipError_t launch_rope_spec_table(const pard_rope_spec& s, int n_pos, float2* table, hipStream_t st) {
  const size_t total = (size_t)n_pos * (s.rot_dim / 2);
  k_rope_spec_table<<<(int)std::min<size_t>((total + 255) / 256, 65536), 256, 0, st>>>(s, n_pos, table);
  return hipGetLastError();
}

hipError_t launch_qk_rope(int dtype, int layout, bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain,
                          hipStream_t st) {
  switch (dtype) {
    case PARD_F32: return launch_elem<ElemF32>(layout, grad, a, q_dgain, k_dgain, st);
    case PARD_BF16: return launch_elem<ElemBF16>(layout, grad, a, q_dgain, k_dgain, st);
    case PARD_F16: return launch_elem<ElemF16>(layout, grad, a, q_dgain, k_dgain, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace pard
