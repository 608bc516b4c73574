// Rotary positions of queries and keys, with an optional RMSNorm of every head
// in the same pass, and the gradient.
//
//   forward   n = x r g,  r = 1 / sqrt(mean(x^2) + eps)   (or n = x)
//             y = R n, R turning pair i of the head by the row's angle
//   gradient  dn = R^T dy;  dg += dn x r;  dx = r (t - x^ mean(t x^)), t = g dn, x^ = x r
//
// Bound: memory (x in, y out; dy, x in, dx out).  bf16, 34 500 rows of 32 + 8
// heads x 64: 76 us, 4.6 TB/s of the 4.9 of a large copy; the norm's gradient,
// 8191 rows of 40 heads x 128: 55 us, 4.7 TB/s, and 7 us for the gains' sums
// (float32: a lane's rows, then the workgroup's lanes, then the workgroups).
// One wavefront per (row, head) with 2-byte accesses took 1090 and 1200 us.
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

// x of another lane of the same 16 (DPP control CTRL).
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Sum over groups of W consecutive lanes (W a power of two from 4 to 64), in
// every lane, by lane permutations of the VALU: neighbours, pairs, then mirrored
// (whose two halves are uniform by then), then swapped rows and halves.
template <int W>
__device__ __forceinline__ float group_sum(float x) {
  x += dpp<0xB1>(x);                                 // quad_perm 1,0,3,2
  x += dpp<0x4E>(x);                                 // quad_perm 2,3,0,1
  if (W >= 8) x += dpp<0x141>(x);                    // row_half_mirror
  if (W >= 16) x += dpp<0x140>(x);                   // row_mirror
  if (W >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (W >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// Any shape (odd dims, unaligned rows): one wavefront per (row, head), a lane's
// elements 64 apart.
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

// Vectorised kernels, V = 8 or 4 elements a vector.  A head is units of two
// vectors: unit u < rot / 2V turns the pairs V u .. V u + V - 1 (half: elements
// V u .. and rot / 2 + V u ..; interleaved: 2V u ..), a later unit is the 2V
// elements 2V u ...  V = 4 where dims or strides fit no vectors of 8: 80 dims, 40
// of them turned, 37 us in place of 390 with one element at a time; where both
// fit, 8 is faster (34 against 38 us at 80 dims).  W lanes (the next power of two) hold one head, one unit
// each, and take the heads of one row H apart, so that a lane's cosines and sines
// are read once per row.
template <class E, int V>
struct Vec {
  static_assert(sizeof(typename E::T) == 2, "two 16-bit elements a word");
  typedef uint32_t Words __attribute__((ext_vector_type(V / 2)));
  Words w;
  __device__ __forceinline__ void load(const char* p) { w = *reinterpret_cast<const Words*>(p); }
  __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      x[2 * i] = E::load((uint16_t)w[i]);
      x[2 * i + 1] = E::load((uint16_t)(w[i] >> 16));
    }
  }
  __device__ __forceinline__ static void store(char* p, const float (&x)[V]) {
    Words w;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) w[i] = (uint32_t)E::store(x[2 * i]) | ((uint32_t)E::store(x[2 * i + 1]) << 16);
    *reinterpret_cast<Words*>(p) = w;
  }
};
template <int V>
struct Vec<ElemF32, V> {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4 w[V / 4];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = reinterpret_cast<const f32x4*>(p)[i];
  }
  __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = w[i / 4][i % 4];
  }
  __device__ __forceinline__ static void store(char* p, const float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
      reinterpret_cast<f32x4*>(p)[i] = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  }
};

// The elements of a unit turned by the row's angles (INV: back).
template <int LAYOUT, bool INV, int V>
__device__ __forceinline__ void turn_unit(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    // the pair: (a[i], b[i]), or neighbours
    constexpr int H = V / 2;
    float& x = LAYOUT == PARD_ROPE_HALF ? a[i] : (i < H ? a[2 * (i % H)] : b[2 * (i % H)]);
    float& y = LAYOUT == PARD_ROPE_HALF ? b[i] : (i < H ? a[2 * (i % H) + 1] : b[2 * (i % H) + 1]);
    const float sn = INV ? -s[i] : s[i], u = x * c[i] - y * sn;
    y = y * c[i] + x * sn;
    x = u;
  }
}

template <class E, int LAYOUT, bool GRAD, bool NORM, int V, int W>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const RopeArgs a, int h_step, int rows_per_block) {
  constexpr int SZ = sizeof(typename E::T), U = GRAD && NORM ? 2 : 4;   // heads in flight
  const int tid = threadIdx.x, unit = tid % W, slot = tid / W;
  const int h0 = slot % h_step, row_slot = slot / h_step, row_step = kRopeThreads / W / h_step;
  const int heads = a.n_q + a.n_k;
  const bool on = unit * 2 * V < a.hd, turns = on && unit * 2 * V < a.rot;
  // element offsets of this lane's two vectors
  const int o0 = !on ? 0 : turns && LAYOUT == PARD_ROPE_HALF ? unit * V : unit * 2 * V;
  const int o1 = !on ? 0 : turns && LAYOUT == PARD_ROPE_HALF ? a.rot / 2 + unit * V : unit * 2 * V + V;
  float gq[2][V], gk[2][V], dgq[2][V], dgk[2][V];
  if (NORM) {
    // (16-byte loads; gains may lie at any float)
    typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
    const float* const kg = a.n_k > 0 ? a.k_gain : a.q_gain;   // (no keys: not used)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.q_gain + (b ? o1 : o0) + i);
        const f32x4 y = *reinterpret_cast<const f32x4*>(kg + (b ? o1 : o0) + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          gq[b][i + j] = x[j];
          gk[b][i + j] = y[j];
          dgq[b][i + j] = dgk[b][i + j] = 0.f;
        }
      }
  }
  const float inv_hd = 1.0f / a.hd;
  // (counted from the workgroup's first row: a row index past the last may not fit an int)
  const int row0 = blockIdx.x * rows_per_block, n_rows = min(a.rows - row0, rows_per_block);
  for (int i_row = row_slot; i_row < n_rows; i_row += row_step) {
    const int row = row0 + i_row, pos = a.pos[row];
    const bool ok = pos >= 0 && pos < a.n_pos;
    float c[V] = {}, s[V] = {};
    if (turns) {
      const float4* t = reinterpret_cast<const float4*>(a.table + (size_t)(ok ? pos : 0) * (a.rot / 2) + unit * V);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float4 v = t[i];
        c[2 * i] = v.x, s[2 * i] = v.y, c[2 * i + 1] = v.z, s[2 * i + 1] = v.w;
      }
    }
    for (int hb = h0; hb < heads; hb += U * h_step) {
      Vec<E, V> v[U][2], w[U][2];
      char* dst[U];
      bool live[U], is_q[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int hh = hb + j * h_step;
        live[j] = hh < heads && on;
        is_q[j] = hh < a.n_q;
        const int head = is_q[j] ? hh : hh - a.n_q;
        const Heads& hi = is_q[j] ? a.q_in : a.k_in;
        const Heads& ho = is_q[j] ? a.q_out : a.k_out;
        dst[j] = ho.data + SZ * (row * ho.rs + head * ho.hs);
        if (live[j]) {
          const char* src = hi.data + SZ * (row * hi.rs + head * hi.hs);
          v[j][0].load(src + SZ * o0);
          v[j][1].load(src + SZ * o1);
          if (GRAD && NORM) {
            const Heads& hx = is_q[j] ? a.q_x : a.k_x;
            const char* sx = hx.data + SZ * (row * hx.rs + head * hx.hs);
            w[j][0].load(sx + SZ * o0);
            w[j][1].load(sx + SZ * o1);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        // (a head's lanes leave together: its sums stay whole.  A head that is not
        // there has no norm: with eps = 0 it would leave NaN in the gains' sums)
        if (NORM ? hb + j * h_step >= heads : !live[j]) continue;
        float x[2][V], y[2][V];
        if (live[j]) {
          v[j][0].get(x[0]);
          v[j][1].get(x[1]);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) x[0][i] = x[1][i] = 0.f;
        }
        if (GRAD) {
          if (turns) turn_unit<LAYOUT, true, V>(x[0], x[1], c, s);
          if (!ok) {
#pragma unroll
            for (int i = 0; i < V; ++i) x[0][i] = x[1][i] = __builtin_nanf("");
          }
        }
        if (NORM) {
          float(&z)[2][V] = GRAD ? y : x;                  // the head before the norm
          if (GRAD) {
            if (live[j]) {
              w[j][0].get(y[0]);
              w[j][1].get(y[1]);
            } else {
#pragma unroll
              for (int i = 0; i < V; ++i) y[0][i] = y[1][i] = 0.f;
            }
          }
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < V; ++i) ss += z[0][i] * z[0][i] + z[1][i] * z[1][i];
          const float r = 1.0f / sqrtf(group_sum<W>(ss) * inv_hd + a.eps);
          if (!GRAD) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < V; ++i) x[b][i] *= r * (is_q[j] ? gq[b][i] : gk[b][i]);
          } else {
            float dot = 0.f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < V; ++i) {
                y[b][i] *= r;                              // x^
                const float d = x[b][i] * y[b][i];
                if (is_q[j]) dgq[b][i] += d;
                else dgk[b][i] += d;
                x[b][i] *= is_q[j] ? gq[b][i] : gk[b][i];
                dot += x[b][i] * y[b][i];
              }
            const float mean = group_sum<W>(dot) * inv_hd;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < V; ++i) x[b][i] = r * (x[b][i] - y[b][i] * mean);
          }
        }
        if (!GRAD) {
          if (turns) turn_unit<LAYOUT, false, V>(x[0], x[1], c, s);
          if (!ok) {
#pragma unroll
            for (int i = 0; i < V; ++i) x[0][i] = x[1][i] = __builtin_nanf("");
          }
        }
        if (live[j]) {
          Vec<E, V>::store(dst[j] + SZ * o0, x[0]);
          Vec<E, V>::store(dst[j] + SZ * o1, x[1]);
        }
      }
    }
  }
  if (GRAD && NORM) {
    // this workgroup's sums of each element, over its slots in their order
    __shared__ float sum_s[2][kRopeThreads * 2 * V];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = b ? o1 + i : o0 + i;
        if (on) {
          sum_s[0][slot * a.hd + e] = dgq[b][i];
          sum_s[1][slot * a.hd + e] = dgk[b][i];
        }
      }
    __syncthreads();
    for (int e = tid; e < 2 * a.hd; e += kRopeThreads) {
      const int kind = e / a.hd, d = e % a.hd;
      float t = 0.f;
      for (int q = 0; q < kRopeThreads / W; ++q) t += sum_s[kind][q * a.hd + d];
      a.part[((size_t)blockIdx.x * 2 + kind) * a.hd + d] = t;
    }
  }
}

// Whether every vector of a tensor is aligned.
bool vector_fit(const Heads& h, int v, int size, int64_t rows, int heads) {
  const int bytes = std::min(v * size, 16);
  return reinterpret_cast<uintptr_t>(h.data) % bytes == 0 && (rows == 1 || h.rs * size % bytes == 0) &&
         (heads == 1 || h.hs * size % bytes == 0);
}

template <class E>
bool vectorised(int v, bool grad, const RopeArgs& a) {
  constexpr int size = sizeof(typename E::T);
  if (a.hd % (2 * v) || a.hd > 512 || a.rot % (2 * v)) return false;
  auto fit = [&](const Heads& q, const Heads& k) {
    return vector_fit(q, v, size, a.rows, a.n_q) && (a.n_k == 0 || vector_fit(k, v, size, a.rows, a.n_k));
  };
  return fit(a.q_in, a.k_in) && fit(a.q_out, a.k_out) && (!grad || !a.q_gain || fit(a.q_x, a.k_x));
}

// (returns the workgroups launched)
template <class E, int LAYOUT, bool GRAD, bool NORM, int V, int W>
int launch_width(const RopeArgs& a, hipStream_t st) {
  // heads of a row side by side: as many as a power of two up to 16 may be while
  // under 1/8 of the slots idle, and all that there are where rows are few
  const int heads = a.n_q + a.n_k, slots = kRopeThreads / W;
  int h_step = 1;
  while (h_step * 2 <= std::min(slots, 16) && (heads + 2 * h_step - 1) / (2 * h_step) * 2 * h_step <= heads + heads / 8) h_step *= 2;
  while (h_step * 2 <= slots && (int64_t)a.rows * h_step < 2048 && h_step < heads) h_step *= 2;
  const int row_step = slots / h_step;
  // gains: few workgroups, which read them (and leave partial sums of their
  // gradients) once (forward, 13 020 rows of 12 heads x 256: 33 us with at most
  // 2048, 40 with 1024, 66 with one for every few rows)
  const int64_t most = !NORM ? 1 << 20 : GRAD ? rope_grad_blocks(a) : 2048;
  const int64_t rows_per_block = ((a.rows + most - 1) / most + row_step - 1) / row_step * row_step;
  const int blocks = (int)((a.rows + rows_per_block - 1) / rows_per_block);
  k_rope<E, LAYOUT, GRAD, NORM, V, W><<<blocks, kRopeThreads, 0, st>>>(a, h_step, (int)rows_per_block);
  return blocks;
}

template <class E, int LAYOUT, bool GRAD, bool NORM, int V>
int launch_vector(const RopeArgs& a, hipStream_t st) {
  if (a.hd <= 64) return launch_width<E, LAYOUT, GRAD, NORM, V, 32 / V>(a, st);
  if (a.hd <= 128) return launch_width<E, LAYOUT, GRAD, NORM, V, 64 / V>(a, st);
  if (a.hd <= 256) return launch_width<E, LAYOUT, GRAD, NORM, V, 128 / V>(a, st);
  return launch_width<E, LAYOUT, GRAD, NORM, V, 256 / V>(a, st);
}

template <class E, int LAYOUT, int V>
void launch_kind(bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain, hipStream_t st) {
  if (!grad) {
    if (a.q_gain) launch_vector<E, LAYOUT, false, true, V>(a, st);
    else launch_vector<E, LAYOUT, false, false, V>(a, st);
  } else if (!a.q_gain) {
    launch_vector<E, LAYOUT, true, false, V>(a, st);
  } else {
    const int blocks = launch_vector<E, LAYOUT, true, true, V>(a, st);
    k_rope_gain_sum<<<2 * a.hd, 64, 0, st>>>(a.part, blocks, a.hd, a.n_k, q_dgain, k_dgain);
  }
}

template <class E, int LAYOUT>
hipError_t launch_layout(bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain, hipStream_t st) {
  const int64_t units = (int64_t)a.rows * (a.n_q + a.n_k);
  const int blocks = (int)std::min<int64_t>((units + 3) / 4, 4096);
  if (units > 0 && vectorised<E>(8, grad, a)) {
    launch_kind<E, LAYOUT, 8>(grad, a, q_dgain, k_dgain, st);
    return hipGetLastError();
  }
  if (units > 0 && vectorised<E>(4, grad, a)) {
    launch_kind<E, LAYOUT, 4>(grad, a, q_dgain, k_dgain, st);
    return hipGetLastError();
  }
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
