// Logits before tokens are picked: penalties for the history's tokens, biases,
// a grammar's mask, the largest logit that is left.
//
// A workgroup owns kChunk ids of a run of rows.  Its part of a row's history
// lies in LDS as one word an id: bit 31, it is there; below, how often after
// the prompt.  The rows of a run that share a sequence and grow (a verify
// pass's) only add their own tokens.  A second word holds an id's bias, by its
// place in the list, so that the order of the atomics shows nowhere.
//
// Bound: memory, a logit read and written once.
#include "serve.h"

#include <algorithm>

namespace pard {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 2048, kThreads = 256;

// Products and sums by themselves: what is left out changes nothing else.
__device__ __forceinline__ float mul(float a, float b) { return __fmul_rn(a, b); }
__device__ __forceinline__ float sub(float a, float b) { return __fsub_rn(a, b); }

// A float as a number in its order, the id below it reversed: the largest key
// is the lowest id of the largest value.  0: no candidate.
__device__ __forceinline__ uint64_t pick_key(float y, int id) {
  if (!(y > -INFINITY)) return 0;                     // (NaN neither)
  const uint32_t b = __float_as_uint(y + 0.f);        // (-0 is 0)
  return (uint64_t)((b >> 31) ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - (uint32_t)id);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t o = (uint64_t)__shfl_xor((unsigned)(k >> 32), d) << 32 | (uint32_t)__shfl_xor((unsigned)k, d);
    k = o > k ? o : k;
  }
  return k;
}

template <class E, bool VEC>
__global__ __launch_bounds__(kThreads) void k_logits(const LogitsArgs a, int run) {
  using T = typename E::T;
  constexpr int PER = kChunk / kThreads;              // ids of a thread
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1;    // that lie together
  __shared__ uint32_t seen[kChunk], bias[kChunk];
  __shared__ uint64_t tops[kThreads / 64];
  const int tid = threadIdx.x, id0 = blockIdx.x * kChunk, n_ids = min(kChunk, a.vocab - id0);
  const int r0 = blockIdx.y * run, r1 = min(r0 + run, a.rows);
  int seq = -2, len = 0, prompt = 0, n_biases = 0;    // what LDS holds
  float rep = 1.f, pres = 0.f, freq = 0.f;
  auto id_of = [&](int i) { return (i / W * kThreads + tid) * W + i % W; };   // within the chunk
  for (int r = r0; r < r1; ++r) {                     // uniform
    float x[PER];
    const T* src = reinterpret_cast<const T*>(a.logits) + r * a.stride + id0;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < PER; i += W) {
        const int at = id_of(i);
        if (at + W <= n_ids) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(src + at);
#pragma unroll
          for (int j = 0; j < W; ++j) {
            if constexpr (sizeof(T) == 4) x[i + j] = __uint_as_float(v[j]);
            else x[i + j] = E::load((uint16_t)(v[j / 2] >> (16 * (j & 1))));
          }
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) x[i + j] = at + j < n_ids ? E::load(src[at + j]) : 0.f;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) x[i] = id_of(i) < n_ids ? E::load(src[id_of(i)]) : 0.f;
    }
    int s = a.row_seq ? a.row_seq[r] : r;
    if ((uint32_t)s >= (uint32_t)a.n_seqs) s = -1;
    const int n = s >= 0 && a.tokens ? (int)min((int64_t)max(a.row_len[r], 0), a.tokens_stride) : 0;
    if (s != seq || n < len) {                        // another history
      if (seq != -2) __syncthreads();
      for (int i = tid; i < kChunk; i += kThreads) seen[i] = bias[i] = 0;
      __syncthreads();
      seq = s;
      len = 0;
      prompt = s >= 0 && a.prompt_len ? max(a.prompt_len[s], 0) : 0;
      rep = s >= 0 && a.tokens && a.repetition ? a.repetition[s] : 1.f;
      pres = s >= 0 && a.tokens && a.presence ? a.presence[s] : 0.f;
      freq = s >= 0 && a.tokens && a.frequency ? a.frequency[s] : 0.f;
      n_biases = 0;
      if (s >= 0 && a.bias_start) {
        const int b0 = min(max(a.bias_start[s], 0), a.n_bias), b1 = min(max(a.bias_start[s + 1], 0), a.n_bias);
        n_biases = max(b1 - b0, 0);
        for (int i = b0 + tid; i < b1; i += kThreads) {
          const int64_t id = (int64_t)a.bias_ids[i] - id0;
          if (id >= 0 && id < n_ids) atomicMax(&bias[id], (uint32_t)i + 1);
        }
      }
      if (n == 0) __syncthreads();
    } else if (n > len) {
      __syncthreads();                                // (the row before has read its words)
    }
    if (n > len) {
      const int32_t* history = a.tokens + s * a.tokens_stride;
      for (int i = len + tid; i < n; i += kThreads) {
        const int64_t id = (int64_t)history[i] - id0;
        if (id >= 0 && id < n_ids) {
          if (i < prompt) atomicOr(&seen[id], 0x80000000u);
          else atomicAdd(&seen[id], 1u);
        }
      }
      len = n;
      __syncthreads();
    }
    int mask_row = a.mask ? (a.mask_row ? a.mask_row[r] : r) : -1;
    const bool none = mask_row >= a.n_masks && a.mask;               // nothing is allowed
    const uint32_t* mask = mask_row >= 0 && !none ? a.mask + mask_row * a.mask_stride : nullptr;
    uint64_t top = 0;
    T y[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = id_of(i);
      float v = x[i];
      const uint32_t h = seen[at];
      if (h) {
        if (a.repetition) v = v > 0.f ? v / rep : mul(v, rep);
        const uint32_t c = h & 0x7fffffffu;
        if (c) {
          if (a.frequency) v = sub(v, mul(freq, (float)c));
          if (a.presence) v = sub(v, pres);
        }
      }
      if (n_biases) {
        const uint32_t k = bias[at];
        if (k) v = __fadd_rn(v, a.bias_values[k - 1]);
      }
      if (none || (mask && at < n_ids && !(mask[(id0 + at) >> 5] >> ((id0 + at) & 31) & 1))) v = -INFINITY;
      y[i] = E::store(v);
      if (a.best && at < n_ids) {
        const uint64_t k = pick_key(E::load(y[i]), id0 + at);
        top = k > top ? k : top;
      }
    }
    T* dst = reinterpret_cast<T*>(a.out) + r * a.out_stride + id0;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < PER; i += W) {
        const int at = id_of(i);
        if (at + W <= n_ids) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) v[j] = __float_as_uint(y[i + j]);
            else v[j] = (uint32_t)y[i + 2 * j] | (uint32_t)y[i + 2 * j + 1] << 16;
          }
          *reinterpret_cast<u32x4*>(dst + at) = v;
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j)
            if (at + j < n_ids) dst[at + j] = y[i + j];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (id_of(i) < n_ids) dst[id_of(i)] = y[i];
    }
    if (a.best) {                                     // uniform
      top = wave_max(top);
      if ((tid & 63) == 0) tops[tid >> 6] = top;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < kThreads / 64; ++w) top = tops[w] > top ? tops[w] : top;
        a.keys[(int64_t)r * gridDim.x + blockIdx.x] = top;
      }
      __syncthreads();
    }
  }
}

__global__ __launch_bounds__(256) void k_logits_best(const uint64_t* keys, int rows, int chunks, int32_t* best) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= rows) return;
  uint64_t top = 0;
  for (int i = lane; i < chunks; i += 64) {
    const uint64_t k = keys[(int64_t)r * chunks + i];
    top = k > top ? k : top;
  }
  top = wave_max(top);
  if (lane == 0) best[r] = top ? (int32_t)(0xffffffffu - (uint32_t)top) : -1;
}

template <class E>
hipError_t launch_type(const LogitsArgs& a, hipStream_t st) {
  const int chunks = logits_chunks(a.rows, a.vocab);
  // rows of a run: about 4 workgroups a CU are left
  int run = (int)std::min<int64_t>(std::max<int64_t>((int64_t)a.rows * chunks / 1024, 1), 16);
  run = std::max(run, (a.rows + 65534) / 65535);     // (a launch's second dimension)
  const int size = sizeof(typename E::T), w = 16 / size;
  const bool vec = a.stride % w == 0 && a.out_stride % w == 0 && reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  const dim3 grid(chunks, (a.rows + run - 1) / run);
  if (vec) k_logits<E, true><<<grid, kThreads, 0, st>>>(a, run);
  else k_logits<E, false><<<grid, kThreads, 0, st>>>(a, run);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.best) return e;
  k_logits_best<<<(a.rows + 3) / 4, 256, 0, st>>>(a.keys, a.rows, chunks, a.best);
  return hipGetLastError();
}

}  // namespace

int logits_chunks(int, int vocab) { return (vocab + kChunk - 1) / kChunk; }

hipError_t launch_logits_adjust(int dtype, const LogitsArgs& a, hipStream_t st) {
  if (dtype == PARD_F32) return launch_type<ElemF32>(a, st);
  if (dtype == PARD_BF16) return launch_type<ElemBF16>(a, st);
  return launch_type<ElemF16>(a, st);
}

}  // namespace pard
