// Logits before tokens are picked: penalties for the history's tokens, biases,
// a grammar's mask, the largest logit that is left.
//
// A workgroup owns kChunk ids of a run of rows, a thread the same 16 of them in
// every row.  The part of a row's history lies in LDS as one word an id: bit 31,
// it is there; below, how often after the prompt.  The rows of a run that share
// a sequence and grow by a token (a verify pass's) only add that token, which
// the thread that owns its id does without a barrier: nobody else reads the
// word.  A second word holds an id's bias, by its place in the list, so that the
// order of the atomics shows nowhere.  The next row's logits are in flight while
// a row is worked on; vectors without a word set only pass the mask.
//
// Bound: memory, a logit read and written once (288 rows of 128 256 floats, histories
// to 1545: 74 us, 4.0 TB/s, the VALU busy 42 % of the time).  Eight ids a thread,
// barriers a row for its token and its pick, and nothing in flight ahead took 119;
// without non-temporal accesses it was 77.
#include "serve.h"

#include <algorithm>

namespace pard {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64, kPer = 16, kChunk = kThreads * kPer, kMaxRun = 32;

// Products and sums by themselves, each rounded: by default the compiler makes one
// operation of both (v - f c as one fused multiply-add), also of __fmul_rn and
// __fsub_rn, which are plain operators here.
__device__ __forceinline__ float mul(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ __forceinline__ float sub(float a, float b) {
#pragma clang fp contract(off)
  return a - b;
}
__device__ __forceinline__ float plus(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

template <class E>
__device__ __forceinline__ typename E::T minus_inf() { return E::store(-INFINITY); }

// A float as a number in its order, the id below it reversed: the largest key
// is the lowest id of the largest value.  0: no candidate.
__device__ __forceinline__ uint64_t pick_key(float y, int id) {
  if (!(y > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(y + 0.f);        // (-0 is 0)
  return (uint64_t)((b >> 31) ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - (uint32_t)id);
}

// The largest value of a wavefront and the lowest id that has it, in every lane
// of the last row of 16 (lane 63).
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_step(float x) {
  return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(x), (int)__float_as_uint(x), CTRL, ROWS, 0xF, false)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int min_step(int x) {
  return min(x, __builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint64_t wave_pick(float y, int id) {
  float m = max_step<0x111, 0xF>(y);                  // row_shr 1, 2, 4, 8; row_bcast 15, 31
  m = max_step<0x112, 0xF>(m);
  m = max_step<0x114, 0xF>(m);
  m = max_step<0x118, 0xF>(m);
  m = max_step<0x142, 0xA>(m);
  m = max_step<0x143, 0xC>(m);
  m = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(m), 63));
  int i = y == m ? id : 0x7fffffff;
  i = min_step<0x111, 0xF>(i);
  i = min_step<0x112, 0xF>(i);
  i = min_step<0x114, 0xF>(i);
  i = min_step<0x118, 0xF>(i);
  i = min_step<0x142, 0xA>(i);
  i = min_step<0x143, 0xC>(i);
  return pick_key(m, __builtin_amdgcn_readlane(i, 63));
}

template <class E, bool VEC>
__global__ __launch_bounds__(kThreads) void k_logits(const LogitsArgs a, int run) {
  using T = typename E::T;
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1, NV = kPer / W;         // ids that lie together, such vectors of a thread
  __shared__ __attribute__((aligned(16))) uint32_t seen[kChunk], bias[kChunk];
  __shared__ int r_seq[kMaxRun], r_len[kMaxRun], r_mask[kMaxRun], r_new[kMaxRun];
  const int tid = threadIdx.x, id0 = blockIdx.x * kChunk, n_ids = min(kChunk, a.vocab - id0);
  const int r0 = a.row0 + blockIdx.y * run, n_rows = min(run, a.rows - r0);
  auto at_of = [&](int i) { return (i * kThreads + tid) * W; };           // first id of vector i, within the chunk

  struct Row {
    T x[kPer];
    uint32_t mask[NV];
  };
  auto load = [&](Row& d, int k) __attribute__((always_inline)) {
    const T* const src = reinterpret_cast<const T*>(a.logits) + (r0 + k) * a.stride + id0;
    const int mr = r_mask[k];
    const uint32_t* const words = mr >= 0 && mr < a.n_masks ? a.mask + mr * a.mask_stride + id0 / 32 : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = at_of(i);
      if (at + W <= n_ids) {
        if constexpr (VEC) {
          const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + at));
#pragma unroll
          for (int j = 0; j < W; ++j) {
            if constexpr (sizeof(T) == 4) d.x[i * W + j] = __uint_as_float(v[j]);
            else d.x[i * W + j] = (T)(v[j / 2] >> (16 * (j & 1)));
          }
        } else {
          d.x[i] = src[at];
        }
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) d.x[i * W + j] = at + j < n_ids ? src[at + j] : minus_inf<E>();
      }
      d.mask[i] = words && at < n_ids ? words[at / 32] : mr < 0 ? ~0u : 0u;   // (a mask that is not there allows nothing)
    }
  };

  // what the run's rows are; the token that a row adds to the one before it
  if (tid < n_rows) {
    auto seq_of = [&](int r) {
      const int s = a.row_seq ? a.row_seq[r] : r;
      return (uint32_t)s < (uint32_t)a.n_seqs ? s : -1;
    };
    auto len_of = [&](int r, int s) { return s >= 0 && a.tokens ? (int)min((int64_t)max(a.row_len[r], 0), a.tokens_stride) : 0; };
    const int r = r0 + tid, s = seq_of(r), n = len_of(r, s);
    r_seq[tid] = s;
    r_len[tid] = n;
    r_mask[tid] = !a.mask ? -1 : a.mask_row ? a.mask_row[r] : r;
    int added = -1;
    if (tid > 0 && n > 0) {
      const int sp = seq_of(r - 1);
      if (sp == s && len_of(r - 1, sp) == n - 1) added = a.tokens[s * a.tokens_stride + n - 1];
    }
    r_new[tid] = added;
  }
  __syncthreads();
  Row d0, d1;
  load(d0, 0);

  int seq = -2, len = 0, prompt = 0;                  // what LDS holds
  bool words = false, biases = false;                 // whether it holds any
  float rep = 1.f, pres = 0.f, freq = 0.f;
  // ids lo .. hi - 1 of the history of row k's sequence, by everyone
  auto add = [&](int lo, int hi) {
    const int32_t* const history = a.tokens + seq * a.tokens_stride;
    for (int i = lo + tid; i < hi; i += kThreads) {
      const int64_t id = (int64_t)history[i] - id0;
      if (id >= 0 && id < n_ids) {
        if (i < prompt) atomicOr(&seen[id], 0x80000000u);
        else atomicAdd(&seen[id], 1u);
      }
    }
  };
  auto row = [&](int k, Row& d, Row& next) __attribute__((always_inline)) {
    if (k + 1 < n_rows) load(next, k + 1);            // uniform
    const int s = __builtin_amdgcn_readfirstlane(r_seq[k]), n = __builtin_amdgcn_readfirstlane(r_len[k]);
    if (s != seq || n < len) {                        // uniform: another history
      if (seq != -2) __syncthreads();
      for (int i = tid; i < kChunk / 4; i += kThreads) {
        reinterpret_cast<u32x4*>(seen)[i] = u32x4{0, 0, 0, 0};
        reinterpret_cast<u32x4*>(bias)[i] = u32x4{0, 0, 0, 0};
      }
      seq = s;
      len = n;
      prompt = s >= 0 && a.prompt_len ? max(a.prompt_len[s], 0) : 0;
      rep = s >= 0 && a.repetition ? a.repetition[s] : 1.f;
      pres = s >= 0 && a.presence ? a.presence[s] : 0.f;
      freq = s >= 0 && a.frequency ? a.frequency[s] : 0.f;
      words = n > 0;
      int b0 = 0, b1 = 0;
      if (s >= 0 && a.bias_start) {
        b0 = min(max(a.bias_start[s], 0), a.n_bias);
        b1 = min(max(a.bias_start[s + 1], 0), a.n_bias);
      }
      biases = b1 > b0;
      __syncthreads();
      for (int i = b0 + tid; i < b1; i += kThreads) {
        const int64_t id = (int64_t)a.bias_ids[i] - id0;
        if (id >= 0 && id < n_ids) atomicMax(&bias[id], (uint32_t)i + 1);
      }
      if (n > 0) add(0, n);
      __syncthreads();
    } else if (n == len + 1) {                        // uniform: its owner adds the token
      const int64_t id = (int64_t)r_new[k] - id0;
      if (id >= 0 && id < n_ids && (int)(id / W) % kThreads == tid) {
        if (len < prompt) seen[id] |= 0x80000000u;
        else seen[id] += 1;
      }
      len = n;
      words = true;
    } else if (n > len) {
      __syncthreads();                                // (the row before has read its words)
      add(len, n);
      len = n;
      words = true;
      __syncthreads();
    }
    float top = -INFINITY;
    int top_id = 0x7fffffff;
    T* const dst = reinterpret_cast<T*>(a.out) + (r0 + k) * a.out_stride + id0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = at_of(i);
      T* const x = d.x + i * W;
      if (words || biases) {                          // uniform
        uint32_t h[W], b[W], any = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) any |= h[j] = seen[at + j];
#pragma unroll
        for (int j = 0; j < W; ++j) b[j] = 0;
        if (biases) {
#pragma unroll
          for (int j = 0; j < W; ++j) any |= b[j] = bias[at + j];
        }
        if (any) {
#pragma unroll
          for (int j = 0; j < W; ++j) {
            if (!(h[j] | b[j])) continue;
            float v = E::load(x[j]);
            if (h[j]) {
              if (a.repetition) v = v > 0.f ? v / rep : mul(v, rep);
              const uint32_t c = h[j] & 0x7fffffffu;
              if (c && a.frequency) v = sub(v, mul(freq, (float)c));
              if (c && a.presence) v = sub(v, pres);
            }
            if (b[j]) v = plus(v, a.bias_values[b[j] - 1]);
            x[j] = E::store(v);
          }
        }
      }
      const uint32_t allowed = d.mask[i] >> (at & 31);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        x[j] = allowed >> j & 1 ? x[j] : minus_inf<E>();
        const float v = E::load(x[j]);
        if (v > top) top = v, top_id = id0 + at + j;     // (past the vocabulary: -infinity)
      }
      if (at + W <= n_ids) {
        if constexpr (VEC) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) v[j] = __float_as_uint(x[j]);
            else v[j] = (uint32_t)x[2 * j] | (uint32_t)x[2 * j + 1] << 16;
          }
          __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(dst + at));
        } else {
          dst[at] = x[0];
        }
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
          if (at + j < n_ids) dst[at + j] = x[j];
      }
    }
    if (a.best) {                                     // uniform
      const uint64_t key = wave_pick(top, top_id);
      if ((tid & 63) == 0) a.keys[((int64_t)(r0 + k) * gridDim.x + blockIdx.x) * kWaves + (tid >> 6)] = key;
    }
  };
  for (int k = 0; k < n_rows; k += 2) {
    row(k, d0, d1);
    if (k + 1 < n_rows) row(k + 1, d1, d0);
  }
}

__global__ __launch_bounds__(256) void k_logits_best(const uint64_t* keys, int rows, int n, int32_t* best) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= rows) return;
  uint64_t top = 0;
  for (int i = lane; i < n; i += 64) top = std::max(top, keys[(int64_t)r * n + i]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    top = std::max(top, (uint64_t)__shfl_xor((unsigned)(top >> 32), d) << 32 | (uint32_t)__shfl_xor((unsigned)top, d));
  if (lane == 0) best[r] = top ? (int32_t)(0xffffffffu - (uint32_t)top) : -1;
}

template <class E>
hipError_t launch_type(const LogitsArgs& a, hipStream_t st) {
  const int chunks = (a.vocab + kChunk - 1) / kChunk;
  // Rows of a run: few balance the ids that histories are full of (288 rows of
  // 128 256 with all steps, histories to 1545: 83 us in 1024 workgroups, 77 in
  // 4096), many scan a history less often (16 000 tokens: 84 and 105 us).
  const int64_t wanted = a.tokens && a.tokens_stride > 2048 ? 1024 : 4096;
  int run = (int)std::min<int64_t>(((int64_t)a.rows * chunks + wanted - 1) / wanted, kMaxRun);
  if ((a.rows + run - 1) / run > 65535) run = kMaxRun;
  const int size = sizeof(typename E::T), w = 16 / size;
  const bool vec = a.stride % w == 0 && a.out_stride % w == 0 && reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  // (more rows than one launch's second dimension holds: several)
  for (LogitsArgs b = a; b.row0 < a.rows; b.row0 += 65535 * run) {
    const dim3 grid(chunks, std::min((a.rows - b.row0 + run - 1) / run, 65535));
    if (vec) k_logits<E, true><<<grid, kThreads, 0, st>>>(b, run);
    else k_logits<E, false><<<grid, kThreads, 0, st>>>(b, run);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.best) return hipSuccess;
  k_logits_best<<<(a.rows + 3) / 4, 256, 0, st>>>(a.keys, a.rows, chunks * kWaves, a.best);
  return hipGetLastError();
}

}  // namespace

int logits_keys(int vocab) { return (vocab + kChunk - 1) / kChunk * kWaves; }

hipError_t launch_logits_adjust(int dtype, const LogitsArgs& a, hipStream_t st) {
  if (dtype == PARD_F32) return launch_type<ElemF32>(a, st);
  if (dtype == PARD_BF16) return launch_type<ElemBF16>(a, st);
  return launch_type<ElemF16>(a, st);
}

}  // namespace pard
