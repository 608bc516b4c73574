// Mask-token loss (eq. 8) over packed rows and its gradient.
//
//   CE = log sum exp(x) - x[label];  d x = w (exp(x - lse) - [label]),
// w the row's share of the loss (1 / its subtask's counted rows, weighted).
// Two launches: the counted rows of every subtask, then the rows, whose last
// workgroup to end adds the workgroups' sums up (in their order).
//
// Bound: memory (the logits in, the gradient out).  So a row is read once: its
// 16-byte vectors stay in the registers of one wavefront (up to 16 KiB) or
// workgroup (at most 20 a thread of 1024: 163 840 logits of two bytes) from the
// sum to the gradient, and as soon as a vector's gradient is stored, its registers
// take the same vector of the next row.  Longer rows are read a second time.  4099 rows of
// 128 256 bf16 logits with gradients: 525 us, 4.0 TB/s of a large copy's 4.9 (the
// row's barrier, and 16 vectors' registers leave one workgroup a CU); 2050
// rows of 152 064 f16 logits alone: 128 us, 4.9 TB/s.  Element by
// element, rows with gradients read twice, took 1414 and 398 us.
#include "train.h"

#include <algorithm>

namespace pard {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kLossThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Subtask of row r, 0 if it does not count.
__device__ __forceinline__ int section_of(const CodLossArgs& a, int r) {
  const int k = a.section ? a.section[r] : 1;
  return a.labels[r] >= 0 && k >= 1 && k <= a.n_sections ? k : 0;
}

// Counted rows of each subtask, kLossCountBlocks partial counts (integers: any
// order of the atomics gives the same).
__global__ __launch_bounds__(kLossThreads) void k_loss_count(const CodLossArgs a) {
  __shared__ int n_s[kCodMaxSections + 1];
  for (int k = threadIdx.x; k <= kCodMaxSections; k += kLossThreads) n_s[k] = 0;
  __syncthreads();
  for (int64_t r = (int64_t)blockIdx.x * kLossThreads + threadIdx.x; r < a.rows; r += (int64_t)kLossCountBlocks * kLossThreads)
    atomicAdd(&n_s[section_of(a, (int)r)], 1);
  __syncthreads();
  for (int k = threadIdx.x; k < kCodMaxSections; k += kLossThreads) a.counts[blockIdx.x * kCodMaxSections + k] = n_s[k + 1];
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
}

// Counted rows of each subtask, in LDS (one barrier).
__device__ __forceinline__ void load_counts(const CodLossArgs& a, int (&n_s)[kCodMaxSections]) {
  for (int k = threadIdx.x; k < a.n_sections; k += blockDim.x) {
    int n = 0;
#pragma unroll
    for (int b = 0; b < kLossCountBlocks; ++b) n += a.counts[b * kCodMaxSections + k];
    n_s[k] = n;
  }
  __syncthreads();
}

// Joins two (maximum, sum of exp(x - maximum)) pairs.  Logits are subtracted
// before they are scaled to base 2: the type's lowest value does not overflow.
__device__ __forceinline__ void join(float& m, float& l, float om, float ol) {
  if (om == -INFINITY) {
    l += ol;                                         // (0, or NaN)
    return;
  }
  const float n = m == -INFINITY ? om : fmaxf(m, om);
  l = l * exp2f((m - n) * kLog2e) + ol * exp2f((om - n) * kLog2e);
  m = n;
}

// 16 bytes of logits.
template <class E>
struct LossVec {
  static constexpr int N = 8;
  uint4 v;
  __device__ __forceinline__ float operator[](int i) const {
    const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return E::load((uint16_t)(i & 1 ? w >> 16 : w));
  }
  __device__ __forceinline__ static LossVec pack(const float (&x)[N]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)E::store(x[2 * i]) | ((uint32_t)E::store(x[2 * i + 1]) << 16);
    return LossVec{uint4{w[0], w[1], w[2], w[3]}};
  }
};
template <>
struct LossVec<ElemF32> {
  static constexpr int N = 4;
  float4 v;
  __device__ __forceinline__ float operator[](int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  __device__ __forceinline__ static LossVec pack(const float (&x)[N]) { return LossVec{float4{x[0], x[1], x[2], x[3]}}; }
};

// Adds the elements of C vectors to a thread's (maximum, sum).
template <class E, int C>
__device__ __forceinline__ void add_vectors(const LossVec<E>* v, float& m, float& l) {
  constexpr int N = LossVec<E>::N;
  float top = v[0][0];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, v[c][i]);
  if (top > m) {
    l *= exp2f((m - top) * kLog2e);                  // (m = -infinity: l is 0)
    m = top;
  }
  // (no finite logit so far: every term is 0, or NaN for a NaN)
  const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) l += __builtin_amdgcn_exp2f((v[c][i] - ref) * kLog2e);
}

// Rows of T threads, NV vectors each; a workgroup's R sets of T threads take rows
// of their own (T = 64: a wavefront a row, no barrier).  A row's elements before its first 16-byte
// boundary and after its last are a thread's own each (fewer than T).
// RESIDENT: the vectors stay in registers, and the next row's follow them in;
// otherwise they are read NV at a time, twice where there is a gradient.
// SCALAR_OUT: the gradient's rows lie at other offsets from a 16-byte boundary.
template <class E, int T, int R, int NV, bool RESIDENT, bool SCALAR_OUT>
__global__ __launch_bounds__(T * R) void k_loss_row(const CodLossArgs a) {
  using Vec = LossVec<E>;
  using Elem = typename E::T;
  constexpr int N = Vec::N, SZ = sizeof(Elem), W = T / 64;
  constexpr int C = NV % (16 / N) == 0 ? 16 / N : 1;   // vectors added at a time: 16 logits
  __shared__ float m_s[2][W], l_s[2][W];
  __shared__ int n_s[kCodMaxSections];
  static_assert(R == 1 || T == 64, "sets of several wavefronts would meet at the rows' barriers");
  __shared__ double sum_s[R][kCodMaxSections];       // each set's losses, in its rows' order
  __shared__ int last_s;
  for (int q = threadIdx.x; q < R * kCodMaxSections; q += T * R) sum_s[q / kCodMaxSections][q % kCodMaxSections] = 0.0;
  load_counts(a, n_s);
  int n_all = 0;
  for (int q = 0; q < a.n_sections; ++q) n_all += n_s[q];
  // (sets of one wavefront: in scalar registers)
  const int set = R == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / T);
  const int tid = threadIdx.x - set * T, lane = tid & 63, wave = tid >> 6;
  const int row0 = blockIdx.x * R + set, row_step = gridDim.x * R;
  Vec v[NV];
  float edge = -INFINITY;                            // this thread's element outside the vectors
  float x_label = 0.f;
  int k = 0, label = -1, head = 0, n_vec = 0;
  auto shape = [&](int r) __attribute__((always_inline)) {
    // elements before the first boundary (all of a row shorter than that)
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) + a.stride * r * SZ;
    head = min((int)((16 - (at & 15)) & 15) / SZ, a.vocab);
    n_vec = (a.vocab - head) / N;
  };
  // element index of this thread's edge element, -1 if it has none
  auto edge_at = [&]() __attribute__((always_inline)) {
    const int i = tid < head ? tid : head + n_vec * N + tid - head;
    return i < a.vocab ? i : -1;
  };
  float low[N];
#pragma unroll
  for (int i = 0; i < N; ++i) low[i] = -INFINITY;
  const Vec none = Vec::pack(low);
  // vector i of this thread in a row whose vectors begin at the (uniform) address
  // base: a scalar address and a 32-bit offset
  const uint32_t voff = tid * 16;
  auto vec_at = [&](const char* base, int i) __attribute__((always_inline)) {
    return reinterpret_cast<const Vec*>(base + (uint64_t)i * (T * 16) + voff);
  };
  auto fetch = [&](const Elem* x, int i0, int i) __attribute__((always_inline)) {
    const char* const base = reinterpret_cast<const char*>(x + head);
    if ((i0 + i + 1) * T <= n_vec) {                 // uniform: the whole workgroup's
      v[i] = *vec_at(base, i0 + i);
    } else {
      v[i] = none;
      if ((i0 + i) * T + tid < n_vec) v[i] = *vec_at(base, i0 + i);
    }
  };
  auto row_of = [&](int r) __attribute__((always_inline)) { return reinterpret_cast<const Elem*>(a.logits) + r * a.stride; };
  auto meta = [&](int r) __attribute__((always_inline)) {
    k = section_of(a, r);
    label = a.labels[r];
  };
  const int rounds = RESIDENT ? 1 : (a.vocab / N + NV * T - 1) / (NV * T);
  if (RESIDENT && row0 < a.rows) {
    shape(row0);
#pragma unroll
    for (int i = 0; i < NV; ++i) fetch(row_of(row0), 0, i);
  }
  int turn = 0;
  for (int r = row0; r < a.rows; r += row_step, turn ^= 1) {
    const Elem* const x = row_of(r);
    Elem* const d = RESIDENT || a.d_logits ? reinterpret_cast<Elem*>(a.d_logits) + r * a.d_stride : nullptr;
    shape(r);
    meta(r);
    const int e = edge_at();
    edge = e >= 0 ? E::load(x[e]) : -INFINITY;
    if (k > 0) x_label = label < a.vocab ? E::load(x[label]) : __builtin_nanf("");
    float m = -INFINITY, l = 0.f;
    for (int q = 0; q < rounds; ++q) {
      if (!RESIDENT) {
#pragma unroll
        for (int i = 0; i < NV; ++i) fetch(x, q * NV, i);
      }
#pragma unroll
      for (int i = 0; i < NV; i += C) {
        add_vectors<E, C>(v + i, m, l);
        __builtin_amdgcn_sched_barrier(0);           // (few unpacked logits at a time)
      }
    }
    join(m, l, edge, edge == -INFINITY ? 0.f : 1.f);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      const float om = __shfl_xor(m, off), ol = __shfl_xor(l, off);
      join(m, l, om, ol);
    }
    // (also: x[label] is read before d, which may be x, is written)
    if (W > 1) {
      if (lane == 0) {
        m_s[turn][wave] = m;
        l_s[turn][wave] = l;
      }
      __syncthreads();
      m = m_s[turn][0];
      l = l_s[turn][0];
      for (int w = 1; w < W; ++w) join(m, l, m_s[turn][w], l_s[turn][w]);
    } else {
      __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0)
      asm volatile("" ::: "memory");
    }
    const float log2_l = log2f(l);                   // log sum exp = m + ln(l)
    if (tid == 0) {
      const float ce = k > 0 ? fmaf(log2_l, kLn2, m - x_label) : 0.f;
      if (a.row_loss) a.row_loss[r] = ce;
      if (k > 0) sum_s[set][k - 1] += ce;
    }
    if (!RESIDENT && !d) continue;
    const float w = k == 0 ? 0.f : label >= a.vocab ? __builtin_nanf("")
                           : a.weighted ? a.weights[k - 1] * a.grad_scale / n_s[k - 1] : a.grad_scale / n_all;
    const int n_now = n_vec, head_now = head;
    const int r_next = min((int64_t)r + row_step, (int64_t)a.rows - 1);   // (past the last row: that one again, unused)
    const Elem* const next = row_of(r_next);
    if (RESIDENT) shape(r_next);
    const char* const x_base = reinterpret_cast<const char*>(x + head_now);
    const char* const d_base = reinterpret_cast<const char*>(d + head_now);
    for (int q = 0; q < rounds; ++q) {
      if (!RESIDENT) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if ((q * NV + i) * T + tid < n_now) v[i] = *vec_at(x_base, q * NV + i);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = (q * NV + i) * T + tid;
        // (unpacked again here: kept from the sum, it would take twice the registers)
        asm("" : "+v"(v[i].v.x), "+v"(v[i].v.y), "+v"(v[i].v.z), "+v"(v[i].v.w));
        if ((q * NV + i + 1) * T <= n_now || at < n_now) {   // (the first part uniform)
          float g[N];
#pragma unroll
          for (int j = 0; j < N; ++j) g[j] = k > 0 ? w * __builtin_amdgcn_exp2f(fmaf(v[i][j] - m, kLog2e, -log2_l)) : 0.f;
          if (SCALAR_OUT) {
#pragma unroll
            for (int j = 0; j < N; ++j) d[head_now + at * N + j] = E::store(g[j]);
          } else {
            const Vec out = Vec::pack(g);
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, out.v),
                                        reinterpret_cast<u32x4*>(const_cast<Vec*>(vec_at(d_base, q * NV + i))));
          }
        }
        if (RESIDENT) fetch(next, 0, i);
        __builtin_amdgcn_sched_barrier(0);           // (one vector at a time: its registers are taken over)
      }
    }
    if (e >= 0) d[e] = E::store(k > 0 ? w * exp2f(fmaf(edge - m, kLog2e, -log2_l)) : 0.f);
    // the label's element again, by the thread that wrote it
    if (k > 0 && label < a.vocab) {
      const int in_vec = label - head_now;
      const bool own = in_vec >= 0 && in_vec < n_now * N ? in_vec / N % T == tid : label == e;
      if (own) d[label] = E::store(w * (exp2f(fmaf(x_label - m, kLog2e, -log2_l)) - 1.f));
    }
  }

  // the workgroups' sums: [workgroup][subtask]
  // (device-scope stores, complete before the ticket, and device-scope loads
  // after it: a release and an acquire would write back and drop whole caches)
  if (R > 1) __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 0; q < a.n_sections; ++q) {
      double s = 0.0;
      for (int i = 0; i < R; ++i) s += sum_s[i][q];
      __hip_atomic_store(&a.sums[(size_t)blockIdx.x * a.n_sections + q], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);              // vmcnt(0)
    asm volatile("" ::: "memory");
    last_s = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last_s) return;                               // uniform
  for (int q = threadIdx.x / 64; q < a.n_sections; q += W * R) {   // a wavefront a subtask
    double s = 0.0;
    for (int b0 = lane; b0 < (int)gridDim.x; b0 += 64 * 16) {   // 16 loads in flight
      double x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int b = min(b0 + 64 * i, (int)gridDim.x - 1);
        x[i] = __hip_atomic_load(&a.sums[(size_t)b * a.n_sections + q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s += b0 + 64 * i < (int)gridDim.x ? x[i] : 0.0;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
    if (lane == 0) {
      sum_s[0][q] = s;
      a.loss[1 + q] = n_s[q] ? (float)(s / n_s[q]) : 0.f;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int q = 0; q < a.n_sections; ++q)
      total += a.weighted ? (n_s[q] ? a.weights[q] * (sum_s[0][q] / n_s[q]) : 0.0) : sum_s[0][q];
    a.loss[0] = (float)(a.weighted ? total : n_all ? total / n_all : 0.0);
  }
}

template <class E, int T, int R, int NV, bool RESIDENT, bool SCALAR_OUT = false>
void launch_variant(const CodLossArgs& a, hipStream_t st) {
  // short and resident rows: as many workgroups as 256 CUs hold at once (1024
  // threads a CU, 2048 of those with few vectors), each with several rows
  const int most = RESIDENT || T <= 256 ? 256 * (NV <= 8 ? 2048 : 1024) / (T * R) : kLossMaxBlocks;
  const int blocks = std::max(1, std::min((a.rows + R - 1) / R, most));
  k_loss_row<E, T, R, NV, RESIDENT, SCALAR_OUT><<<blocks, T * R, 0, st>>>(a);
}

// A row's threads: as few as hold it with 8 or 16 vectors each, so that a CU has
// several rows, which wait at different times (bf16 with gradients: 60 000 rows of
// 1024 logits 95 us by wavefronts, 180 by 256 threads; 30 000 of 4096 132 and 167;
// 4000 of 32 000 113 by 256 threads, 149 by 1024).
template <class E>
hipError_t launch_rows(const CodLossArgs& a, hipStream_t st) {
  constexpr int N = LossVec<E>::N, SZ = 16 / N;
  k_loss_count<<<kLossCountBlocks, kLossThreads, 0, st>>>(a);
  const int n = (a.vocab + N - 1) / N;               // vectors of a row
  const bool same = !a.d_logits || ((a.logits - a.d_logits) % 16 == 0 && (a.rows == 1 || (a.stride - a.d_stride) * SZ % 16 == 0));
  if (!same) launch_variant<E, 1024, 1, 4, false, true>(a, st);
  else if (!a.d_logits || n > 20480) {
    // (2050 rows of 152 064 logits: 512 threads 139 us, 1024 181)
    if (n <= 256) launch_variant<E, 64, 4, 4, false>(a, st);
    else if (n <= 1024) launch_variant<E, 64, 4, 8, false>(a, st);
    else if (n <= 4096) launch_variant<E, 256, 1, 8, false>(a, st);
    else launch_variant<E, 512, 1, 8, false>(a, st);
  }
  else if (n <= 64) launch_variant<E, 64, 4, 1, true>(a, st);
  else if (n <= 256) launch_variant<E, 64, 4, 4, true>(a, st);
  else if (n <= 1024) launch_variant<E, 64, 4, 16, true>(a, st);
  else if (n <= 2048) launch_variant<E, 256, 1, 8, true>(a, st);
  else if (n <= 4096) launch_variant<E, 256, 1, 16, true>(a, st);
  else if (n <= 8192) launch_variant<E, 512, 1, 16, true>(a, st);
  else if (n <= 16384) launch_variant<E, 1024, 1, 16, true>(a, st);
  else launch_variant<E, 1024, 1, 20, true>(a, st);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cod_loss(int dtype, const CodLossArgs& a, hipStream_t st) {
  switch (dtype) {
    case PARD_F32: return launch_rows<ElemF32>(a, st);
    case PARD_BF16: return launch_rows<ElemBF16>(a, st);
    case PARD_F16: return launch_rows<ElemF16>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace pard
