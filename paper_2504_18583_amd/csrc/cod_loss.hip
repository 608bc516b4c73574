// Mask-token loss (eq. 8) over packed rows and its gradient.
//
//   CE = log sum exp(x) - x[label];  d x = w (exp(x - lse) - [label]),
// w the row's share of the loss (1 / its subtask's counted rows, weighted).
// Three launches: the counted rows of every subtask, one workgroup per row,
// the means.  Bound: memory (the logits in, the gradient out).
#include "train.h"

#include <algorithm>

namespace pard {
namespace {

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

__device__ __forceinline__ int count_of(const CodLossArgs& a, int k) {
  int n = 0;
  for (int b = 0; b < kLossCountBlocks; ++b) n += a.counts[b * kCodMaxSections + k - 1];
  return n;
}

// Joins two (maximum, sum of 2^(z - maximum)) pairs.
__device__ __forceinline__ void join(float& m, float& l, float om, float ol) {
  if (om == -INFINITY) return;                       // (a NaN goes on: it makes l NaN)
  const float n = m == -INFINITY ? om : fmaxf(m, om);
  l = l * exp2f(m - n) + ol * exp2f(om - n);
  m = n;
}

template <class E>
__global__ __launch_bounds__(kLossThreads) void k_loss_row(const CodLossArgs a) {
  using T = typename E::T;
  __shared__ float m_s[kLossThreads / 64], l_s[kLossThreads / 64];
  const int r = blockIdx.x, k = section_of(a, r);
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.stride;
  T* d = a.d_logits ? reinterpret_cast<T*>(a.d_logits) + r * a.d_stride : nullptr;
  if (k == 0) {                                      // uniform
    for (int i = threadIdx.x; d && i < a.vocab; i += kLossThreads) d[i] = E::store(0.f);
    if (threadIdx.x == 0) a.row_loss[r] = 0.f;
    return;
  }
  const int label = a.labels[r];
  const float x_label = label < a.vocab ? E::load(x[label]) : __builtin_nanf("");
  float m = -INFINITY, l = 0.f;
  for (int i = threadIdx.x; i < a.vocab; i += kLossThreads) join(m, l, E::load(x[i]) * kLog2e, 1.f);
  for (int off = 32; off > 0; off >>= 1) {
    const float om = __shfl_xor(m, off), ol = __shfl_xor(l, off);
    join(m, l, om, ol);
  }
  if ((threadIdx.x & 63) == 0) {
    m_s[threadIdx.x >> 6] = m;
    l_s[threadIdx.x >> 6] = l;
  }
  __syncthreads();
  m = -INFINITY;
  l = 0.f;
  for (int w = 0; w < kLossThreads / 64; ++w) join(m, l, m_s[w], l_s[w]);
  const float lse2 = m + log2f(l);
  if (threadIdx.x == 0) a.row_loss[r] = lse2 * kLn2 - x_label;
  if (!d) return;
  int n = 0;
  float w = a.grad_scale;
  if (a.weighted) {
    n = count_of(a, k);
    w *= a.weights[k - 1];
  } else {
    for (int q = 1; q <= a.n_sections; ++q) n += count_of(a, q);
  }
  w = label < a.vocab ? w / n : __builtin_nanf("");
  __syncthreads();                                   // (x[label] is read: d may be x)
  for (int i = threadIdx.x; i < a.vocab; i += kLossThreads) {
    const float p = exp2f(E::load(x[i]) * kLog2e - lse2);
    d[i] = E::store(w * (i == label ? p - 1.f : p));
  }
}

// Workgroup k - 1: subtask k's mean; the last one to end adds the means up.
__global__ __launch_bounds__(1024) void k_loss_mean(const CodLossArgs a) {
  __shared__ double s_s[16];
  __shared__ int last_s;
  const int k = blockIdx.x + 1;
  double s = 0.0;
  for (int r = threadIdx.x; r < a.rows; r += 1024)
    if (section_of(a, r) == k) s += a.row_loss[r];
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) s_s[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  for (int w = 0; w < 16; ++w) s += s_s[w];
  const int n = count_of(a, k);
  __hip_atomic_store(&a.loss[k], n ? (float)(s / n) : 0.f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  last_s = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  if (last_s != a.n_sections - 1) return;
  double total = 0.0;
  int64_t all = 0;
  for (int q = 1; q <= a.n_sections; ++q) {
    const double mean = __hip_atomic_load(&a.loss[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int c = count_of(a, q);
    total += a.weighted ? a.weights[q - 1] * mean : c * mean;
    all += c;
  }
  a.loss[0] = (float)(a.weighted ? total : all ? total / all : 0.0);
}

template <class E>
hipError_t launch_rows(const CodLossArgs& a, hipStream_t st) {
  k_loss_count<<<kLossCountBlocks, kLossThreads, 0, st>>>(a);
  if (a.rows > 0) k_loss_row<E><<<a.rows, kLossThreads, 0, st>>>(a);
  k_loss_mean<<<a.n_sections, 1024, 0, st>>>(a);
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
