// Plan of attention over packed COD rows.
//
// With c = j - k + 1 (the chain of packed row (k, j): the real token that ends
// its context), row (k, j) attends to the real tokens 0 .. c and to the mask
// rows (k', c + k' - 1), 2 <= k' <= k, of its chain.  Numbered by (c, k), the
// rows of a chain are neighbours and the context grows along the order: a tile
// of neighbours sees the same real tokens but for its own chains' ends, and
// beyond them only rows of the tile (or of the chain it begins in).  In the
// packed order (k, c) a tile of subtask k would need a run of every earlier
// subtask as well: 7 more key tiles, mostly masked, at K = 8.
//
// One workgroup per sample: a 64-bit mask of the subtasks present in every
// chain (LDS), a scan of their counts, and each row's place is its chain's
// start plus the number of lower subtasks in the mask.  Bound: latency, a few
// dependent passes over the rows of the longest sample: 10 us for 16 samples of
// up to 1024 tokens, 55 for one of 8193, once per batch; the tiles 8 us.
#include "train.h"

#include <algorithm>

namespace pard {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxChains = 8192;

// Inclusive sum over the workgroup's threads; *total: the last one's.
__device__ __forceinline__ int block_incl_scan(int x, int* wave_s, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(x, off);
    if (lane >= off) x += o;
  }
  if (lane == 63) wave_s[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    before += w < wave ? wave_s[w] : 0;
    all += wave_s[w];
  }
  __syncthreads();
  *total = all;
  return x + before;
}

__global__ __launch_bounds__(kPlanThreads) void k_cod_plan(const int32_t* section, const int32_t* column,
                                                            const int32_t* out_len, int n_chains, const CodPlanView v) {
  // dynamic LDS: subtasks present in each chain, its first position
  extern __shared__ unsigned long long mask_s[];
  int* start_s = reinterpret_cast<int*>(mask_s + n_chains);
  __shared__ int wave_s[kPlanThreads / 64];
  const int s = blockIdx.x, tid = threadIdx.x;
  const int off = (int)v.offsets[s], cap = (int)(v.offsets[s + 1] - v.offsets[s]);
  const int want = out_len[s], len = min(max(want, 0), cap);
  bool bad = want != len;
  for (int c = tid; c < n_chains; c += kPlanThreads) mask_s[c] = 0;
  __syncthreads();
  const int32_t* sec = section + off;
  const int32_t* col = column + off;
  int n_real = 0;
  for (int r = tid; r < len; r += kPlanThreads) {
    const int k = sec[r], j = col[r];
    // 64-bit: the columns may hold anything
    const int64_t c = (int64_t)j - k + 1;
    bool ok = k >= 1 && k <= kCodMaxSections && c >= 0 && c < n_chains && (k > 1 || j == r);
    if (r > 0) ok = ok && (sec[r - 1] < k || (sec[r - 1] == k && col[r - 1] < j));
    if (ok) atomicOr(&mask_s[c], 1ull << (k - 1));
    bad |= !ok;
    n_real += ok && k == 1;
  }
  __syncthreads();
  int total = 0;
  (void)block_incl_scan(n_real, wave_s, &n_real);
  const int per = (n_chains + kPlanThreads - 1) / kPlanThreads, c0 = tid * per;
  int count = 0;
  for (int c = c0; c < min(c0 + per, n_chains); ++c) {
    count += __popcll(mask_s[c]);
    bad |= mask_s[c] != 0 && !(mask_s[c] & 1);
  }
  int at = block_incl_scan(count, wave_s, &total) - count;
  for (int c = c0; c < min(c0 + per, n_chains); ++c) {
    start_s[c] = at;
    at += __popcll(mask_s[c]);
  }
  __syncthreads();
  // (a bad batch's places may be wrong, but are below its length)
  for (int r = tid; r < cap; r += kPlanThreads) {
    if (r >= len) {
      v.order[(size_t)off + r] = int4{r, 0, cap, r};
      continue;
    }
    const int k = sec[r], c = col[r] - k + 1;
    if (k < 1 || k > kCodMaxSections || c < 0 || c >= n_chains) continue;
    const unsigned long long m = mask_s[c];
    const int p = start_s[c] + __popcll(m & ((1ull << (k - 1)) - 1));
    v.order[(size_t)off + p] = int4{r, c + 1, start_s[c] + (int)(m & 1), start_s[c] + __popcll(m)};
    if (k == 1 && r == c) v.first[(size_t)off + c] = start_s[c];
  }
  if (tid == 0) v.samples[s] = CodSampleInfo{off, len, n_real, cap, len > 0 ? min(max(sec[len - 1], 1), kCodMaxSections) - 1 : 0};
  if (bad) *v.bad = 1;
}

// Tiles of all samples in two orders: those with the largest index in their
// sample first (as queries they see the most keys), and sample by sample, those
// with the most tiles first (as keys, the tiles of a sample read the same rows at
// the same time).
__global__ __launch_bounds__(kPlanThreads) void k_cod_tiles(int n_samples, int n_levels, const CodPlanView v) {
  extern __shared__ int level_s[];           // next free place of each level, and of the samples with so many tiles
  int* const size_s = level_s + n_levels;
  __shared__ int wave_s[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  auto tiles_of = [&](int s) { return (int)((v.offsets[s + 1] - v.offsets[s] + kCodTile - 1) / kCodTile); };
  for (int l = tid; l < n_levels; l += kPlanThreads) level_s[l] = 0;
  __syncthreads();
  for (int s = tid; s < n_samples; s += kPlanThreads) {
    const int n = tiles_of(s);
    if (n > 0) atomicAdd(&level_s[n - 1], 1);
  }
  __syncthreads();
  // tiles of the samples with more tiles
  {
    int carry = 0;
    for (int b = 0; b < n_levels; b += kPlanThreads) {
      const int l = n_levels - 1 - (b + tid), x = l >= 0 ? level_s[l] * (l + 1) : 0;
      int total;
      const int incl = block_incl_scan(x, wave_s, &total) + carry;
      if (l >= 0) size_s[l] = incl - x;
      carry += total;
    }
  }
  // samples with exactly l + 1 tiles -> samples with more than l -> tiles of
  // later levels: two scans from the last level down
  for (int pass = 0; pass < 2; ++pass) {
    int carry = 0;
    for (int b = 0; b < n_levels; b += kPlanThreads) {
      const int l = n_levels - 1 - (b + tid), x = l >= 0 ? level_s[l] : 0;
      int total;
      const int incl = block_incl_scan(x, wave_s, &total) + carry;
      if (l >= 0) level_s[l] = pass == 0 ? incl : incl - x;
      carry += total;
    }
    __syncthreads();
  }
  for (int s = tid >> 6; s < n_samples; s += kPlanThreads / 64) {
    const int n = tiles_of(s);
    const CodSampleInfo info = v.samples[s];
    if (n == 0) continue;                    // uniform
    int base = lane == 0 ? atomicAdd(&size_s[n - 1], n) : 0;
    base = __shfl(base, 0);
    for (int l = lane; l < n; l += 64) {
      const CodTileInfo t{info, s, l, 0};
      v.tiles[atomicAdd(&level_s[l], 1)] = t;
      v.by_sample[base + l] = t;
    }
  }
}

}  // namespace

size_t cod_plan_layout(int64_t rows, int n_samples, void* data, CodPlanView* v) {
  char* const base = static_cast<char*>(data);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += (bytes + 255) & ~(size_t)255;
    return p;
  };
  char* const order = take((size_t)rows * sizeof(int4));
  char* const first = take((size_t)rows * sizeof(int));
  char* const samples = take((size_t)n_samples * sizeof(CodSampleInfo));
  char* const tiles = take(((size_t)rows / kCodTile + n_samples) * sizeof(CodTileInfo));
  char* const by_sample = take(((size_t)rows / kCodTile + n_samples) * sizeof(CodTileInfo));
  char* const offsets = take(((size_t)n_samples + 1) * sizeof(int64_t));
  char* const bad = take(sizeof(int));
  if (v) {
    v->order = reinterpret_cast<int4*>(order);
    v->first = reinterpret_cast<int*>(first);
    v->samples = reinterpret_cast<CodSampleInfo*>(samples);
    v->tiles = reinterpret_cast<CodTileInfo*>(tiles);
    v->by_sample = reinterpret_cast<CodTileInfo*>(by_sample);
    v->offsets = reinterpret_cast<int64_t*>(offsets);
    v->bad = reinterpret_cast<int*>(bad);
  }
  return at;
}

hipError_t launch_cod_plan(const int32_t* section, const int32_t* column, const int32_t* out_len, int n_samples,
                           int max_region, const CodPlanView& v, hipStream_t st) {
  const int n_chains = std::min(kMaxChains, (max_region + 63) / 64 * 64);
  const int n_levels = (max_region + kCodTile - 1) / kCodTile;
  k_cod_plan<<<n_samples, kPlanThreads, (size_t)n_chains * 12, st>>>(section, column, out_len, n_chains, v);
  k_cod_tiles<<<1, kPlanThreads, (size_t)n_levels * 2 * sizeof(int), st>>>(n_samples, n_levels, v);
  return hipGetLastError();
}

}  // namespace pard
