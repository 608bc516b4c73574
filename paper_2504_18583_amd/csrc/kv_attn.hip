// Attention of a batch's new rows over a paged cache, on gfx950 MFMA.
//
// A sequence's rows and query heads of one key head are its pairs (row by row).
// A workgroup owns a tile of them and one share of the keys that its rows see;
// with a window these are the first tokens, then the keys from the first row's
// window on.  Only steps that some row does not see whole compare keys with rows.
// A tile of the products is S^T = K Q^T, online softmax in base 2, O^T += V^T P^T
// (softmax_step).  Which of two kernels runs, and how many pairs a tile has,
// follows from the pairs of a sequence (tile_pairs):
//   k_kv_few   16 or 32 pairs: every wavefront has all of them and a quarter of
//              the keys
//   k_kv_attn  64 or 128 pairs: the wavefronts share stages of 64 keys in LDS
// Work is shared out on the device, from lengths that only the device knows:
// from all sequences' stages follows the length of a share, and from the running
// number of shares the one that is a workgroup's.  Sequences of more than one
// share leave partial sums, which a last launch joins in the order of the keys.
//
// Bound.  Single tokens: memory (16 contexts of 8000 to 32 000 keys, 32 / 8 heads x
// 128: 255 us in bf16, 5.4 TB/s; 155 in e4m3, 4.6; 88 in e2m1, 4.1).  Verify
// passes: memory behind a chain of dependent reads (lengths, table, keys: 5 us of
// a workgroup's life) and the join (32 sequences of 512 to 1536 keys, 9 rows: 32
// us for 136 MB and 5 for the join).  Chunks: the SIMDs' issue (4096 rows at 4096,
// 32 / 8 heads x 128: 425 us, 970 TFLOP/s in bf16 and e4m3; x 64: 255 us in bf16, 267 in
// e2m1, 809 and 772: products 42 % of the SIMDs' cycles, other instructions 75 %, as
// the softmax of a score is the same for half the products; two chunks of 3641 and
// 2606 rows x 128 860 us: 43 and 45 %).  Within a window of 1024 a tile sees 18 stages,
// of which four compare, and a row of 150 makes 4.7 tiles: products 23 %, others 57.
// A wavefront per row and head, key by key, took 23.9 ms for the contexts in e4m3
// and 139 for the chunks.
#include "serve.h"

#include <algorithm>

#include "cod_attn_tile.h"
#include "kv_span.h"
#include "tensor_args.h"

namespace pard {
namespace {

using namespace cod;

constexpr int kStageKeys = 64;
constexpr int kMinKeys = 256;              // keys of a share at least
// Shares that all stages are cut into, about: what the chip holds at once, or
// twice that for the smallest tiles, up to 64 a tile (single tokens of 16 contexts of
// 20 000 keys, 512 and 1024 shares: e4m3 168 and 154 us, 64 dims in bf16 146 and
// 128; of one of 131 000 102 and 109; tiles of 32 pairs, 32 sequences of 8000
// keys in e4m3 192 and 229).
template <int QP>
constexpr int kShares = QP == 16 ? 1024 : 512;

// ---- sharing out ------------------------------------------------------------

// One sequence's work.
struct SeqWork {
  int row0, rows, len;                     // first row, rows, positions
  int tiles;                               // of QP pairs
  int stages;                              // of a tile, at most
};

template <int QP, int KEYS>
__device__ __forceinline__ SeqWork seq_work(const KvAttnArgs& a, int s) {
  SeqWork w{};
  if (s >= a.batch.n_seqs) return w;
  const int r0 = a.batch.row_start[s], r1 = a.batch.row_start[s + 1];
  w.row0 = min(max(r0, 0), a.batch.rows);
  w.rows = max(min(r1, a.batch.rows) - w.row0, 0);
  w.len = max(a.batch.kv_len[s], 0);
  w.tiles = (w.rows * a.group + QP - 1) / QP;
  int keys = min(max(w.len, 0), a.batch.cap);
  // (with a window: what a tile's rows see between them, and a partial stage)
  if (a.window) keys = (int)min((int64_t)keys, (int64_t)a.window + min(w.rows, QP / a.group + 2) + min(a.sinks, keys) + KEYS);
  w.stages = w.tiles ? max((keys + KEYS - 1) / KEYS, 1) : 0;
  return w;
}

// Inclusive sums over a wavefront's lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ int shifted(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int scan(int x) {
  x += shifted<0x111, 0xF>(x);             // row_shr 1, 2, 4, 8
  x += shifted<0x112, 0xF>(x);
  x += shifted<0x114, 0xF>(x);
  x += shifted<0x118, 0xF>(x);
  x += shifted<0x142, 0xA>(x);             // row_bcast 15, 31
  x += shifted<0x143, 0xC>(x);
  return x;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float plus_shifted(float x) {
  return x + __uint_as_float((uint32_t)shifted<CTRL, ROWS>((int)__float_as_uint(x)));
}
__device__ __forceinline__ float sum_lanes(float x) {
  x = plus_shifted<0x111, 0xF>(x);
  x = plus_shifted<0x112, 0xF>(x);
  x = plus_shifted<0x114, 0xF>(x);
  x = plus_shifted<0x118, 0xF>(x);
  x = plus_shifted<0x142, 0xA>(x);
  x = plus_shifted<0x143, 0xC>(x);
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}

__device__ __forceinline__ int shares_of(const SeqWork& w, int share) { return (w.stages + share - 1) / share; }

// The length of a share from all stages and tiles: kShares of it hold all stages,
// or half as many where there are so many tiles that only the longest need be
// cut.  (Up to kShares tiles are counted.)
template <int QP, int KEYS>
__device__ __forceinline__ int share_of(const KvAttnArgs& a, float stages, int tiles) {
  const int all = min(max(64 * min(tiles * a.cache.n_kv, 1024), 512), kShares<QP>);
  const float shares = tiles * a.cache.n_kv >= all / 2 ? all / 2 : all;
  return max(kMinKeys / KEYS, (int)fminf(ceilf(stages * a.cache.n_kv / shares), 1 << 24));
}

// Sequences that every wavefront adds up by itself, one to a lane; more have a
// plan (decode of 300 keys each, 8 key heads x 128, by steps of 64 and with a
// plan: 256 sequences 86 and 73 us, 4096 5358 and 957).
constexpr int kMaxAlone = 64;

template <int QP, int KEYS>
__device__ __forceinline__ int share_length(const KvAttnArgs& a, const SeqWork& mine) {
  if (a.plan) return a.plan[0];                        // uniform
  const int tiles = __builtin_amdgcn_readlane(scan(min(mine.tiles, kShares<QP>)), 63);
  return share_of<QP, KEYS>(a, sum_lanes((float)mine.tiles * mine.stages), min(tiles, kShares<QP>));
}

// The first sequence whose running number `upto` is past `left`, 64 candidates
// at a time (n_seqs: none), and its work.
struct Found {
  SeqWork w;
  int seq;
};
template <int QP, int KEYS>
__device__ __forceinline__ Found search(const KvAttnArgs& a, const int* upto, int left, int lane) {
  int lo = 0, n = a.batch.n_seqs;
  while (n > 64) {                                     // uniform
    const int step = (n + 63) / 64;
    const uint64_t past = __ballot(upto[min(lo + (lane + 1) * step, lo + n) - 1] > left);
    if (!past) return Found{SeqWork{}, a.batch.n_seqs};
    const int l = __builtin_ctzll(past);
    n = min(step, n - l * step);
    lo += l * step;
  }
  const SeqWork w = seq_work<QP, KEYS>(a, lo + min(lane, n - 1));
  const uint64_t past = __ballot(lane < n && upto[lo + min(lane, n - 1)] > left);
  if (!past) return Found{SeqWork{}, a.batch.n_seqs};
  const int l = __builtin_ctzll(past);
  auto from = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
  return Found{SeqWork{from(w.row0), from(w.rows), from(w.len), from(w.tiles), from(w.stages)}, lo + l};
}

struct Item {
  SeqWork w;
  int seq, tile, split, splits;            // splits 0: no such item
  int slot;                                // of its partial sums
  // whether the numbers fit together: they do if row_start ascends
  __device__ __forceinline__ bool valid(const KvAttnArgs& a) const {
    return tile >= 0 && tile < w.tiles && split >= 0 && (splits == 1 || (slot >= 0 && slot < a.slots));
  }
};

// Item `left` of a key head: a tile's shares first, then tiles (the last first:
// they see the most keys), then sequences.
template <int QP, int KEYS>
__device__ __forceinline__ Item find_item(const KvAttnArgs& a, const SeqWork& own, int share, int left, int kvh, int lane) {
  Item it{};
  if (a.plan) {                                        // uniform
    const Found f = search<QP, KEYS>(a, a.plan + 1, left, lane);
    if (f.seq == a.batch.n_seqs) return it;
    it.w = f.w;
    it.seq = f.seq;
    it.splits = shares_of(f.w, share);
    const int mine = left - (f.seq ? a.plan[f.seq] : 0);
    it.tile = f.w.tiles - 1 - mine / it.splits;
    it.split = mine % it.splits;
    it.slot = ((f.seq ? a.plan[a.batch.n_seqs + f.seq] : 0) + mine) * a.cache.n_kv + kvh;
    return it;
  }
  const int n = shares_of(own, share), items = own.tiles * n, split = n > 1 ? items : 0;
  const int upto = scan(items), slots_upto = scan(split);
  const uint64_t past = __ballot(upto > left);
  if (!past) return it;
  const int l = __builtin_ctzll(past);
  auto from = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
  it.w = SeqWork{from(own.row0), from(own.rows), from(own.len), from(own.tiles), from(own.stages)};
  const int mine = left - (from(upto) - from(items));
  it.seq = l;
  it.splits = from(n);
  it.tile = it.w.tiles - 1 - mine / it.splits;
  it.split = mine % it.splits;
  it.slot = (from(slots_upto) - from(split) + mine) * a.cache.n_kv + kvh;
  return it;
}

// Running numbers of a large batch, by one workgroup ahead of the others: the
// length of a share, then up to each sequence its shares, those that leave
// partial sums, and the pairs of split sequences.
template <int QP, int KEYS>
__global__ __launch_bounds__(1024) void k_kv_plan(const KvAttnArgs a) {
  __shared__ float f_sum[16];
  __shared__ int n_sum[16], i_sum[3][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.batch.n_seqs;
  float total = 0.f;
  int tiles = 0;
  for (int s = tid; s < n; s += 1024) {
    const SeqWork w = seq_work<QP, KEYS>(a, s);
    total += (float)w.tiles * w.stages;
    tiles = min(tiles + w.tiles, kShares<QP>);
  }
  total = sum_lanes(total);
  tiles = __builtin_amdgcn_readlane(scan(tiles), 63);
  if (lane == 0) f_sum[wave] = total, n_sum[wave] = tiles;
  __syncthreads();
  total = 0.f;
  tiles = 0;
  for (int w = 0; w < 16; ++w) total += f_sum[w], tiles = min(tiles + n_sum[w], kShares<QP>);
  const int share = share_of<QP, KEYS>(a, total, tiles);
  if (tid == 0) a.plan[0] = share;
  int before[3] = {};
  for (int s0 = 0; s0 < n; s0 += 1024) {               // uniform
    const SeqWork w = seq_work<QP, KEYS>(a, s0 + tid);
    const int k = shares_of(w, share), items = w.tiles * k;
    const int x[3] = {items, k > 1 ? items : 0, k > 1 ? w.rows * a.group : 0};
    int upto[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      upto[i] = scan(x[i]);
      if (lane == 63) i_sum[i][wave] = upto[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int all = 0;
      for (int v = 0; v < 16; ++v) {
        if (v < wave) upto[i] += i_sum[i][v];
        all += i_sum[i][v];
      }
      if (s0 + tid < n) a.plan[1 + i * n + s0 + tid] = before[i] + upto[i];
      before[i] += all;
    }
    __syncthreads();
  }
}

// ---- keys and values into LDS --------------------------------------------------

// A wavefront's 16 keys of a stage on their way: 16 bits, none; else a lane
// holds row lane % 16, its parts g = lane / 16, g + 4, ..
template <int HD, class M, int DT>
struct Staged {};
template <int HD, class M>
struct Staged<HD, M, PARD_E4M3> {
  u32x4 x[HD / 64];                                   // elements 16 g + 64 h ..
  uint32_t scale;
  __device__ __forceinline__ void load(const char* row, const uint8_t* scales, int g) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) x[h] = *reinterpret_cast<const u32x4*>(row + g * 16 + h * 64);
    if constexpr (HD == 128) scale = *reinterpret_cast<const uint32_t*>(scales);
    else scale = *reinterpret_cast<const uint16_t*>(scales);
  }
  __device__ __forceinline__ void store(u32x4* block, int row, int g) const {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) {
      const float s = __uint_as_float((scale >> (16 * h + 8 * (g >> 1)) & 255) << 23);
      u32x4* const at = block + (g + 4 * h) * 32 + row * 2;
      at[0] = u32x4{M::fp8(x[h][0], s, false), M::fp8(x[h][0], s, true), M::fp8(x[h][1], s, false), M::fp8(x[h][1], s, true)};
      at[1] = u32x4{M::fp8(x[h][2], s, false), M::fp8(x[h][2], s, true), M::fp8(x[h][3], s, false), M::fp8(x[h][3], s, true)};
    }
  }
};
template <int HD, class M>
struct Staged<HD, M, PARD_E2M1> {
  uint32_t x[HD / 32];                                // elements HD / 4 g ..
  uint32_t scale;
  __device__ __forceinline__ void load(const char* row, const uint8_t* scales, int g) {
    if constexpr (HD == 128) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(row + g * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v[i];
      scale = scales[g];
    } else {
      const u32x2 v = *reinterpret_cast<const u32x2*>(row + g * 8);
      x[0] = v[0], x[1] = v[1];
      scale = scales[g >> 1];
    }
  }
  __device__ __forceinline__ void store(u32x4* block, int row, int g) const {
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
      block[(g * (HD / 64) + i / 2) * 32 + row * 2 + i % 2] =
          u32x4{M::template fp4<0>(x[i], s), M::template fp4<1>(x[i], s), M::template fp4<2>(x[i], s), M::template fp4<3>(x[i], s)};
  }
};

// Conversions of the small types to an operand's type, two elements at a time.
struct KvBF16 : MmaBF16 {
  static __device__ __forceinline__ uint32_t fp8(uint32_t v, float s, bool hi) {
    return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, s, false));
  }
  template <int BYTE>
  static __device__ __forceinline__ uint32_t fp4(uint32_t v, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, BYTE));
  }
};
struct KvF16 : MmaF16 {
  static __device__ __forceinline__ uint32_t fp8(uint32_t v, float s, bool hi) {
    return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, s, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, s, false));
  }
  template <int BYTE>
  static __device__ __forceinline__ uint32_t fp4(uint32_t v, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, s, BYTE));
  }
};

// At most N loads still in flight.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x0f70 | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}

// Zeros in the place of 16 keys without a page.
template <int HD>
__device__ __forceinline__ void clear_block(u32x4* block, int lane) {
#pragma unroll
  for (int i = 0; i < kBlockUnits<HD>; i += 64) block[i + lane] = u32x4{0, 0, 0, 0};
  asm volatile("" ::: "memory");
}

// Everyone's LDS accesses are done; loads stay in flight.
__device__ __forceinline__ void meet_with_loads() {
  __builtin_amdgcn_s_waitcnt(0xc07f);                  // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Partial sums of a tile: [QP][HD] of O, [QP] maxima, [QP] sums.
template <int HD, int QP>
constexpr int kRecord = QP * (HD + 2);

// Wavefronts a SIMD, as LDS and registers allow.  (Two tiles of pairs x 64 dims in 16
// bits: four keep 12 registers in memory, and chunks of 4096 rows at 4096 took 255 us
// for 276 with three, of 1000 at 9000 193 for 189.  In 8 and 4 bits four spill more:
// 101 us for 83 in the window.)
template <int HD, int NQ, int DT>
constexpr int kResident = NQ == 1 ? 4 : HD == 128 ? 2 : kv_scale_bytes(DT, HD) ? 3 : 4;

// Many pairs: 64 NQ to a workgroup.  A stage of 64 keys lies in one of two LDS
// buffers, the next one in flight during the current one.
//   * 16 bits: LDS-DMA, 16 keys to a wavefront; pages have 16 keys or more, so
//     such a block lies in one page, whose table entry is read two stages ahead.
//   * 8 and 4 bits: bytes and scales into registers, two stages ahead, widened into
//     LDS at the end of a stage (v_cvt_scalef32_*), so that everything behind is
//     the same.
// KH wavefronts share 16 NQ pairs, each with its part of a stage's keys: with one
// tile of pairs (NQ 1) a stage's dependent steps, not its bytes, were the time, and
// two half as long ones run beside each other (verify pass of 32 sequences 40 and 33 us,
// before the join).  Three stages ahead in one workgroup a CU (four buffers) took
// 39, and two workgroups with two buffers 33.
template <int HD, int NQ, int KH, class M, int DT>
__global__ __launch_bounds__(256 * KH, (kResident<HD, NQ, DT>)) void k_kv_attn(const KvAttnArgs a) {
  constexpr int QW = 16 * NQ, QP = 4 * QW;             // pairs of a wavefront, of the workgroup
  constexpr int NB = 4 / KH;                           // blocks of 16 keys of a wavefront
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  constexpr int RB = kv_row_bytes(DT, HD), SB = kv_scale_bytes(DT, HD);
  // stages in flight beside the current one; loads of a stage
  constexpr int AHEAD = SB ? 2 : 1, LOADS = 2 * KS / KH;
  // a stage: four blocks of K, four of V; two arrays of their own (the
  // compiler's waits before an LDS read cover the loads into that array only)
  __shared__ __attribute__((aligned(16))) u32x4 b0[8 * BU], b1[8 * BU];
  __shared__ int any_bad;                              // a stage of this item has a key without a page
  __shared__ float ml[KH == 2 ? 4 : 1][2][16];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  // its pairs (and the block of every stage that it loads), its part of the keys
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, part = __builtin_amdgcn_readfirstlane(tid >> 8);
  const KvBatchView& b = a.batch;
  const SeqWork own = a.plan ? SeqWork{} : seq_work<QP, kStageKeys>(a, lane);   // of sequence `lane`
  const int share = share_length<QP, kStageKeys>(a, own);
  // key heads fastest: with 8 of them each keeps to an XCD and its L2
  const int kvh = blockIdx.x % a.cache.n_kv;
  for (int u = blockIdx.x / a.cache.n_kv;; u += gridDim.x / a.cache.n_kv) {
    const Item it = find_item<QP, kStageKeys>(a, own, share, u, kvh, lane);
    if (it.splits == 0) return;                        // uniform: past the last item
    if (!it.valid(a)) continue;                        // uniform (row_start does not ascend)
    __syncthreads();                                   // (the item before has read LDS)
    if (tid == 0) any_bad = 0;
    __syncthreads();
    const int n_pairs = it.w.rows * a.group, pair0 = it.tile * QP;
    const int pos0 = it.w.len - it.w.rows;             // of the sequence's first row
    auto row_of = [&](int pair) { return quotient(min(pair, n_pairs - 1), a.by_group); };

    // what the tile's rows see
    const int pos_lo = pos0 + row_of(pair0), pos_hi = pos0 + row_of(pair0 + QP - 1);
    const KvSpan sp = kv_span(pos_lo, pos_hi, b.cap, a.window, a.sinks, kStageKeys);
    const int lo = sp.lo, last = sp.last, a_last = sp.a_last, from = sp.from, n_a = sp.n_a, n_all = sp.n_all;
    const int st0 = (int)((int64_t)n_all * it.split / it.splits), st1 = (int)((int64_t)n_all * (it.split + 1) / it.splits);

    // this wavefront's 16 keys of a stage: blocks past a run repeat its last key
    auto block_of = [&](int st) __attribute__((always_inline)) { return kv_run(sp, kStageKeys, st, wave * 16); };
    const int32_t* const table = b.table + (int64_t)it.seq * b.max_pages;
    auto entry_of = [&](int st) __attribute__((always_inline)) {
      const KvRun k = block_of(st);
      return table[min(k.key, k.high) >> a.cache.page_log2];
    };
    struct Parts { Staged<HD, M, DT> x[2 / KH]; };     // of K and V; with two parts, the first's wavefronts load K
    Parts p0, p1;
    auto load = [&](Parts& p, u32x4* buf, int st, int entry) __attribute__((always_inline)) {
      const KvRun k = block_of(st);
      int page = __builtin_amdgcn_readfirstlane(entry);
      const bool none = (uint32_t)page >= (uint32_t)a.cache.n_pages;         // uniform
      if (none) {
        page = 0;
        if (lane == 0) any_bad = 1;
      }
      const int r = SB ? c16 : block_row(lane);
      const int place = max(min(k.key + r, k.high), k.low) & ((1 << a.cache.page_log2) - 1);
      const int64_t slot = (((int64_t)page * a.cache.n_kv + kvh) << a.cache.page_log2) + place;
#pragma unroll
      for (int i = 0; i < 2 / KH; ++i) {
        const bool is_v = KH == 2 ? part : i;
        const char* const src = (is_v ? a.cache.v : a.cache.k) + slot * RB;
        if constexpr (SB) p.x[i].load(src, (is_v ? a.cache.v_scale : a.cache.k_scale) + slot * SB, g4);
        else load_block<HD>(src + block_byte(lane), buf + (4 * is_v + wave) * BU);
      }
      if (none) {                                      // (what page 0 holds reaches nobody)
        if constexpr (SB) {
          p = Parts{};
        } else {
          wait_loads<0>();
#pragma unroll
          for (int i = 0; i < 2 / KH; ++i) clear_block<HD>(buf + (4 * (KH == 2 ? part : i) + wave) * BU, lane);
        }
      }
    };
    auto widen = [&](const Parts& p, u32x4* buf) __attribute__((always_inline)) {
      if constexpr (SB) {
#pragma unroll
        for (int i = 0; i < 2 / KH; ++i) p.x[i].store(buf + (4 * (KH == 2 ? part : i) + wave) * BU, c16, g4);
      }
    };

    // this lane's pairs: those past the sequence repeat its last and are not stored
    const int w_pair = pair0 + wave * QW;
    const bool idle = w_pair >= n_pairs;               // uniform: no pairs of its own
    const int w_lo = pos0 + row_of(w_pair), w_hi = pos0 + row_of(w_pair + QW - 1);
    u32x4 q[NQ][KS];
    float m[NQ], l[NQ];
    f32x4 o[NQ][DB];
    int pos[NQ];
    // table entries of the stages to be loaded next (any stage's may be read),
    // read as many stages before their loads that these wait for nothing newer
    int e0 = 0, e1 = 0, e2 = 0, e3 = 0;
    if (st0 < st1) {                                   // uniform
      e0 = entry_of(st0), e1 = entry_of(st0 + 1), e2 = entry_of(st0 + 2), e3 = entry_of(st0 + 3);
    }
    const uint32_t sign = scale_sign(a.scale);
    const float scale2 = base2_scale(a.scale);
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int pair = min(w_pair + t * 16 + c16, n_pairs - 1), r = quotient(pair, a.by_group);
      pos[t] = pos0 + r;
      const char* src = at(a.q, it.w.row0 + r, kvh * a.group + remainder(pair, r, a.by_group)) + g4 * 16;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[t][ks] = *reinterpret_cast<const u32x4*>(src + ks * 64);
      m[t] = -1e30f;
      l[t] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[t][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (st0 < st1) {                                   // uniform
      load(p0, b0, st0, e0);
      if (st0 + 1 < st1) load(p1, b1, st0 + 1, e1);
    }
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[t][ks][i] ^= sign;

    auto compute = [&](int st, const u32x4* cur) __attribute__((always_inline)) {
      // (kv_run, spelled out: called here it costs the compiler 170 scalar spills)
      const bool in_a = st < n_a;
      const int key0 = (in_a ? st * kStageKeys : from + (st - n_a) * kStageKeys) + part * NB * 16, end = key0 + NB * 16 - 1;
      const int low = in_a ? 0 : lo, high = in_a ? a_last : last;
      const int gone = a.window ? w_lo - a.window : -1;  // keys up to it are no row's but first tokens
      if (idle || key0 > min(w_hi, high) || (end <= gone && key0 >= a.sinks)) return;   // uniform: no row of this wavefront sees them
      const u32x4* const kc = cur + part * NB * BU;
      const u32x4* const vc = kc + 4 * BU;
      f32x4 sc[NQ][NB];
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) sc[t][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 kf = rows_frag(kc + kb * BU, ks, lane);
#pragma unroll
          for (int t = 0; t < NQ; ++t) sc[t][kb] = M::mma(kf, q[t][ks], sc[t][kb]);
        }
      const bool bad = any_bad;
      const bool whole = key0 >= low && end <= min(w_lo, high) && (!a.window || key0 > w_hi - a.window || end < a.sinks);
      if (bad || !whole) {                             // uniform
        // (first tokens beside the window's keys are a run of their own or, where the
        // two meet, the start of the one run)
        const bool both = a.window && !in_a && a.sinks > low;
        int span0[NQ];
        uint32_t span[NQ];                             // keys span0 .. span0 + span - 1
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          span0[t] = a.window && !in_a ? max(low, pos[t] - a.window + 1) : low;
          span[t] = (uint32_t)max(min(pos[t], high) + 1 - span0[t], 0);
        }
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
          const int k16 = key0 + kb * 16;
          const bool none = bad && (uint32_t)table[min(k16, high) >> a.cache.page_log2] >= (uint32_t)a.cache.n_pages;
#pragma unroll
          for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = k16 + g4 * 4 + i;
              if (none) sc[t][kb][i] = __uint_as_float(0x7fc00000u);
              if ((uint32_t)(key - span0[t]) >= span[t] && !(both && key < min(a.sinks, pos[t] + 1))) sc[t][kb][i] = -INFINITY;
            }
        }
      }
      u32x4 pf[NQ][NB / 2];
      softmax_step<NQ, NB, DB, M>(sc, m, l, o, pf, scale2);
#pragma unroll
      for (int tt = 0; tt < NB / 2; ++tt)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u32x4 vf = cols_frag<HD>(vc + 2 * tt * BU, db, lane);
#pragma unroll
          for (int t = 0; t < NQ; ++t) o[t][db] = M::mma(vf, pf[t][tt], o[t][db]);
        }
    };
    // One stage; entry: of stage st + AHEAD, loaded into nxt (16 bits) or p (then
    // q1, the next stage, is widened into nxt).
    auto stage = [&](int st, const u32x4* cur, u32x4* nxt, int& entry, Parts& p, const Parts& q1) __attribute__((always_inline)) {
      // this wavefront's loads of the stage are in LDS, and its LDS accesses done;
      // then everyone's
      if constexpr (SB) meet_with_loads();
      else wait_and_meet();
      if (st + AHEAD < st1) {                          // uniform
        load(p, nxt, st + AHEAD, entry);
        entry = entry_of(st + AHEAD + 2);
      }
      __builtin_amdgcn_sched_barrier(0);
      compute(st, cur);
      if (SB && st + 1 < st1) widen(q1, nxt);
    };
    if constexpr (SB) {
      if (st0 < st1) widen(p0, b0);
      for (int st = st0; st < st1; st += 2) {          // uniform
        stage(st, b0, b1, e2, p0, p1);
        if (st + 1 < st1) stage(st + 1, b1, b0, e3, p1, p0);
      }
    } else {
      // (the second stage's loads stay in flight during the first)
      if (st0 < st1) {
        if (st0 + 1 < st1) wait_loads<LOADS>();
        else wait_loads<0>();
        meet_with_loads();
        compute(st0, b0);
      }
      for (int st = st0 + 1; st < st1; st += 2) {
        stage(st, b1, b0, e2, p0, p0);
        if (st + 1 < st1) stage(st + 1, b0, b1, e3, p0, p0);
      }
    }

    // the second part's sums are added to the first's
    float sums[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) sums[t] = sum4g(l[t]);
    if constexpr (KH == 2) {
      static_assert(NQ == 1, "one tile of pairs");
      __syncthreads();                                 // (LDS is no longer read)
      if (part == 1) {
#pragma unroll
        for (int db = 0; db < DB; ++db) b0[(wave * DB + db) * 64 + lane] = __builtin_bit_cast(u32x4, o[0][db]);
        if (g4 == 0) ml[wave][0][c16] = m[0], ml[wave][1][c16] = sums[0];
      }
      __syncthreads();
      if (part == 1) continue;                         // uniform by wavefront: the barriers of the next item meet again
      const float m1 = ml[wave][0][c16], top = fmaxf(m[0], m1);
      const float f0 = __builtin_amdgcn_exp2f(m[0] - top), f1 = __builtin_amdgcn_exp2f(m1 - top);
      m[0] = top;
      sums[0] = sums[0] * f0 + ml[wave][1][c16] * f1;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[0][db] = o[0][db] * f0 + __builtin_bit_cast(f32x4, b0[(wave * DB + db) * 64 + lane]) * f1;
    }

    // lane (c16, g4) holds elements 16 db + 4 g4 .. + 3 of pair 16 t + c16
    const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int pair = w_pair + t * 16 + c16, in_tile = wave * QW + t * 16 + c16;
      float sum = sums[t];
      if (pair >= n_pairs) continue;
      if (pos[t] >= b.cap) sum = nan;                  // (past the table)
      if (it.splits > 1) {                             // uniform
        float* const rec = static_cast<float*>(a.work) + (int64_t)it.slot * kRecord<HD, QP>;
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(rec + in_tile * HD + db * 16 + g4 * 4) = o[t][db];
        if (g4 == 0) rec[QP * HD + in_tile] = m[t], rec[QP * HD + QP + in_tile] = sum;
        continue;
      }
      const int r = quotient(pair, a.by_group), head = kvh * a.group + remainder(pair, r, a.by_group), row = it.w.row0 + r;
      const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);   // (1 ulp of float32, before the rounding to 16 bits)
      char* const dst = at(a.out, row, head) + g4 * 8;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const f32x4 v = o[t][db] * inv;
        *reinterpret_cast<u32x2*>(dst + db * 32) = u32x2{M::pack(v[0], v[1]), M::pack(v[2], v[3])};
      }
      if (a.lse && g4 == 0)
        a.lse[(int64_t)head * b.rows + row] = sum == 0.f ? -INFINITY : (m[t] + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// Few pairs: a workgroup owns 16 NT of them, each of its wavefronts all of these
// against a quarter of the keys, 32 of every stage of 128, so that a token's
// bytes pass through one wavefront only and no wavefront waits for another
// until the end.  K goes straight into operand registers (8 and 4 bits:
// a lane's 16 bytes are elements next to each other, and Q's are put in the same
// order), V through the wavefront's own LDS, which transposes it; the next tile
// is in flight during the current one.  (16 contexts in e4m3 with the wavefronts
// around shared stages: 206 us against 169 then.)  Four tiles of 16 pairs (NT 4)
// need 500 registers and took 76 us for the 32 sequences' verify pass.
constexpr int kFewKeys = 128;

// K of a block of 16 keys as operands: of step s, lane (c16, g4) holds key c16's
// elements first(s, g4) .. + 7.
template <int HD, class M, int DT>
struct Keys {
  u32x4 x[HD / 32];
  static __device__ __forceinline__ int first(int s, int g) { return 32 * s + 8 * g; }
  __device__ __forceinline__ void load(const char* row, const uint8_t*, int g) {
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) x[s] = *reinterpret_cast<const u32x4*>(row + s * 64 + g * 16);
  }
  __device__ __forceinline__ u32x4 frag(int s) const { return x[s]; }
};
template <int HD, class M>
struct Keys<HD, M, PARD_E4M3> {
  u32x4 x[HD / 64];
  uint32_t scale;
  static __device__ __forceinline__ int first(int s, int g) { return 64 * (s / 2) + 16 * g + 8 * (s % 2); }
  __device__ __forceinline__ void load(const char* row, const uint8_t* scales, int g) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) x[h] = *reinterpret_cast<const u32x4*>(row + h * 64 + g * 16);
    if constexpr (HD == 128) scale = *reinterpret_cast<const uint32_t*>(scales) >> (8 * (g >> 1));
    else scale = *reinterpret_cast<const uint16_t*>(scales) >> (8 * (g >> 1));
  }
  __device__ __forceinline__ u32x4 frag(int s) const {
    const float f = __uint_as_float((scale >> (16 * (s / 2)) & 255) << 23);
    const uint32_t a = x[s / 2][2 * (s % 2)], b = x[s / 2][2 * (s % 2) + 1];
    return u32x4{M::fp8(a, f, false), M::fp8(a, f, true), M::fp8(b, f, false), M::fp8(b, f, true)};
  }
};
template <int HD, class M>
struct Keys<HD, M, PARD_E2M1> {
  uint32_t x[HD / 32];
  uint32_t scale;
  static __device__ __forceinline__ int first(int s, int g) { return HD / 4 * g + 8 * s; }
  __device__ __forceinline__ void load(const char* row, const uint8_t* scales, int g) {
    if constexpr (HD == 128) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(row + g * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v[i];
      scale = scales[g];
    } else {
      const u32x2 v = *reinterpret_cast<const u32x2*>(row + g * 8);
      x[0] = v[0], x[1] = v[1];
      scale = scales[g >> 1];
    }
  }
  __device__ __forceinline__ u32x4 frag(int s) const {
    const float f = __uint_as_float(scale << 23);
    return u32x4{M::template fp4<0>(x[s], f), M::template fp4<1>(x[s], f), M::template fp4<2>(x[s], f), M::template fp4<3>(x[s], f)};
  }
};

template <int HD, int NT, class M, int DT>
__global__ __launch_bounds__(256, 2) void k_kv_few(const KvAttnArgs a) {
  constexpr int QP = 16 * NT;
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  constexpr int RB = kv_row_bytes(DT, HD), SB = kv_scale_bytes(DT, HD);
  constexpr int NEXT = 4 * KS;                         // 16 bits: loads of a tile
  // V of a tile by wavefront; 16 bits: of the next one too
  __shared__ __attribute__((aligned(16))) u32x4 v0[8 * BU], v1[SB ? 1 : 8 * BU];
  __shared__ float ml[4][2][16];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KvBatchView& b = a.batch;
  const SeqWork own = a.plan ? SeqWork{} : seq_work<QP, kFewKeys>(a, lane);     // of sequence `lane`
  const int share = share_length<QP, kFewKeys>(a, own);
  const int kvh = blockIdx.x % a.cache.n_kv;           // (as k_kv_attn)
  for (int u = blockIdx.x / a.cache.n_kv;; u += gridDim.x / a.cache.n_kv) {
    const Item it = find_item<QP, kFewKeys>(a, own, share, u, kvh, lane);
    if (it.splits == 0) return;                        // uniform: past the last item
    if (!it.valid(a)) continue;                        // uniform (row_start does not ascend)
    const int n_pairs = it.w.rows * a.group, pair0 = it.tile * QP;
    const int pos0 = it.w.len - it.w.rows;
    auto row_of = [&](int pair) { return quotient(min(pair, n_pairs - 1), a.by_group); };
    const int pos_lo = pos0 + row_of(pair0), pos_hi = pos0 + row_of(pair0 + QP - 1);
    const KvSpan sp = kv_span(pos_lo, pos_hi, b.cap, a.window, a.sinks, kFewKeys);
    const int n_all = sp.n_all;
    const int st0 = (int)((int64_t)n_all * it.split / it.splits), st1 = (int)((int64_t)n_all * (it.split + 1) / it.splits);

    // this wavefront's 32 keys of a stage
    auto tile_of = [&](int st) __attribute__((always_inline)) { return kv_run(sp, kFewKeys, st, wave * 32); };
    const int32_t* const table = b.table + (int64_t)it.seq * b.max_pages;
    struct Entries { int e[2]; };
    auto entries_of = [&](int st) __attribute__((always_inline)) {
      const KvRun k = tile_of(st);
      return Entries{{table[min(k.key, k.high) >> a.cache.page_log2], table[min(k.key + 16, k.high) >> a.cache.page_log2]}};
    };
    struct Loaded {
      Keys<HD, M, DT> k[2];
      Staged<HD, M, DT> v[2];
      bool none[2];                                    // blocks without a page
    };
    auto load = [&](Loaded& d, u32x4* vbuf, int st, const Entries& e) __attribute__((always_inline)) {
      const KvRun k = tile_of(st);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int page = __builtin_amdgcn_readfirstlane(e.e[i]);
        d.none[i] = (uint32_t)page >= (uint32_t)a.cache.n_pages;
        page = d.none[i] ? 0 : page;
        const int64_t base = ((int64_t)page * a.cache.n_kv + kvh) << a.cache.page_log2;
        auto place = [&](int r) { return max(min(k.key + 16 * i + r, k.high), k.low) & ((1 << a.cache.page_log2) - 1); };
        const int64_t slot = base + place(c16);
        d.k[i].load(a.cache.k + slot * RB, SB ? a.cache.k_scale + slot * SB : nullptr, g4);
        if constexpr (SB) d.v[i].load(a.cache.v + slot * RB, a.cache.v_scale + slot * SB, g4);
      }
      if constexpr (!SB) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int page = d.none[i] ? 0 : __builtin_amdgcn_readfirstlane(e.e[i]);
          const int64_t base = ((int64_t)page * a.cache.n_kv + kvh) << a.cache.page_log2;
          const int place = max(min(k.key + 16 * i + block_row(lane), k.high), k.low) & ((1 << a.cache.page_log2) - 1);
          load_block<HD>(a.cache.v + (base + place) * RB + block_byte(lane), vbuf + (wave * 2 + i) * BU);
        }
      }
      if (d.none[0] || d.none[1]) {                    // uniform (what page 0 holds reaches nobody)
        if constexpr (!SB) wait_loads<0>();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (!d.none[i]) continue;
          if constexpr (SB) d.v[i] = Staged<HD, M, DT>{};
          else clear_block<HD>(vbuf + (wave * 2 + i) * BU, lane);
        }
      }
    };

    Loaded d0, d1;
    Entries next{};
    // (a run's last stage may have no keys for this wavefront: such a tile is skipped)
    auto here = [&](int st) __attribute__((always_inline)) { const KvRun k = tile_of(st); return k.key <= k.high; };
    Entries now{};
    if (st0 < st1) {                                   // uniform
      now = entries_of(st0);
      if (st0 + 1 < st1) next = entries_of(st0 + 1);
    }
    u32x4 q[NT][KS];
    float m[NT], l[NT];
    f32x4 o[NT][DB];
    int pos[NT];
    const uint32_t sign = scale_sign(a.scale);
    const float scale2 = base2_scale(a.scale);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int pair = min(pair0 + t * 16 + c16, n_pairs - 1), r = quotient(pair, a.by_group);
      pos[t] = pos0 + r;
      const char* src = at(a.q, it.w.row0 + r, kvh * a.group + remainder(pair, r, a.by_group));
#pragma unroll
      for (int s = 0; s < KS; ++s) q[t][s] = *reinterpret_cast<const u32x4*>(src + 2 * Keys<HD, M, DT>::first(s, g4));
      m[t] = -1e30f;
      l[t] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[t][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (st0 < st1) load(d0, v0, st0, now);             // uniform
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[t][s][i] ^= sign;

    auto tile = [&](int st, Loaded& d, u32x4* vbuf, Loaded& dn, u32x4* vnext) __attribute__((always_inline)) {
      const bool more = st + 1 < st1;
      __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0): the tile before has left LDS
      asm volatile("" ::: "memory");
      if (more) {                                      // uniform
        const Entries e = next;
        if (st + 2 < st1) next = entries_of(st + 2);
        load(dn, vnext, st + 1, e);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (!here(st)) return;                           // uniform
      const KvRun k = tile_of(st);
      const int end = k.key + 31;
      f32x4 sc[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const u32x4 kf = d.k[i].frag(s);
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][i] = M::mma(kf, q[t][s], sc[t][i]);
        }
      const bool whole = k.key >= k.low && end <= min(pos_lo, k.high) && (!a.window || k.key > pos_hi - a.window || end < a.sinks);
      if (d.none[0] || d.none[1] || !whole) {          // uniform
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int key = k.key + i * 16 + g4 * 4 + j;
              const bool seen = key >= k.low && key <= min(pos[t], k.high) && (!a.window || key > pos[t] - a.window || key < a.sinks);
              if (!seen) sc[t][i][j] = -INFINITY;
              else if (d.none[i]) sc[t][i][j] = __uint_as_float(0x7fc00000u);
            }
      }
      u32x4 pf[NT][1];
      softmax_step<NT, 2, DB, M>(sc, m, l, o, pf, scale2);
      u32x4* const mine = vbuf + wave * 2 * BU;
      if constexpr (SB) {
        // (this wavefront's reads of the tile before are done: their products were waited for)
        d.v[0].store(mine, c16, g4);
        d.v[1].store(mine + BU, c16, g4);
        asm volatile("" ::: "memory");
      } else {
        if (more) wait_loads<NEXT>();
        else wait_loads<0>();
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 vf = cols_frag<HD>(mine, db, lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t][db] = M::mma(vf, pf[t][0], o[t][db]);
      }
    };
    int st = st0;
    for (; st + 2 <= st1; st += 2) {
      tile(st, d0, v0, d1, SB ? v0 : v1);
      tile(st + 1, d1, SB ? v0 : v1, d0, v0);
    }
    if (st < st1) tile(st, d0, v0, d1, SB ? v0 : v1);

    // The wavefronts' sums, 16 pairs at a time: each adds up, in the wavefronts'
    // order, a quarter of the elements.
    const float nan = __uint_as_float(0x7fc00000u);
    float* const rec = static_cast<float*>(a.work) + (int64_t)it.slot * kRecord<HD, QP>;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float sum = sum4g(l[t]);
      __syncthreads();                                 // (LDS is no longer read)
      if (g4 == 0) ml[wave][0][c16] = m[t], ml[wave][1][c16] = sum;
      __syncthreads();
      float top = m[t];
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][0][c16]);
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) sum += ml[w][1][c16] * __builtin_amdgcn_exp2f(ml[w][0][c16] - top);
      const float f = __builtin_amdgcn_exp2f(m[t] - top);
#pragma unroll
      for (int db = 0; db < DB; ++db) v0[(wave * DB + db) * 64 + lane] = __builtin_bit_cast(u32x4, o[t][db] * f);
      __syncthreads();
      const int pair = pair0 + t * 16 + c16, in_tile = t * 16 + c16;
      if (pos[t] >= b.cap) sum = nan;                  // (past the table)
      const int r = quotient(min(pair, n_pairs - 1), a.by_group);
      const int head = kvh * a.group + remainder(min(pair, n_pairs - 1), r, a.by_group), row = it.w.row0 + r;
      const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);     // (1 ulp of float32, before the rounding to 16 bits)
      if (pair < n_pairs) {
#pragma unroll
        for (int j = 0; j < DB / 4; ++j) {
          const int db = wave * (DB / 4) + j;
          f32x4 v = __builtin_bit_cast(f32x4, v0[db * 64 + lane]);
#pragma unroll
          for (int w = 1; w < 4; ++w) v += __builtin_bit_cast(f32x4, v0[(w * DB + db) * 64 + lane]);
          if (it.splits > 1) {                         // uniform
            *reinterpret_cast<f32x4*>(rec + in_tile * HD + db * 16 + g4 * 4) = v;
          } else {
            v = v * inv;
            *reinterpret_cast<u32x2*>(at(a.out, row, head) + db * 32 + g4 * 8) = u32x2{M::pack(v[0], v[1]), M::pack(v[2], v[3])};
          }
        }
        if (wave == 0 && g4 == 0) {
          if (it.splits > 1) rec[QP * HD + in_tile] = top, rec[QP * HD + QP + in_tile] = sum;
          else if (a.lse) a.lse[(int64_t)head * b.rows + row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
      }
    }
    __syncthreads();                                   // (the next item's loads write LDS)
  }
}

// Joins the shares of split sequences: NW wavefronts per pair; 16 (32) lanes hold
// its 64 (128) elements, and a wavefront's four (two) groups of lanes take turns
// with the shares.
template <int HD, int QP, int KEYS, int NW, class M>
__global__ __launch_bounds__(256) void k_kv_join(const KvAttnArgs a) {
  constexpr int W = HD / 4, GROUPS = 64 / W, TURNS = GROUPS * NW, AT_ONCE = NW == 1 ? 8 : 4;
  __shared__ f32x4 o_s[NW][W];
  __shared__ float m_s[NW], l_s[NW];
  const int lane = threadIdx.x & 63, e = lane % W, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int turn = (NW == 1 ? 0 : wave * GROUPS) + lane / W;
  const int n_units = gridDim.x * (4 / NW);            // at once
  const SeqWork own = a.plan ? SeqWork{} : seq_work<QP, KEYS>(a, lane);
  const int share = share_length<QP, KEYS>(a, own);
  int unit = blockIdx.x * (4 / NW) + (NW == 1 ? wave : 0);               // pair of all split sequences, key heads fastest
  const int n_seqs = a.batch.n_seqs;
  const int own_n = shares_of(own, share), items = own_n > 1 ? own.tiles * own_n : 0, upto = scan(items);
  const int pairs = own_n > 1 ? own.rows * a.group : 0, pairs_upto = scan(pairs);
  const int all = a.plan ? a.plan[3 * n_seqs] : __builtin_amdgcn_readlane(pairs_upto, 63);   // (of the last sequence)
  for (; unit < all * a.cache.n_kv; unit += n_units) { // uniform
    const int kvh = unit % a.cache.n_kv, left = unit / a.cache.n_kv;
    int pair, splits, slot0, row0;
    if (a.plan) {
      const Found f = search<QP, KEYS>(a, a.plan + 1 + 2 * n_seqs, left, lane);
      if (f.seq == n_seqs) continue;
      pair = left - (f.seq ? a.plan[2 * n_seqs + f.seq] : 0);
      splits = shares_of(f.w, share);
      slot0 = (f.seq ? a.plan[n_seqs + f.seq] : 0) + (f.w.tiles - 1 - pair / QP) * splits;
      row0 = f.w.row0;
      // (numbers that do not fit together: row_start does not ascend)
      if (pair < 0 || pair >= f.w.rows * a.group || splits < 2) continue;
    } else {
      const int l = __builtin_ctzll(__ballot(pairs_upto > left));
      auto from = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      pair = left - (from(pairs_upto) - from(pairs));
      splits = from(own_n);
      slot0 = from(upto) - from(items) + (from(own.tiles) - 1 - pair / QP) * splits;
      row0 = from(own.row0);
    }
    const int in_tile = pair % QP;
    if (slot0 < 0 || (int64_t)(slot0 + splits) * a.cache.n_kv > a.slots) continue;   // (row_start does not ascend)
    const float* const rec = static_cast<const float*>(a.work) + ((int64_t)slot0 * a.cache.n_kv + kvh) * kRecord<HD, QP>;
    const int64_t step = (int64_t)a.cache.n_kv * kRecord<HD, QP>;
    // the group's shares (maxima are finite; past the last one: nothing)
    float top = -1e30f, sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = turn; i0 < splits + turn; i0 += TURNS * AT_ONCE) {      // uniform by wavefront
      f32x4 x[AT_ONCE];
      float m[AT_ONCE], s[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int i = min(i0 + j * TURNS, splits - 1);
        x[j] = *reinterpret_cast<const f32x4*>(rec + i * step + in_tile * HD + e * 4);
        m[j] = rec[i * step + QP * HD + in_tile];
        s[j] = rec[i * step + QP * HD + QP + in_tile];
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        if (i0 + j * TURNS >= splits) continue;
        const float t = fmaxf(top, m[j]), f0 = __builtin_amdgcn_exp2f(top - t), f1 = __builtin_amdgcn_exp2f(m[j] - t);
        top = t;
        sum = sum * f0 + s[j] * f1;
        o = o * f0 + x[j] * f1;
      }
    }
#pragma unroll
    for (int d = W; d < 64; d *= 2) {                                    // the groups', in a tree
      const float m2 = __shfl_xor(top, d), s2 = __shfl_xor(sum, d), t = fmaxf(top, m2);
      const float f0 = __builtin_amdgcn_exp2f(top - t), f1 = __builtin_amdgcn_exp2f(m2 - t);
      top = t;
      sum = sum * f0 + s2 * f1;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * f0 + __shfl_xor(o[j], d) * f1;
    }
    if constexpr (NW > 1) {                            // the wavefronts', in order
      if (lane < W) {
        o_s[wave][e] = o;
        if (e == 0) m_s[wave] = top, l_s[wave] = sum;
      }
      __syncthreads();
      for (int w = 0; w < NW; ++w) {
        if (w == 0) {
          top = m_s[0], sum = l_s[0], o = o_s[0][e];
        } else {
          const float t = fmaxf(top, m_s[w]), f0 = __builtin_amdgcn_exp2f(top - t), f1 = __builtin_amdgcn_exp2f(m_s[w] - t);
          top = t;
          sum = sum * f0 + l_s[w] * f1;
          o = o * f0 + o_s[w][e] * f1;
        }
      }
      __syncthreads();
    }
    if (turn == 0) {
      const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
      const int r = quotient(pair, a.by_group), head = kvh * a.group + remainder(pair, r, a.by_group), row = row0 + r;
      *reinterpret_cast<u32x2*>(at(a.out, row, head) + e * 8) = u32x2{M::pack(o[0] * inv, o[1] * inv), M::pack(o[2] * inv, o[3] * inv)};
      if (a.lse && e == 0)
        a.lse[(int64_t)head * a.batch.rows + row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// Tiles of QP pairs that the rows can make, and whether a sequence can have
// more than one share.
int64_t max_tiles(const KvAttnArgs& a, int qp) {
  return std::min<int64_t>(a.batch.n_seqs, a.batch.rows) + (int64_t)a.batch.rows * a.group / qp;
}
bool may_split(const KvAttnArgs& a) { return a.batch.cap > kMinKeys; }

// Pairs of a workgroup, by those that a sequence has on average (8 key heads x
// 128, us for 16, 32, 64 and 128 pairs a workgroup):
//   up to 16 or 32: as few as that (16 sequences of 20 000 keys in e2m1, 4 pairs:
//     81, 121, 157, 208)
//   up to 64: 64 (32 sequences of 1000 keys, 36 pairs: 42, 35, 28, 40), but 32 for
//     8 and 4 bits, where a wavefront of k_kv_few widens its own keys and waits for
//     nobody's (of 8000 keys in e4m3: 233, 158, 179, 220; with 2 key heads x 64 and
//     pages of 16 in any order 39 with 32 and 51 with 64, in a row 40 and 36)
//   more: 128 (68 pairs: 137, 98, 75, 57), but 64 where 128 leave much empty (132
//     pairs: 219, 140, 95, 124)
// A long chunk beside single tokens counts, where it is known: 1000 single
// tokens and 2000 rows of one sequence 896, 575, 444, 437; 63 and 1000 405, 254,
// 185, 222.
int tile_pairs(const KvAttnArgs& a, int max_seq_rows) {
  const int64_t mean = ((int64_t)a.batch.rows * a.group + a.batch.n_seqs - 1) / a.batch.n_seqs;
  const int64_t most = (int64_t)max_seq_rows * a.group;
  const int64_t pairs = max_seq_rows > 0 ? std::min(most, mean) : mean;
  const bool chunk = most >= 4 * mean && most > 64 && 4ll * max_seq_rows >= a.batch.rows;
  if (pairs <= 64) return chunk ? 64 : pairs <= 16 ? 16 : pairs <= 32 || a.cache.k_scale ? 32 : 64;
  return pairs <= 192 && (pairs > 128 || chunk) ? 64 : 128;
}

// Records of partial sums: a sequence of k > 1 shares has k - 1 of them full, so
// that k is at most twice the number of full ones, of which kShares hold
// everything.
int64_t max_slots(const KvAttnArgs& a, int qp) {
  if (!may_split(a)) return 0;
  const int64_t shares = (a.batch.cap + kMinKeys - 1) / kMinKeys + 2;
  return std::min<int64_t>(max_tiles(a, qp) * a.cache.n_kv * shares, 2 * (qp == 16 ? kShares<16> : kShares<64>) + 2);
}

template <int HD, int QP, class M, int DT>
hipError_t launch_pairs(KvAttnArgs a, hipStream_t st) {
  a.slots = (int)max_slots(a, QP);
  a.plan = nullptr;
  if (a.batch.n_seqs > kMaxAlone)
    a.plan = reinterpret_cast<int*>(static_cast<char*>(a.work) + align256((size_t)a.slots * kRecord<HD, QP> * sizeof(float)));
  const int64_t items = max_tiles(a, QP) + (may_split(a) ? kShares<QP> / a.cache.n_kv + 1 : 0);   // of a key head
  const int64_t most = std::max((1 << 20) / a.cache.n_kv, 1);
  const unsigned grid = (unsigned)(std::min(items, most) * a.cache.n_kv);
  constexpr int KEYS = QP >= 64 ? kStageKeys : kFewKeys;
  if (a.plan) {
    k_kv_plan<QP, KEYS><<<1, 1024, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if constexpr (QP == 128) k_kv_attn<HD, 2, 1, M, DT><<<grid, 256, 0, st>>>(a);
  else if constexpr (QP == 64) k_kv_attn<HD, 1, 2, M, DT><<<grid, 512, 0, st>>>(a);
  else k_kv_few<HD, QP / 16, M, DT><<<grid, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !may_split(a)) return e;
  // few pairs: a workgroup each (9 rows of 32 heads over 16 384 keys, 52 shares: 7.5 us by
  // wavefronts, 4.7 by workgroups)
  const int64_t pairs = (int64_t)a.batch.rows * a.n_heads;
  if (pairs <= 1024) k_kv_join<HD, QP, KEYS, 4, M><<<(unsigned)pairs, 256, 0, st>>>(a);
  else k_kv_join<HD, QP, KEYS, 1, M><<<(unsigned)std::min<int64_t>((pairs + 3) / 4, 2048), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int HD, class M, int DT>
hipError_t launch_cache(const KvAttnArgs& a, int max_seq_rows, hipStream_t st) {
  switch (tile_pairs(a, max_seq_rows)) {
    case 16: return launch_pairs<HD, 16, M, DT>(a, st);
    case 32: return launch_pairs<HD, 32, M, DT>(a, st);
    case 64: return launch_pairs<HD, 64, M, DT>(a, st);
    default: return launch_pairs<HD, 128, M, DT>(a, st);
  }
}

template <int HD, class M, int SAME>
hipError_t launch_hd(int cache_dtype, const KvAttnArgs& a, int max_seq_rows, hipStream_t st) {
  if (cache_dtype == PARD_E4M3) return launch_cache<HD, M, PARD_E4M3>(a, max_seq_rows, st);
  if (cache_dtype == PARD_E2M1) return launch_cache<HD, M, PARD_E2M1>(a, max_seq_rows, st);
  return launch_cache<HD, M, SAME>(a, max_seq_rows, st);
}

}  // namespace

size_t kv_attn_workspace(const KvAttnArgs& a, int head_dim, int max_seq_rows) {
  const int qp = tile_pairs(a, max_seq_rows);
  const size_t plan = a.batch.n_seqs > kMaxAlone ? (1 + 3 * (size_t)a.batch.n_seqs) * sizeof(int) : 0;
  return std::max<size_t>(align256((size_t)max_slots(a, qp) * qp * (head_dim + 2) * sizeof(float)) + plan, 256);
}

hipError_t launch_kv_attn(int head_dim, int dtype, int cache_dtype, const KvAttnArgs& a, int max_seq_rows, hipStream_t st) {
  if (head_dim == 64)
    return dtype == PARD_BF16 ? launch_hd<64, KvBF16, PARD_BF16>(cache_dtype, a, max_seq_rows, st)
                              : launch_hd<64, KvF16, PARD_F16>(cache_dtype, a, max_seq_rows, st);
  return dtype == PARD_BF16 ? launch_hd<128, KvBF16, PARD_BF16>(cache_dtype, a, max_seq_rows, st)
                            : launch_hd<128, KvF16, PARD_F16>(cache_dtype, a, max_seq_rows, st);
}

}  // namespace pard
