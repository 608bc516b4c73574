// Attention of a batch's new rows over a paged cache, on gfx950 MFMA.
//
// A sequence's rows and query heads of one key head are its pairs (row by row).
// A workgroup of four wavefronts owns 64 NQ of them, a wavefront 16 NQ, and
// walks the keys that its rows see in stages of 64 through two LDS buffers, the
// next stage in flight during the current one.  With a window the stages cover
// the first tokens, then the keys from the first row's window on; only stages
// that some row does not see whole compare keys with rows.  A tile is S^T = K
// Q^T, online softmax in base 2, O^T += V^T P^T (softmax_step).
//   * 16 bits: LDS-DMA, 16 keys to a wavefront; pages have 16 keys or more, so
//     such a block lies in one page, whose table entry is read a stage ahead.
//   * 8 and 4 bits: bytes and scales into registers, widened into LDS at the end
//     of the stage (v_cvt_scalef32_*: exact in bfloat16), so that everything
//     behind is the same.
// Work is shared out on the device, from lengths that only the device knows:
// every wavefront adds up the batch's stages (64 sequences at a step), finds
// the length of a share, and from the running number of shares the one that is
// its workgroup's (plan()).  Sequences of more than one share leave partial
// sums, which a second launch joins in the order of the keys.
#include "serve.h"

#include <algorithm>

#include "cod_attn_tile.h"

namespace pard {
namespace {

using namespace cod;

constexpr int kStageKeys = 64;
constexpr int kMinShare = 4;               // stages of a share at least
constexpr int kShares = 512;               // shares that long contexts are cut into, about

// ---- sharing out ------------------------------------------------------------

// One sequence's work.
struct SeqWork {
  int row0, rows, len;                     // first row, rows, positions
  int tiles;                               // of 64 NQ pairs
  int stages;                              // of a tile, at most
};

template <int QP>
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
  if (a.window) keys = (int)min((int64_t)keys, (int64_t)a.window + min(w.rows, QP / a.group + 2) + min(a.sinks, keys) + kStageKeys);
  w.stages = w.tiles ? max((keys + kStageKeys - 1) / kStageKeys, 1) : 0;
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

__device__ __forceinline__ int shares_of(const SeqWork& w, int share) { return (w.stages + share - 1) / share; }

// The length of a share, such that about kShares of them hold all stages; every
// wavefront finds the same.
template <int QP>
__device__ __forceinline__ int share_length(const KvAttnArgs& a, const SeqWork& first, int lane) {
  float total = 0.f;
  for (int s0 = 0; s0 < a.batch.n_seqs; s0 += 64) {   // uniform
    const SeqWork w = s0 ? seq_work<QP>(a, s0 + lane) : first;
    float x = (float)w.tiles * w.stages;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    total += x;
  }
  total *= a.cache.n_kv;
  return max(kMinShare, (int)fminf(ceilf(total / kShares), 1 << 24));
}

struct Item {
  SeqWork w;
  int seq, tile, split, splits;            // splits 0: no such item
  int slot;                                // of its partial sums
};

// Item `left` of a key head: a tile's shares first, then tiles (the last first:
// they see the most keys), then sequences.
template <int QP>
__device__ __forceinline__ Item find_item(const KvAttnArgs& a, const SeqWork& first, int share, int left, int kvh, int lane) {
  Item it{};
  int slots = 0;
  for (int s0 = 0; s0 < a.batch.n_seqs; s0 += 64) {
    const SeqWork w = s0 ? seq_work<QP>(a, s0 + lane) : first;
    const int n = shares_of(w, share), items = w.tiles * n, split = n > 1 ? items : 0;
    const int upto = scan(items), slots_upto = scan(split);
    const uint64_t past = __ballot(upto > left);
    if (past) {
      const int l = __builtin_ctzll(past);
      auto from = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      it.w = SeqWork{from(w.row0), from(w.rows), from(w.len), from(w.tiles), from(w.stages)};
      const int mine = left - (from(upto) - from(items));
      it.seq = s0 + l;
      it.splits = from(n);
      it.tile = it.w.tiles - 1 - mine / it.splits;
      it.split = mine % it.splits;
      it.slot = (slots + from(slots_upto) - from(split) + mine) * a.cache.n_kv + kvh;
      return it;
    }
    left -= __builtin_amdgcn_readlane(upto, 63);
    slots += __builtin_amdgcn_readlane(slots_upto, 63);
  }
  return it;
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

// Partial sums of a tile: [QP][HD] of O, [QP] maxima, [QP] sums.
template <int HD, int QP>
constexpr int kRecord = QP * (HD + 2);

template <int HD, int NQ, class M, int DT>
__global__ __launch_bounds__(256, HD == 128 ? 2 : NQ == 2 ? 3 : 4) void k_kv_attn(const KvAttnArgs a) {
  constexpr int QW = 16 * NQ, QP = 4 * QW;             // pairs of a wavefront, of the workgroup
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  constexpr int RB = kv_row_bytes(DT, HD), SB = kv_scale_bytes(DT, HD);
  // a stage: four blocks of K, four of V; two arrays of their own (the
  // compiler's waits before an LDS read cover the loads into that array only)
  __shared__ __attribute__((aligned(16))) u32x4 b0[8 * BU], b1[8 * BU];
  __shared__ int any_bad;                              // a stage of this item has a key without a page
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KvBatchView& b = a.batch;
  const SeqWork first = seq_work<QP>(a, lane);
  const int share = share_length<QP>(a, first, lane);
  // key heads fastest: with 8 of them each keeps to an XCD and its L2
  const int kvh = blockIdx.x % a.cache.n_kv;
  for (int u = blockIdx.x / a.cache.n_kv;; u += gridDim.x / a.cache.n_kv) {
    const Item it = find_item<QP>(a, first, share, u, kvh, lane);
    if (it.splits == 0) return;                        // uniform: past the last item
    if (it.splits > 1 && it.slot >= a.slots) continue; // uniform (row_start does not ascend)
    __syncthreads();                                   // (the item before has read LDS)
    if (tid == 0) any_bad = 0;
    __syncthreads();
    const int n_pairs = it.w.rows * a.group, pair0 = it.tile * QP;
    const int pos0 = it.w.len - it.w.rows;             // of the sequence's first row
    auto row_of = [&](int pair) { return quotient(min(pair, n_pairs - 1), a.by_group); };

    // what the tile's rows see: keys 0 .. a_last, then lo .. last
    const int pos_lo = pos0 + row_of(pair0), pos_hi = pos0 + row_of(pair0 + QP - 1);
    const int last = min(pos_hi, b.cap - 1);
    int lo = a.window ? max(pos_lo - a.window + 1, 0) : 0;
    int a_last = min(a.sinks, lo) - 1;
    if (a.sinks >= lo) lo = 0, a_last = -1;            // one run of keys
    const int from = lo & ~15, n_a = (a_last + kStageKeys) / kStageKeys;
    const int n_all = last < 0 ? 0 : n_a + (last - from) / kStageKeys + 1;
    const int st0 = (int)((int64_t)n_all * it.split / it.splits), st1 = (int)((int64_t)n_all * (it.split + 1) / it.splits);

    // this wavefront's 16 keys of a stage: blocks past a run repeat its last key
    struct Block { int key, low, high; };
    auto block_of = [&](int st) __attribute__((always_inline)) {
      const bool in_a = st < n_a;
      const int key = (in_a ? st * kStageKeys : from + (st - n_a) * kStageKeys) + wave * 16, high = in_a ? a_last : last;
      return Block{key, in_a ? 0 : lo, high};
    };
    const int32_t* const table = b.table + (int64_t)it.seq * b.max_pages;
    auto entry_of = [&](int st) __attribute__((always_inline)) {
      const Block k = block_of(st);
      return table[min(k.key, k.high) >> a.cache.page_log2];
    };
    Staged<HD, M, DT> sk, sv;
    auto load = [&](u32x4* buf, int st, int entry) __attribute__((always_inline)) {
      const Block k = block_of(st);
      int page = __builtin_amdgcn_readfirstlane(entry);
      if ((uint32_t)page >= (uint32_t)a.cache.n_pages) {  // uniform
        page = 0;
        if (lane == 0) any_bad = 1;
      }
      const int r = DT == PARD_E4M3 || DT == PARD_E2M1 ? c16 : block_row(lane);
      const int place = max(min(k.key + r, k.high), k.low) & ((1 << a.cache.page_log2) - 1);
      const int64_t slot = (((int64_t)page * a.cache.n_kv + kvh) << a.cache.page_log2) + place;
      if constexpr (SB) {
        sk.load(a.cache.k + slot * RB, a.cache.k_scale + slot * SB, g4);
        sv.load(a.cache.v + slot * RB, a.cache.v_scale + slot * SB, g4);
      } else {
        load_block<HD>(a.cache.k + slot * RB + block_byte(lane), buf + wave * BU);
        load_block<HD>(a.cache.v + slot * RB + block_byte(lane), buf + (4 + wave) * BU);
      }
    };
    auto widen = [&](u32x4* buf) __attribute__((always_inline)) {
      if constexpr (SB) {
        sk.store(buf + wave * BU, c16, g4);
        sv.store(buf + (4 + wave) * BU, c16, g4);
      }
    };

    int entry = 0;
    if (st0 < st1) {                                   // uniform
      load(b0, st0, entry_of(st0));
      if (st0 + 1 < st1) entry = entry_of(st0 + 1);
    }
    // this lane's pairs: those past the sequence repeat its last and are not stored
    const int w_pair = pair0 + wave * QW;
    const bool idle = w_pair >= n_pairs;               // uniform: no pairs of its own
    const int w_lo = pos0 + row_of(w_pair), w_hi = pos0 + row_of(w_pair + QW - 1);
    u32x4 q[NQ][KS];
    float m[NQ], l[NQ];
    f32x4 o[NQ][DB];
    int pos[NQ];
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
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[t][ks][i] ^= sign;

    auto compute = [&](int st, const u32x4* cur) __attribute__((always_inline)) {
      const bool in_a = st < n_a;
      const int key0 = in_a ? st * kStageKeys : from + (st - n_a) * kStageKeys, end = key0 + kStageKeys - 1;
      const int low = in_a ? 0 : lo, high = in_a ? a_last : last, gone = a.window ? w_lo - a.window : -1;   // keys up to `gone` are no row's but first tokens
      if (idle || key0 > w_hi || (end <= gone && key0 >= a.sinks)) return;   // uniform: no row of this wavefront sees it
      f32x4 sc[NQ][4];
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) sc[t][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 kf = rows_frag(cur + kb * BU, ks, lane);
#pragma unroll
          for (int t = 0; t < NQ; ++t) sc[t][kb] = M::mma(kf, q[t][ks], sc[t][kb]);
        }
      const bool bad = any_bad;
      const bool whole = key0 >= low && end <= min(w_lo, high) && (!a.window || key0 > w_hi - a.window || end < a.sinks);
      if (bad || !whole) {                             // uniform
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const int k16 = key0 + kb * 16;
          const bool none = bad && (uint32_t)table[min(k16, high) >> a.cache.page_log2] >= (uint32_t)a.cache.n_pages;
#pragma unroll
          for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = k16 + g4 * 4 + i;
              const bool seen = key >= low && key <= min(pos[t], high) && (!a.window || key > pos[t] - a.window || key < a.sinks);
              if (!seen) sc[t][kb][i] = -INFINITY;
              else if (none) sc[t][kb][i] = __uint_as_float(0x7fc00000u);
            }
        }
      }
      u32x4 pf[NQ][2];
      softmax_step<NQ, 4, DB, M>(sc, m, l, o, pf, scale2);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u32x4 vf = cols_frag<HD>(cur + (4 + 2 * tt) * BU, db, lane);
#pragma unroll
          for (int t = 0; t < NQ; ++t) o[t][db] = M::mma(vf, pf[t][tt], o[t][db]);
        }
    };
    auto stage = [&](int st, const u32x4* cur, u32x4* nxt) __attribute__((always_inline)) {
      wait_and_meet();
      const bool more = st + 1 < st1;
      if (more) {                                      // uniform
        const int e = entry;
        if (st + 2 < st1) entry = entry_of(st + 2);
        load(nxt, st + 1, e);
      }
      __builtin_amdgcn_sched_barrier(0);
      compute(st, cur);
      if (more) widen(nxt);
    };
    if (st0 < st1) widen(b0);
    int st = st0;
    for (; st + 2 <= st1; st += 2) {
      stage(st, b0, b1);
      stage(st + 1, b1, b0);
    }
    if (st < st1) stage(st, b0, b1);

    // lane (c16, g4) holds elements 16 db + 4 g4 .. + 3 of pair 16 t + c16
    const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int pair = w_pair + t * 16 + c16, in_tile = wave * QW + t * 16 + c16;
      float sum = sum4g(l[t]);
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

// Joins the shares of split sequences: a wavefront per pair, shares in order.
template <int HD, int QP, class M>
__global__ __launch_bounds__(256) void k_kv_join(const KvAttnArgs a) {
  constexpr int PER = HD / 64;
  const int lane = threadIdx.x & 63;
  const int n_waves = gridDim.x * 4;
  const SeqWork first = seq_work<QP>(a, lane);
  const int share = share_length<QP>(a, first, lane);
  int unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // pair of all split sequences, key heads fastest
  int before = 0, slots = 0;
  for (int s0 = 0; s0 < a.batch.n_seqs; s0 += 64) {                       // uniform
    const SeqWork w = s0 ? seq_work<QP>(a, s0 + lane) : first;
    const int n = shares_of(w, share), items = n > 1 ? w.tiles * n : 0;
    const int upto = scan(items), pairs = n > 1 ? w.rows * a.group : 0, pairs_upto = scan(pairs);
    const int all = __builtin_amdgcn_readlane(pairs_upto, 63);
    for (; unit < (before + all) * a.cache.n_kv; unit += n_waves) {
      const int kvh = unit % a.cache.n_kv, left = unit / a.cache.n_kv - before;
      const int l = __builtin_ctzll(__ballot(pairs_upto > left));
      auto from = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      const int pair = left - (from(pairs_upto) - from(pairs)), splits = from(n), in_tile = pair % QP;
      const int slot0 = slots + from(upto) - from(items) + (from(w.tiles) - 1 - pair / QP) * splits;
      if ((slot0 + splits) * a.cache.n_kv > a.slots) continue;             // (row_start does not ascend)
      const float* const rec = static_cast<const float*>(a.work) + ((int64_t)slot0 * a.cache.n_kv + kvh) * kRecord<HD, QP>;
      const int64_t step = (int64_t)a.cache.n_kv * kRecord<HD, QP>;
      float top = -1e30f, sum = 0.f;
      for (int i = lane; i < splits; i += 64) {        // (maxima are finite)
        const float m = rec[i * step + QP * HD + in_tile], s = rec[i * step + QP * HD + QP + in_tile], t = fmaxf(top, m);
        sum = sum * __builtin_amdgcn_exp2f(top - t) + s * __builtin_amdgcn_exp2f(m - t);
        top = t;
      }
      const float own = top;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      sum *= __builtin_amdgcn_exp2f(own - top);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
      float o[PER] = {};
#pragma unroll 8
      for (int i = 0; i < splits; ++i) {
        const float f = __builtin_amdgcn_exp2f(rec[i * step + QP * HD + in_tile] - top);
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] += f * rec[i * step + in_tile * HD + lane * PER + e];
      }
      const float inv = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);
      const int r = quotient(pair, a.by_group), head = kvh * a.group + remainder(pair, r, a.by_group), row = from(w.row0) + r;
      char* const dst = at(a.out, row, head);
      if constexpr (PER == 2) {
        reinterpret_cast<uint32_t*>(dst)[lane] = M::pack(o[0] * inv, o[1] * inv);
      } else {
        reinterpret_cast<uint16_t*>(dst)[lane] = (uint16_t)M::pack(o[0] * inv, 0.f);
      }
      if (a.lse && lane == 0)
        a.lse[(int64_t)head * a.batch.rows + row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    before += all;
    slots += __builtin_amdgcn_readlane(upto, 63);
  }
}

// Tiles of QP pairs that the rows can make, and whether a sequence can have
// more than one share.
int64_t max_tiles(const KvAttnArgs& a, int qp) {
  return std::min<int64_t>(a.batch.n_seqs, a.batch.rows) + (int64_t)a.batch.rows * a.group / qp;
}
bool may_split(const KvAttnArgs& a) { return a.batch.cap > kMinShare * kStageKeys; }

// Pairs of a workgroup: 64 where sequences have few, on average.
int tile_pairs(const KvAttnArgs& a, int max_seq_rows) {
  const int64_t most = (int64_t)max_seq_rows * a.group;
  return (max_seq_rows > 0 && most <= 64) || (int64_t)a.batch.rows * a.group <= 64ll * a.batch.n_seqs ? 64 : 128;
}

// Records of partial sums: a sequence of k > 1 shares has k - 1 of them full, so
// that k is at most twice the number of full ones, of which kShares hold
// everything.
int64_t max_slots(const KvAttnArgs& a, int qp) {
  if (!may_split(a)) return 0;
  const int64_t cap_stages = (a.batch.cap + kStageKeys - 1) / kStageKeys + 2;
  return std::min<int64_t>(max_tiles(a, qp) * a.cache.n_kv * ((cap_stages + kMinShare - 1) / kMinShare), 2 * kShares + 2);
}

template <int HD, int NQ, class M, int DT>
hipError_t launch_tiles(KvAttnArgs a, hipStream_t st) {
  constexpr int QP = 64 * NQ;
  a.slots = (int)max_slots(a, QP);
  const int64_t items = max_tiles(a, QP) + (may_split(a) ? kShares / a.cache.n_kv + 1 : 0);   // of a key head
  const int64_t most = std::max((1 << 20) / a.cache.n_kv, 1);
  k_kv_attn<HD, NQ, M, DT><<<(unsigned)(std::min(items, most) * a.cache.n_kv), 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !may_split(a)) return e;
  const int64_t waves = (int64_t)a.batch.rows * a.n_heads;
  k_kv_join<HD, QP, M><<<(unsigned)std::min<int64_t>((waves + 3) / 4, 1024), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int HD, class M, int DT>
hipError_t launch_cache(const KvAttnArgs& a, int max_seq_rows, hipStream_t st) {
  return tile_pairs(a, max_seq_rows) == 64 ? launch_tiles<HD, 1, M, DT>(a, st) : launch_tiles<HD, 2, M, DT>(a, st);
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
  return std::max<size_t>((size_t)max_slots(a, qp) * qp * (head_dim + 2) * sizeof(float), 256);
}

hipError_t launch_kv_attn(int head_dim, int dtype, int cache_dtype, const KvAttnArgs& a, int max_seq_rows, hipStream_t st) {
  if (head_dim == 64)
    return dtype == PARD_BF16 ? launch_hd<64, KvBF16, PARD_BF16>(cache_dtype, a, max_seq_rows, st)
                              : launch_hd<64, KvF16, PARD_F16>(cache_dtype, a, max_seq_rows, st);
  return dtype == PARD_BF16 ? launch_hd<128, KvBF16, PARD_BF16>(cache_dtype, a, max_seq_rows, st)
                            : launch_hd<128, KvF16, PARD_F16>(cache_dtype, a, max_seq_rows, st);
}

}  // namespace pard
