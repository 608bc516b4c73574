// Gradient of attention over packed COD rows on gfx950 MFMA: with P = exp(scale
// Q K^T - lse) over the pairs of rows that see each other,
//   dV = P^T dO,  dS = P (dO V^T - delta),  delta = rowsum(dO O),
//   dQ = scale dS K,  dK = scale dS^T Q.
//
// Three launches (the first finds delta), no atomics, so that every sum has one
// order:
//   k_cod_dq  as the forward kernel: a workgroup owns 64 NQ (row, head) pairs of
//     a key head and walks their keys.  It also leaves lse, delta, the real
//     tokens seen and the place of every pair, in pair order, for the other.
//   k_cod_dkv  a workgroup owns 64 NK real tokens of a key head (K and V in operand
//     registers) and walks the pairs that see them, all heads of the group, in
//     stages through LDS.  Mask rows are seen by the rows of
//     their chain alone: workgroups behind those own 64 places of the order and
//     walk the pairs from the first place to the last chain's end.
//
// Both recompute the scores (9 products in place of 7 with the forward's), since
// neither dQ nor dK and dV of a sample fit on chip.  Bound: the SIMDs' issue, as
// in the forward: at head_dim 64 the products take 36 % of the busy CUs' cycles for
// dQ and 41 % for dK and dV, the other instructions 38 and 31 %.  In dK and dV a
// fifth of the CUs' time is idle besides: nearly all workgroups start at once, and
// walk from a few to some 200 stages.  1B layer (16 samples of 256 to 1024 tokens,
// 32 / 8 heads x 64): delta 38, dQ 332, dK and dV 466 us; 8B heads (x 128, 6 samples
// of 900 to 2048): 35, 650 and 993.  Scalar kernels took 160 and 557 ms.
//
// P and dS enter their products with 16 bits, as the matrix instructions want; the
// sums are float32.  (fp16: a dS below 2^-25 vanishes and one above 65504 is
// infinite, so d_out's scale has to keep them between.)
#include "cod_attn_tile.h"

namespace pard {
namespace {

using namespace cod;

constexpr int kStage = 64;                           // keys of a stage (dq)
// Blocks of 16 keys of a dkv wavefront: at head_dim 128 the sums of two, with K
// and V, leave too few registers (1700 us with spills, 1250 with V in LDS).
constexpr int dkv_blocks(int hd) { return hd == 64 ? 2 : 1; }
// Pairs of a stage (dkv): three workgroups' stages fit a CU's LDS (head_dim 128:
// 64 pairs, two workgroups, took 1110 us).
constexpr int dkv_pairs(int hd) { return hd == 64 ? 64 : 32; }

// Statistics of 64 pairs of one key head: base-2 log-sum (+infinity past the
// sample: probability 0), -delta, real tokens seen, place in the order.
struct PairStats {
  float lse2[64], ndelta[64];
  int seen[64], pos[64];
};

// First block of 64 pairs of a sample (every sample has blocks of its own).
__device__ __forceinline__ int64_t stats_base(const CodAttnArgs& a, int64_t off, int sample) {
  return off * a.group / 64 + sample;
}
// Blocks of one key head.
__host__ __device__ inline int64_t stats_blocks(int64_t rows, int group, int n_samples) {
  return rows * group / 64 + n_samples + 1;
}

// delta comes from the rounded output, whose error all score gradients of a row
// share.  Rows that see few keys (at most two stages of real tokens) have the
// largest gradients: theirs is made exact by a launch before (FIND), which walks
// the same keys to sum P (dO V^T - delta), what delta lacks, into the statistics.
// Errors of dQ and dK over all rows of packed samples of 256 to 1024 tokens, in
// those of rounding the exact gradients: 1.51 without, 1.4 with it.
template <int HD, int NQ, class M, bool FIND>
__global__ __launch_bounds__(256, 2) void k_cod_dq(const CodAttnArgs a) {
  constexpr int QW = 16 * NQ;                        // pairs per wavefront
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  __shared__ __attribute__((aligned(16))) u32x4 b0[8 * BU], b1[8 * BU];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = a.group, per_tile = kCodTile / (64 * NQ) * group;
  const int kvh = blockIdx.x % a.n_kv, rest = blockIdx.x / a.n_kv;
  const CodTileInfo tile = a.plan.tiles[rest / per_tile];
  const CodSampleInfo s = tile.s;
  const int pair0 = (rest % per_tile) * 64 * NQ, p0 = tile.tile * kCodTile;
  if (p0 + pair0 / group >= s.cap) return;           // uniform
  // (a chain has at most reach + 1 places, so place p sees more than p / (reach + 1) tokens)
  if (FIND && p0 >= 2 * kStage * (s.reach + 1)) return;   // uniform
  const int4* const order = a.plan.order + s.off;
  const int last = s.len - 1;
  // (as in the forward kernel: the places of all rows read first, then the rows)
  const int w_row0 = p0 + (pair0 + wave * QW) / group;             // of this wavefront's pairs
  const int w_last = min(p0 + (pair0 + (wave + 1) * QW - 1) / group, last);
  const int chain0 = max(w_row0 - s.reach, 0);
  int row[NQ], head[NQ];                             // this pair's place and query head
  int4 e[NQ] = {};                                   // packed row, real tokens seen, first mask row seen (and chain's end)
  float lse2[NQ];
  f32x4 ndelta[NQ];                                  // -delta, as dO V^T starts from
  float lacks[NQ];                                   // FIND
  float* stat[NQ];                                   // -delta in the statistics, null past the sample's blocks
  u32x4 q[NQ][KS], go[NQ][KS];
  f32x4 dq[NQ][DB];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const int pair = pair0 + wave * QW + t * 16 + c16, r = quotient(pair, a.by_group);
    row[t] = p0 + r;
    head[t] = kvh * group + remainder(pair, r, a.by_group);
#pragma unroll
    for (int db = 0; db < DB; ++db) dq[t][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    lacks[t] = 0.f;
  }
  if (last >= p0 + pair0 / group) {                  // uniform: the block has rows
    const float scale2 = a.scale * kLog2e;
    const uint64_t k_step = a.k.rs, v_step = a.v.rs;
    const char* const k0 = at(a.k, s.off, kvh);
    const char* const v0 = at(a.v, s.off, kvh);
    auto load = [&](u32x4* buf, int st) __attribute__((always_inline)) {
      const int key = min(st * kStage + wave * 16 + block_row(lane), s.n_real - 1);
      load_block<HD>(k0 + (uint32_t)key * k_step + block_byte(lane), buf + wave * BU);
      load_block<HD>(v0 + (uint32_t)key * v_step + block_byte(lane), buf + (4 + wave) * BU);
    };
    const int st_seen = order[min(p0 + (pair0 + 64 * NQ - 1) / group, last)].y;
    const int n_st = (st_seen + kStage - 1) / kStage;
    const bool few = n_st <= 2;                      // uniform
    if (FIND && !few) return;
    const int last_seen = w_row0 > last ? 0 : order[w_last].y;
    int k_row[2], v_row[2];                          // 32 keys from c0 on
    auto chain_rows = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        v_row[b] = order[min(c0 + b * 16 + c16, last)].x;
        k_row[b] = order[min(c0 + b * 16 + block_row(lane), last)].x;
      }
    };
#pragma unroll
    for (int t = 0; t < NQ; ++t) e[t] = order[min(row[t], last)];
    chain_rows(chain0);
    load(b0, 0);
    u32x4* const mine = b1 + wave * 2 * BU;
    u32x4 vf[2][KS];
    auto load_chain = [&](int next) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) vf[b][ks] = *reinterpret_cast<const u32x4*>(v0 + (uint32_t)v_row[b] * v_step + g4 * 16 + ks * 64);
        load_block<HD>(k0 + (uint32_t)k_row[b] * k_step + block_byte(lane), mine + b * BU);
      }
      if (next <= w_last) chain_rows(next);          // uniform
    };
    if (s.reach > 0) load_chain(chain0 + 32);        // uniform
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const uint32_t r = s.off + e[t].x;
      const char* const qs = at(a.q, r, head[t]) + g4 * 16;
      const char* const gs = at(a.d_out, r, head[t]) + g4 * 16;
      const char* const os = at(a.out, r, head[t]) + g4 * 16;
      lse2[t] = a.lse[head[t] * a.rows + r] * kLog2e;
      float sum = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        q[t][ks] = *reinterpret_cast<const u32x4*>(qs + ks * 64);
        go[t][ks] = *reinterpret_cast<const u32x4*>(gs + ks * 64);
        const u32x4 ov = *reinterpret_cast<const u32x4*>(os + ks * 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 x = M::unpack(go[t][ks][i]), y = M::unpack(ov[i]);
          sum = fmaf(x[0], y[0], sum);
          sum = fmaf(x[1], y[1], sum);
        }
      }
      float delta = sum4g(sum);
      const int in_sample = p0 * group + pair0 + wave * QW + t * 16 + c16;   // (below 2^30)
      stat[t] = nullptr;
      if ((in_sample & ~63) < s.len * group) {
        PairStats& st = reinterpret_cast<PairStats*>(a.stats)[kvh * a.stats_blocks + stats_base(a, s.off, tile.sample) + in_sample / 64];
        const int i = in_sample & 63;
        stat[t] = st.ndelta + i;
        if (!FIND && few) delta = -*stat[t];         // uniform
        if (!FIND && g4 == 0) {
          st.lse2[i] = row[t] <= last ? lse2[t] : INFINITY;
          if (!few) st.ndelta[i] = -delta;
          st.seen[i] = e[t].y;
          st.pos[i] = min(row[t], last);
        }
      }
      ndelta[t] = f32x4{-delta, -delta, -delta, -delta};
    }

    // dQ += dS K (FIND: the sums of dS) over 32 keys: their scores and dO V^T - delta
    // are in sc and dp, K in two LDS blocks; hidden(t, kb, i): key kb * 16 + 4 g4 + i
    auto add = [&](f32x4 (&sc)[NQ][2], f32x4 (&dp)[NQ][2], const u32x4* kblocks, bool masked, auto hidden)
                   __attribute__((always_inline)) {
      u32x4 ds[NQ];
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(sc[t][kb][i], scale2, -lse2[t]));
          if (masked) {                              // uniform
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = hidden(t, kb, i) ? 0.f : x[i];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] *= dp[t][kb][i];
          ds[t][kb * 2] = M::pack(x[0], x[1]);
          ds[t][kb * 2 + 1] = M::pack(x[2], x[3]);
          lacks[t] += FIND ? (x[0] + x[1]) + (x[2] + x[3]) : 0.f;
        }
      if (FIND) return;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 kf = cols_frag<HD>(kblocks, db, lane);
#pragma unroll
        for (int t = 0; t < NQ; ++t) dq[t][db] = M::mma(kf, ds[t], dq[t][db]);
      }
    };

    // the wavefront's chains
    uint32_t own[NQ];                                // mask rows of its chain that a row sees, itself included
#pragma unroll
    for (int t = 0; t < NQ; ++t) own[t] = min(row[t], last) - e[t].z + 1;
    for (int c0 = chain0; c0 <= w_last && s.reach > 0; c0 += 32) {           // uniform
      f32x4 sc[NQ][2], dp[NQ][2];
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        dp[t][0] = dp[t][1] = ndelta[t];
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int t = 0; t < NQ; ++t) dp[t][kb] = M::mma(vf[kb][ks], go[t][ks], dp[t][kb]);
      wait_all();
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 kf = rows_frag(mine + kb * BU, ks, lane);
#pragma unroll
          for (int t = 0; t < NQ; ++t) sc[t][kb] = M::mma(kf, q[t][ks], sc[t][kb]);
        }
      add(sc, dp, mine, true, [&](int t, int kb, int i) {
        return (uint32_t)(c0 + kb * 16 + g4 * 4 + i - e[t].z) >= own[t];
      });
      wait_all();                                    // (its reads are done before the next loads)
      if (c0 + 32 <= w_last) load_chain(c0 + 64);    // uniform
    }

    const int first_seen = __builtin_amdgcn_readfirstlane(e[0].y);           // of this wavefront's pairs
    auto stage = [&](int st, const u32x4* cur, u32x4* nxt) __attribute__((always_inline)) {
      wait_and_meet();
      if (st + 1 < n_st) load(nxt, st + 1);          // uniform
      __builtin_amdgcn_sched_barrier(0);
      const int key0 = st * kStage;
      if (key0 >= last_seen) return;                 // uniform
      const bool masked = key0 + kStage > first_seen;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        f32x4 sc[NQ][2], dp[NQ][2];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
          dp[t][0] = dp[t][1] = ndelta[t];
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4 kf = rows_frag(cur + (2 * hh + kb) * BU, ks, lane);
            const u32x4 vf = rows_frag(cur + (4 + 2 * hh + kb) * BU, ks, lane);
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
              sc[t][kb] = M::mma(kf, q[t][ks], sc[t][kb]);
              dp[t][kb] = M::mma(vf, go[t][ks], dp[t][kb]);
            }
          }
        add(sc, dp, cur + 2 * hh * BU, masked,
            [&](int t, int kb, int i) { return key0 + hh * 32 + kb * 16 + g4 * 4 + i >= e[t].y; });
      }
    };
    int st = 0;
    for (; st + 2 <= n_st; st += 2) {
      stage(st, b0, b1);
      stage(st + 1, b1, b0);
    }
    if (st < n_st) stage(st, b0, b1);
    if (FIND) {
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const float more = sum4g(lacks[t]);
        if (stat[t] && g4 == 0) *stat[t] = ndelta[t][0] - more;
      }
    }
  }
  if (FIND) return;

#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    if (row[t] >= s.cap) continue;
    const bool real = row[t] <= last;
    char* const dst = at(a.dq, s.off + (real ? e[t].x : order[row[t]].x), head[t]) + g4 * 8;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const f32x4 v = real ? dq[t][db] * a.scale : f32x4{0.f, 0.f, 0.f, 0.f};
      *reinterpret_cast<u32x2*>(dst + db * 32) = u32x2{M::pack(v[0], v[1]), M::pack(v[2], v[3])};
    }
  }
}

// dK and dV of NK blocks of 16 keys (operands kf, vf) over 32 pairs, two LDS
// blocks each of Q and dO, with the statistics st from i0 on.  If masked, key
// block k of this lane is hidden from the pairs for whose `by` entry (st.seen or
// st.pos) hidden(k, entry) holds.  dO V^T starts from -delta.
template <int HD, int NK, class M, class H>
__device__ __forceinline__ void dkv_step(const u32x4* qb, const u32x4* gb, const PairStats& st, int i0,
                                         const u32x4 (&kf)[NK][HD / 32],
                                         const u32x4 (&vf)[NK][HD / 32], f32x4 (&dk)[NK][HD / 16],
                                         f32x4 (&dv)[NK][HD / 16], float scale2, int lane, bool masked, const int* by,
                                         H&& hidden) {
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  const int g4 = lane >> 4;
  u32x4 p[NK], ds[NK];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int i = i0 + b * 16 + g4 * 4;              // this lane's four pairs
    const f32x4 lse2 = *reinterpret_cast<const f32x4*>(st.lse2 + i);
    f32x4 sc[NK], dp[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      sc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      dp[k] = *reinterpret_cast<const f32x4*>(st.ndelta + i);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 qf = rows_frag(qb + b * BU, ks, lane), gf = rows_frag(gb + b * BU, ks, lane);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        sc[k] = M::mma(qf, kf[k][ks], sc[k]);
        dp[k] = M::mma(gf, vf[k][ks], dp[k]);
      }
    }
    float x[NK][4];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[k][j] = __builtin_amdgcn_exp2f(fmaf(sc[k][j], scale2, -lse2[j]));
    if (masked) {                                    // uniform
      const i32x4 entry = *reinterpret_cast<const i32x4*>(by + i);
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[k][j] = hidden(k, entry[j]) ? 0.f : x[k][j];
    }
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      p[k][b * 2] = M::pack(x[k][0], x[k][1]);
      p[k][b * 2 + 1] = M::pack(x[k][2], x[k][3]);
      ds[k][b * 2] = M::pack(x[k][0] * dp[k][0], x[k][1] * dp[k][1]);
      ds[k][b * 2 + 1] = M::pack(x[k][2] * dp[k][2], x[k][3] * dp[k][3]);
    }
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const u32x4 gc = cols_frag<HD>(gb, db, lane), qc = cols_frag<HD>(qb, db, lane);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      dv[k][db] = M::mma(gc, p[k], dv[k][db]);
      dk[k][db] = M::mma(qc, ds[k], dk[k][db]);
    }
  }
}

// A lane's 4 elements of every 16 of one row of dK and dV.
template <int HD, class M>
__device__ __forceinline__ void store_dkv(const CodAttnArgs& a, uint32_t row, int kvh, const f32x4 (&dk)[HD / 16],
                                          const f32x4 (&dv)[HD / 16], int g4) {
  char* const ks = at(a.dk, row, kvh) + g4 * 8;
  char* const vs = at(a.dv, row, kvh) + g4 * 8;
#pragma unroll
  for (int db = 0; db < HD / 16; ++db) {
    const f32x4 x = dk[db] * a.scale, y = dv[db];
    *reinterpret_cast<u32x2*>(ks + db * 32) = u32x2{M::pack(x[0], x[1]), M::pack(x[2], x[3])};
    *reinterpret_cast<u32x2*>(vs + db * 32) = u32x2{M::pack(y[0], y[1]), M::pack(y[2], y[3])};
  }
}

// Four wavefronts, of which several workgroups share a CU: between two barriers a
// wavefront's LDS reads, products and exponentials follow each other, and other
// workgroups fill the units meanwhile (8 and 12 wavefronts over a ring of stages
// took 600 to 800 us in place of 450).  Real tokens: wavefront w has keys 16 NK w
// .. of the workgroup's 64 NK; mask rows: 16 of 64 places.  The pairs are walked
// from the last to the first, so that the tiles of a sample, which all end with
// its last pair, read the same stages at the same time (the loads alone at
// head_dim 128: 460 us, 616 from the first on).
template <int HD, class M>
__global__ __launch_bounds__(256, 3) void k_cod_dkv(const CodAttnArgs a, unsigned real_blocks) {
  constexpr int NK = dkv_blocks(HD), KW = 16 * NK;   // keys per wavefront
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  // a stage: SB blocks of Q, SB of dO, the pairs' statistics (of 64); two arrays
  // of their own
  constexpr int SP = dkv_pairs(HD), SB = SP / 16, SU = 2 * SB * BU + 64;
  __shared__ __attribute__((aligned(16))) u32x4 b0[SU], b1[SU];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = a.group;
  const float scale2 = a.scale * kLog2e;
  const bool real = blockIdx.x < real_blocks;        // uniform
  const unsigned id = real ? blockIdx.x : blockIdx.x - real_blocks;
  const int keys = real ? 4 * KW : 64, per_tile = kCodTile / keys;
  const int kvh = id % a.n_kv, rest = id / a.n_kv;
  const CodTileInfo tile = a.plan.by_sample[rest / per_tile];
  const CodSampleInfo s = tile.s;
  const int4* const order = a.plan.order + s.off;
  const int last = s.len - 1, n_pairs = s.len * group;
  const int t0 = tile.tile * kCodTile + rest % per_tile * keys;
  if (t0 >= (real ? s.n_real : s.cap)) return;       // uniform
  const PairStats* const stats =
      reinterpret_cast<const PairStats*>(a.stats) + kvh * a.stats_blocks + stats_base(a, s.off, tile.sample);

  // Stages: a wavefront loads 16 pairs (past the sample: its last row) of Q and of
  // dO, or of one of them, and a quarter of the statistics; the packed rows that a
  // stage is at are read a stage before its loads.
  const int part = wave % SB, in_stage = part * 16 + block_row(lane);
  auto stages = [&](int st0, int st1, auto step) __attribute__((always_inline)) {
    int packed = 0;
    auto find = [&](int st) __attribute__((always_inline)) {
      packed = order[min(quotient(max(st, st0) * SP + in_stage, a.by_group), last)].x;
    };
    auto load = [&](u32x4* buf, int st) __attribute__((always_inline)) {
      const int x = st * SP + in_stage;
      const uint32_t head = kvh * group + remainder(x, quotient(x, a.by_group), a.by_group), r = s.off + packed;
      if (SB == 4 || wave < 2) load_block<HD>(at(a.q, r, head) + block_byte(lane), buf + part * BU);
      if (SB == 4 || wave >= 2) load_block<HD>(at(a.d_out, r, head) + block_byte(lane), buf + (SB + part) * BU);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(reinterpret_cast<const char*>(stats + st * SP / 64) + wave * 256 + lane * 4),
          (__attribute__((address_space(3))) void*)(buf + 2 * SB * BU + wave * 16), 4, 0, 0);
      find(st - 1);
    };
    auto one = [&](int st, const u32x4* cur, u32x4* nxt) __attribute__((always_inline)) {
      wait_and_meet();
      if (st > st0) load(nxt, st - 1);               // uniform
      __builtin_amdgcn_sched_barrier(0);
      step(st, cur, *reinterpret_cast<const PairStats*>(cur + 2 * SB * BU));
    };
    find(st1 - 1);
    load(b0, st1 - 1);
    int st = st1 - 1;
    for (; st > st0; st -= 2) {
      one(st, b0, b1);
      one(st - 1, b1, b0);
    }
    if (st == st0) one(st, b0, b1);
  };

  if (real) {
    const int w0 = t0 + wave * KW;                   // this wavefront's first key
    u32x4 kf[NK][KS], vf[NK][KS];
    f32x4 dk[NK][DB], dv[NK][DB];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const uint32_t key = s.off + min(w0 + k * 16 + c16, s.n_real - 1);
      const char* const ks_ = at(a.k, key, kvh) + g4 * 16;
      const char* const vs_ = at(a.v, key, kvh) + g4 * 16;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        kf[k][ks] = *reinterpret_cast<const u32x4*>(ks_ + ks * 64);
        vf[k][ks] = *reinterpret_cast<const u32x4*>(vs_ + ks * 64);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) dk[k][db] = dv[k][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // pairs from which on this wavefront's first and last key are seen
    const int* const first = a.plan.first + s.off;
    const int from = first[min(w0, s.n_real - 1)] * group, free = first[min(w0 + KW, s.n_real) - 1] * group;
    stages(first[t0] * group / SP, (n_pairs + SP - 1) / SP,
           [&](int st, const u32x4* cur, const PairStats& ps) __attribute__((always_inline)) {
#pragma unroll 1
             for (int h = 0; h < SP / 32; ++h) {
               const int c0 = st * SP + h * 32;
               if (c0 + 32 <= from) continue;        // uniform: no pair sees this wavefront's keys
               // (before `free` some pair does not see some key)
               dkv_step<HD, NK, M>(cur + 2 * h * BU, cur + (SB + 2 * h) * BU, ps, c0 % 64, kf, vf, dk, dv, scale2, lane,
                                   c0 < free, ps.seen, [&](int k, int seen) { return seen <= w0 + k * 16 + c16; });
             }
           });
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int key = w0 + k * 16 + c16;
      if (key < s.n_real) store_dkv<HD, M>(a, s.off + key, kvh, dk[k], dv[k], g4);
    }
    return;
  }

  // mask rows (and padding)
  const int w0 = t0 + wave * 16, mine = w0 + c16;
  const int4 e = order[min(mine, s.cap - 1)];
  const bool branch = mine <= last && e.x >= s.n_real;
  const uint32_t chain_left = branch ? e.w - mine : 0;   // places that see this row, from its own on
  f32x4 dk[1][DB], dv[1][DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[0][db] = dv[0][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (t0 <= last) {                                  // uniform
    u32x4 kf[1][KS], vf[1][KS];
    const uint32_t r = s.off + (mine <= last ? e.x : 0);
    const char* const ks_ = at(a.k, r, kvh) + g4 * 16;
    const char* const vs_ = at(a.v, r, kvh) + g4 * 16;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[0][ks] = *reinterpret_cast<const u32x4*>(ks_ + ks * 64);
      vf[0][ks] = *reinterpret_cast<const u32x4*>(vs_ + ks * 64);
    }
    const int from = w0 * group, end = w0 <= last ? order[min(w0 + 15, last)].w * group : 0;   // this wavefront's pairs
    stages(t0 * group / SP, (order[min(t0 + 63, last)].w * group + SP - 1) / SP,
           [&](int st, const u32x4* cur, const PairStats& ps) __attribute__((always_inline)) {
#pragma unroll 1
             for (int h = 0; h < SP / 32; ++h) {
               const int c0 = st * SP + h * 32;
               if (c0 >= end || c0 + 32 <= from) continue;   // uniform
               dkv_step<HD, 1, M>(cur + 2 * h * BU, cur + (SB + 2 * h) * BU, ps, c0 % 64, kf, vf, dk, dv, scale2, lane, true,
                                  ps.pos, [&](int, int pos) { return (uint32_t)(pos - mine) >= chain_left; });
             }
           });
  }
  if (mine > last) {                                 // (whatever the sample's rows hold)
#pragma unroll
    for (int db = 0; db < DB; ++db) dk[0][db] = dv[0][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (mine < s.cap && (branch || mine > last)) store_dkv<HD, M>(a, s.off + e.x, kvh, dk[0], dv[0], g4);
}

template <int HD, class M>
hipError_t launch_hd(const CodAttnArgs& a, hipStream_t st) {
  constexpr int NQ = 2;
  const int64_t tiles = (int64_t)a.n_tiles * a.n_kv, dq = tiles * (kCodTile / (64 * NQ)) * a.group;
  const int64_t real = tiles * (kCodTile / (64 * dkv_blocks(HD))), all = real + tiles * (kCodTile / 64);
  k_cod_dq<HD, NQ, M, true><<<(unsigned)dq, 256, 0, st>>>(a);
  k_cod_dq<HD, NQ, M, false><<<(unsigned)dq, 256, 0, st>>>(a);
  k_cod_dkv<HD, M><<<(unsigned)all, 256, 0, st>>>(a, (unsigned)real);
  return hipGetLastError();
}

}  // namespace

size_t cod_attn_grad_workspace(int64_t rows, int n_samples, int n_kv, int group) {
  return sizeof(PairStats) * (size_t)stats_blocks(rows, group, n_samples) * n_kv;
}

hipError_t launch_cod_attn_grad(int head_dim, int dtype, const CodAttnArgs& args, hipStream_t st) {
  CodAttnArgs a = args;
  a.stats_blocks = stats_blocks(a.rows, a.group, a.n_samples);
  if (head_dim == 64) return dtype == PARD_BF16 ? launch_hd<64, MmaBF16>(a, st) : launch_hd<64, MmaF16>(a, st);
  return dtype == PARD_BF16 ? launch_hd<128, MmaBF16>(a, st) : launch_hd<128, MmaF16>(a, st);
}

}  // namespace pard
