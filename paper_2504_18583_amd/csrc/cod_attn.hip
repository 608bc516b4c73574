// Attention over packed COD rows on gfx950 MFMA.
//
// In the plan's order a row attends to the real tokens 0 .. c (one run of rows
// in memory) and to the mask rows of its chain before it.  A workgroup of four
// wavefronts owns 64 NQ (row, head) pairs of one key head, in order; a
// wavefront 16 NQ of them.
//   * First the wavefront's own chains: at most 16 NQ / group + K - 1 keys, by
//     their places in the order, 32 at a time; K straight into operand
//     registers, V through the wavefront's quarter of an LDS buffer.
//   * Then all four walk the real tokens in stages of 64 keys through two LDS
//     buffers (LDS-DMA, the next stage in flight during the current one).  Only
//     stages around the wavefront's own tokens compare keys with rows.
// A tile is S^T = K Q^T, online softmax in base 2, O^T += V^T P^T, with the
// running maximum raised only when a score passes it by 2^kLazy.
//
// Bound: the SIMDs' issue.  On one sample of 8193 tokens (8 / 4 heads x 64: 250 us,
// 930 TFLOP/s of 1228 of a large product) a score costs an exponential and about
// four more instructions beside its share of the products, whose cycles and the
// rest's add up to 109 % of the kernel's: they overlap a little.  Rows of short
// samples pay more for each score: in a 1B layer (16 samples of 256 to 1024 tokens,
// 32 / 8 heads x 64: 250 us, 530 TFLOP/s) a row sees 400 keys, 16 % more scores are
// computed than seen (the last stages, the chains' 32 keys), and a pair's fixed
// work makes 8 instructions of a seen score's five; 8B heads (x 128, 6 samples of
// 900 to 2048) 505 us, 7.  Two tiles of 16 pairs a wavefront (NQ) share every LDS
// read (1B layer 302 us against 389 with one tile when that was measured).
// head_dim 128 with stages of 32 keys and a third workgroup a CU spilled (584 us).
// A scalar kernel, one wavefront per pair, took 24.8 ms.
#include "cod_attn_tile.h"

namespace pard {
namespace {

using namespace cod;

constexpr int kStageKeys = 64;
constexpr float kLazy = 8.f;

// Softmax of NB blocks of 16 keys: scores s become packed probabilities pf,
// running maximum m (base 2), sum l and output o follow.  Hidden scores are
// -infinity; m starts finite, so that a row without keys keeps l = 0.  The product
// takes probabilities of 16 bits (the sum does not): what is lost is of the size of
// the output's own rounding (1B layer, bf16: 2.2e-3 of the output's magnitude off,
// where rounding the exact output is 1.6e-3).
template <int NQ, int NB, int DB, class M>
__device__ __forceinline__ void softmax_step(const f32x4 (&s)[NQ][NB], float (&m)[NQ], float (&l)[NQ], f32x4 (&o)[NQ][DB],
                                             u32x4 (&pf)[NQ][NB / 2], float scale2) {
  bool raise = false;
  float mx[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    float v = fmaxf(s[t][0][0], s[t][0][1]);
#pragma unroll
    for (int i = 2; i < 4 * NB; i += 2) v = fmaxf(fmaxf(v, s[t][i / 4][i % 4]), s[t][i / 4][i % 4 + 1]);
    mx[t] = v * scale2;
    raise |= mx[t] > m[t] + kLazy;
  }
  if (__any(raise)) {                                // uniform
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const float mr = max4g(mx[t]);
      const float m_new = mr > m[t] + kLazy ? mr : m[t];
      const float corr = __builtin_amdgcn_exp2f(m[t] - m_new);
      m[t] = m_new;
      l[t] *= corr;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[t][db] *= corr;
    }
  }
#pragma unroll
  for (int t = 0; t < NQ; ++t)
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[t][kb][i], scale2, -m[t]));
        l[t] += p[i];
      }
      pf[t][kb >> 1][(kb & 1) * 2] = M::pack(p[0], p[1]);
      pf[t][kb >> 1][(kb & 1) * 2 + 1] = M::pack(p[2], p[3]);
    }
}

template <int HD, int NQ, class M>
__global__ __launch_bounds__(256, HD == 64 ? 4 : 2) void k_cod_attn(const CodAttnArgs a) {
  constexpr int QW = 16 * NQ;                        // pairs per wavefront
  constexpr int KS = HD / 32, DB = HD / 16, BU = kBlockUnits<HD>;
  // a stage: four blocks of K, four of V; two arrays of their own (the
  // compiler's waits before an LDS read cover the loads into that array only)
  __shared__ __attribute__((aligned(16))) u32x4 b0[8 * BU], b1[8 * BU];
  const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = a.group, per_tile = kCodTile / (64 * NQ) * group;   // workgroups of a tile and key head
  const int kvh = blockIdx.x % a.n_kv, rest = blockIdx.x / a.n_kv;
  const CodTileInfo tile = a.plan.tiles[rest / per_tile];
  const CodSampleInfo s = tile.s;
  const int pair0 = (rest % per_tile) * 64 * NQ, p0 = tile.tile * kCodTile;
  if (p0 + pair0 / group >= s.cap) return;           // uniform: the whole block leaves
  const int4* const order = a.plan.order + s.off;
  const int last = s.len - 1;

  // The places of this lane's pairs (those past the sample repeat its last row
  // and are not stored) and of the keys before them are read at once, then the
  // rows they name: two round trips to memory before the first product.
  const int w_row0 = p0 + (pair0 + wave * QW) / group;             // of this wavefront's pairs
  const int w_last = min(p0 + (pair0 + (wave + 1) * QW - 1) / group, last);
  const int chain0 = max(w_row0 - s.reach, 0);
  int row[NQ], head[NQ];                             // this pair's place and query head
  int4 e[NQ] = {};                                   // packed row, real tokens seen, first mask row seen (and chain's end)
  u32x4 q[NQ][KS];
  float m[NQ], l[NQ];
  f32x4 o[NQ][DB];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const int pair = pair0 + wave * QW + t * 16 + c16, r = quotient(pair, a.by_group);
    row[t] = p0 + r;
    head[t] = kvh * group + remainder(pair, r, a.by_group);
    m[t] = -1e30f;
    l[t] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[t][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (last >= p0 + pair0 / group) {                  // uniform: the block has rows
    const uint64_t k_step = a.k.rs, v_step = a.v.rs;
    const char* const k0 = at(a.k, s.off, kvh);
    const char* const v0 = at(a.v, s.off, kvh);
    // this wavefront's 16 keys of every stage (past the real tokens: the last one)
    auto load = [&](u32x4* buf, int st) __attribute__((always_inline)) {
      const int key = min(st * kStageKeys + wave * 16 + block_row(lane), s.n_real - 1);
      load_block<HD>(k0 + (uint32_t)key * k_step + block_byte(lane), buf + wave * BU);
      load_block<HD>(v0 + (uint32_t)key * v_step + block_byte(lane), buf + (4 + wave) * BU);
    };
    const int st_seen = order[min(p0 + (pair0 + 64 * NQ - 1) / group, last)].y;
    const int last_seen = w_row0 > last ? 0 : order[w_last].y;
    int k_row[2], v_row[2];                          // 32 keys from c0 on
    auto chain_rows = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        k_row[b] = order[min(c0 + b * 16 + c16, last)].x;
        v_row[b] = order[min(c0 + b * 16 + block_row(lane), last)].x;
      }
    };
#pragma unroll
    for (int t = 0; t < NQ; ++t) e[t] = order[min(row[t], last)];
    chain_rows(chain0);
    load(b0, 0);
    const uint32_t sign = scale_sign(a.scale);
    const float scale2 = base2_scale(a.scale);
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const char* src = at(a.q, s.off + e[t].x, head[t]) + g4 * 16;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[t][ks] = *reinterpret_cast<const u32x4*>(src + ks * 64);
    }
    // the wavefront's chains
    u32x4* const mine = b1 + wave * 2 * BU;
    u32x4 kf[2][KS];
    auto load_chain = [&](int next) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[b][ks] = *reinterpret_cast<const u32x4*>(k0 + (uint32_t)k_row[b] * k_step + g4 * 16 + ks * 64);
        load_block<HD>(v0 + (uint32_t)v_row[b] * v_step + block_byte(lane), mine + b * BU);
      }
      if (next <= w_last) chain_rows(next);          // uniform
    };
    if (s.reach > 0) load_chain(chain0 + 32);        // uniform
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[t][ks][i] ^= sign;
    uint32_t own[NQ];                                // mask rows of its chain that a row sees, itself included
#pragma unroll
    for (int t = 0; t < NQ; ++t) own[t] = min(row[t], last) - e[t].z + 1;
    for (int c0 = chain0; c0 <= w_last && s.reach > 0; c0 += 32) {           // uniform
      f32x4 sc[NQ][2];
#pragma unroll
      for (int t = 0; t < NQ; ++t) sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int t = 0; t < NQ; ++t) sc[t][b] = M::mma(kf[b][ks], q[t][ks], sc[t][b]);
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if ((uint32_t)(c0 + b * 16 + g4 * 4 + i - e[t].z) >= own[t]) sc[t][b][i] = -INFINITY;
          }
      u32x4 pf[NQ][1];
      softmax_step<NQ, 2, DB, M>(sc, m, l, o, pf, scale2);
      wait_all();
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const u32x4 vf = cols_frag<HD>(mine, db, lane);
#pragma unroll
        for (int t = 0; t < NQ; ++t) o[t][db] = M::mma(vf, pf[t][0], o[t][db]);
      }
      wait_all();                                    // (its reads are done before the next loads)
      if (c0 + 32 <= w_last) load_chain(c0 + 64);    // uniform
    }

    const int first_seen = __builtin_amdgcn_readfirstlane(e[0].y);           // of this wavefront's pairs
    const int n_st = (st_seen + kStageKeys - 1) / kStageKeys;
    auto stage = [&](int st, const u32x4* cur, u32x4* nxt) __attribute__((always_inline)) {
      wait_and_meet();
      if (st + 1 < n_st) load(nxt, st + 1);          // uniform
      __builtin_amdgcn_sched_barrier(0);
      const int key0 = st * kStageKeys;
      if (key0 >= last_seen) return;                 // uniform: past this wavefront's rows
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
      if (key0 + kStageKeys > first_seen) {          // uniform: around this wavefront's own tokens
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + kb * 16 + g4 * 4 + i >= e[t].y) sc[t][kb][i] = -INFINITY;
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
    int st = 0;
    for (; st + 2 <= n_st; st += 2) {
      stage(st, b0, b1);
      stage(st + 1, b1, b0);
    }
    if (st < n_st) stage(st, b0, b1);
  }

  // lane (c16, g4) holds elements 16 db + 4 g4 .. + 3 of pair 16 t + c16
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const float sum = sum4g(l[t]);
    if (row[t] >= s.cap) continue;
    const bool real = row[t] <= last;
    const uint32_t r = s.off + (real ? e[t].x : order[row[t]].x);
    const float inv = __builtin_amdgcn_rcpf(sum);    // (1 ulp of float32, before the rounding to 16 bits)
    char* const dst = at(a.out, r, head[t]) + g4 * 8;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const f32x4 v = real ? o[t][db] * inv : f32x4{0.f, 0.f, 0.f, 0.f};
      *reinterpret_cast<u32x2*>(dst + db * 32) = u32x2{M::pack(v[0], v[1]), M::pack(v[2], v[3])};
    }
    if (a.lse && g4 == 0)
      a.lse[head[t] * a.rows + r] = real ? (m[t] + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
  }
}

template <int HD, class M>
hipError_t launch_hd(const CodAttnArgs& a, hipStream_t st) {
  constexpr int NQ = 2;
  const int64_t blocks = (int64_t)a.n_tiles * (kCodTile / (64 * NQ)) * a.group * a.n_kv;
  k_cod_attn<HD, NQ, M><<<(unsigned)blocks, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cod_attn(int head_dim, int dtype, const CodAttnArgs& a, hipStream_t st) {
  if (head_dim == 64) return dtype == PARD_BF16 ? launch_hd<64, MmaBF16>(a, st) : launch_hd<64, MmaF16>(a, st);
  return dtype == PARD_BF16 ? launch_hd<128, MmaBF16>(a, st) : launch_hd<128, MmaF16>(a, st);
}

}  // namespace pard
