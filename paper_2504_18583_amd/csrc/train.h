// Mask-token training operators (rotary positions, attention over packed COD
// rows, the loss): argument blocks of the kernels, and element conversions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/pard.h"

namespace pard {

// Stored element types: to and from float (rounded to nearest even).
struct ElemF32 {
  using T = float;
  static __device__ __forceinline__ float load(T v) { return v; }
  static __device__ __forceinline__ T store(float v) { return v; }
};
struct ElemBF16 {
  using T = uint16_t;
  static __device__ __forceinline__ float load(T v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ T store(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};
struct ElemF16 {
  using T = uint16_t;
  static __device__ __forceinline__ float load(T v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ T store(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

// One [rows][heads][head_dim] tensor (element strides).
struct Heads {
  char* data;
  int64_t rs, hs;
};

struct RopeArgs {
  int rows, n_q, n_k, hd, rot, n_pos;
  float eps;
  const int32_t* pos;
  const float2* table;
  const float *q_gain, *k_gain;     // null: no norm
  Heads q_in, k_in;                 // forward: x; gradient: dy
  Heads q_x, k_x;                   // gradient of the norm: the forward call's x
  Heads q_out, k_out;               // y or dx
  float* part;                      // gradient of the norm: [blocks][2][hd] partial gain gradients
};
// Workgroups that leave partial gain gradients.
int rope_grad_blocks(const RopeArgs& a);
hipError_t launch_rope_spec_table(const pard_rope_spec& s, int n_pos, float2* table, hipStream_t st);
// grad: the gradient; with gains its workgroups' partial sums are summed and
// written to q_dgain and k_dgain by a second launch.
hipError_t launch_qk_rope(int dtype, int layout, bool grad, const RopeArgs& a, float* q_dgain, float* k_dgain,
                          hipStream_t st);

// Plan of a batch of packed samples.  In a sample, a row (k, j) belongs to the
// chain c = j - k + 1, which starts with the real token of column c; `order`
// positions number the rows by (c, k), so that every row attends to the real
// tokens 0 .. c (subtask 1's rows, contiguous in the packed order) and to the
// rows of its own chain before it: no other row is ever looked at.
constexpr int kCodTile = 128;              // order positions of a tile
constexpr int kCodMaxSections = 64;
struct CodSampleInfo {
  int off, len, n_real, cap;               // region start, rows, subtask 1's rows, region size
  int reach;                               // rows of a chain before its last at most (largest subtask - 1)
};
struct CodTileInfo {
  CodSampleInfo s;
  int sample, tile, pad;
};
struct CodPlanView {
  // [off + position]: packed row in the region, real tokens it sees, position
  // of its chain's first mask row, end of its chain; padding rows follow the
  // sample's (0 real tokens)
  int4* order;
  int* first;                              // [off + real token]: its position
  CodSampleInfo* samples;
  CodTileInfo* tiles;                      // later tiles first
  CodTileInfo* by_sample;                  // samples with the most tiles first, each one's tiles in order
  int64_t* offsets;                        // the caller's out_offsets
  int* bad;                                // nonzero: rows not in the documented form
};
size_t cod_plan_layout(int64_t rows, int n_samples, void* data, CodPlanView* v);
hipError_t launch_cod_plan(const int32_t* section, const int32_t* column, const int32_t* out_len, int n_samples,
                           int max_region, const CodPlanView& v, hipStream_t st);

// Tensor of 16-bit elements: strides in bytes.  32-bit strides make an address
// one multiply-add per index.
struct Heads16 {
  char* data;
  uint32_t rs, hs;
};
// Division of 0 <= x < 2^30 by d <= 1024: x / d = (x m) >> (30 + l) with m =
// ceil(2^(30 + l) / d), l = ceil(log2 d) (m d exceeds 2^(30 + l) by less than
// d <= 2^l, which times x stays below 2^(30 + l)).
struct FastDiv {
  uint32_t m, l, d;
};
struct CodAttnArgs {
  CodPlanView plan;
  int n_tiles, n_samples, n_heads, n_kv, group;
  FastDiv by_group;
  int64_t rows;                            // of lse
  float scale;
  Heads16 q, k, v, out;
  float* lse;                              // forward: written (may be null); gradient: read
  Heads16 d_out, dq, dk, dv;
  void* stats;                             // gradient: the pairs' statistics (workspace)
  int64_t stats_blocks;                    // blocks of 64 pairs of a key head
};
size_t cod_attn_grad_workspace(int64_t rows, int n_samples, int n_kv, int group);
hipError_t launch_cod_attn(int head_dim, int dtype, const CodAttnArgs& a, hipStream_t st);
hipError_t launch_cod_attn_grad(int head_dim, int dtype, const CodAttnArgs& a, hipStream_t st);

struct CodLossArgs {
  int rows, vocab, n_sections;
  const char* logits;
  int64_t stride;
  const int32_t *labels, *section;
  char* d_logits;
  int64_t d_stride;
  float grad_scale;
  int weighted;                            // 0: the mean over all counted rows
  float weights[kCodMaxSections];
  float *loss, *row_loss;
  int* counts;                             // workspace: [kLossCountBlocks][kCodMaxSections]
  int* ticket;                             // workspace: finished workgroups
  double* sums;                            // workspace: [workgroups][n_sections]
};
constexpr int kLossMaxBlocks = 4096;       // workgroups of the rows
constexpr int kLossCountBlocks = 16;
hipError_t launch_cod_loss(int dtype, const CodLossArgs& a, hipStream_t st);

}  // namespace pard
