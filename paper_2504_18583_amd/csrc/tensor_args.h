// Checks of the tensors that the operators' entry points are given (host only).
#pragma once

#include "train.h"

namespace pard {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

inline pard_status status_of(hipError_t e) { return e == hipSuccess ? PARD_OK : PARD_ERR_DEVICE; }

inline int elem_size(int dtype) { return dtype == PARD_F32 ? 4 : dtype == PARD_BF16 || dtype == PARD_F16 ? 2 : 0; }

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A tensor of `heads` heads of `hd` elements in `rows` rows that is read, or
// (out) written: then no two of its heads share an element.
inline bool heads_ok(const pard_heads* t, int64_t rows, int heads, int hd, bool out) {
  if (!t || t->row_stride < 0 || t->head_stride < 0) return false;
  if (rows == 0 || heads == 0) return true;
  if (!t->data) return false;
  if (!out) return true;
  // heads within a row, or rows within a head
  const __int128 r = t->row_stride, h = t->head_stride;
  const bool by_row = (heads == 1 || h >= hd) && (rows == 1 || r >= h * (heads - 1) + hd);
  const bool by_head = (rows == 1 || r >= hd) && (heads == 1 || h >= r * (rows - 1) + hd);
  return by_row || by_head;
}

// Whether an output may lie where an input does: as the input, or apart from it
// (overlaps of tensors that start elsewhere are the caller's to avoid).
inline bool apart(const pard_heads* a, const pard_heads* b) { return a->data != b->data; }
inline bool same_or_apart(const pard_heads* a, const pard_heads* b, int64_t rows, int heads) {
  return apart(a, b) || ((rows == 1 || a->row_stride == b->row_stride) && (heads == 1 || a->head_stride == b->head_stride));
}

inline Heads view(const pard_heads* t) {
  return t ? Heads{static_cast<char*>(t->data), t->row_stride, t->head_stride} : Heads{nullptr, 0, 0};
}

inline Heads16 view16(const pard_heads* t) {
  return Heads16{static_cast<char*>(t->data), (uint32_t)(2 * t->row_stride), (uint32_t)(2 * t->head_stride)};
}

inline FastDiv fast_div(int d) {
  FastDiv f{};
  f.d = d;
  while ((1u << f.l) < f.d) ++f.l;
  f.m = (uint32_t)(((1ull << (30 + f.l)) + f.d - 1) / f.d);
  return f;
}

}  // namespace pard
