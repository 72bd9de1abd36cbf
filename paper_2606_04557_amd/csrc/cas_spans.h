// Which bytes strided tensors cover, and whether two of them share any (host only).
#pragma once

#include <stdint.h>

#include <numeric>
#include <utility>

namespace cas {

// What a strided [tokens, heads, head_dim] tensor covers, in bytes: rows of
// `ext` bytes (of one or several heads or tokens), `stride` apart, made of pieces of
// `width` bytes (a head), `inner` apart (0: one piece).
struct Footprint {
  uintptr_t base, end;
  uint64_t stride, ext, inner, width;
  bool distinct;   // no two elements share an address
};

inline Footprint footprint(const void *x, int64_t tokens, int64_t heads, int64_t st, int64_t sh, int64_t D, int es) {
  int64_t outer = st, n_outer = tokens, inner = sh, n_inner = heads;
  if (n_outer == 1 || (n_inner > 1 && inner > outer)) {
    std::swap(outer, inner);
    std::swap(n_outer, n_inner);
  }
  const int64_t in = n_inner > 1 ? inner : 0, out = n_outer > 1 ? outer : 0;
  Footprint f;
  f.base = (uintptr_t)x;
  f.width = (uint64_t)D * es;
  f.inner = (uint64_t)in * es;
  f.ext = (uint64_t)(n_inner - 1) * f.inner + f.width;
  f.stride = (uint64_t)out * es;
  f.end = f.base + (uint64_t)(n_outer - 1) * f.stride + f.ext;
  f.distinct = (n_inner == 1 || in >= D) && (n_outer == 1 || f.stride >= f.ext);
  return f;
}

// The footprint of `bytes` bytes in a row.
inline Footprint span_of(const void *x, uint64_t bytes) {
  return Footprint{(uintptr_t)x, (uintptr_t)x + bytes, 0, bytes, 0, bytes, true};
}

// Two tensors that share a range of addresses are still apart when their rows
// interleave (slices of one projection's output, [tokens, Hq + 2 Hkv, d]), or their
// heads do ([tokens, heads, 3, d]): counted modulo a step that divides all their
// strides, every row (or head) of a tensor lies in the same place.
inline bool apart(const Footprint &a, const Footprint &b) {
  if (a.end <= b.base || b.end <= a.base) return true;
  auto modulo = [&](uint64_t step, uint64_t wa, uint64_t wb) {
    if (step == 0) return false;
    const uint64_t delta = b.base >= a.base ? (b.base - a.base) % step : (step - (a.base - b.base) % step) % step;
    return delta >= wa && delta + wb <= step;
  };
  const uint64_t rows = std::gcd(a.stride, b.stride);
  return modulo(rows, a.ext, b.ext) || modulo(std::gcd(rows, std::gcd(a.inner, b.inner)), a.width, b.width);
}

}  // namespace cas
