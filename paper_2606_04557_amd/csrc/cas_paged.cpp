// Host side of the rotary positions, of appending to the paged cache and of the
// chunk attention over it: argument validation, plans and launches. Validation is host code and runs
// before any HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <chrono>
#include <cmath>
#include <cstring>
#include <exception>
#include <functional>
#include <map>
#include <memory>
#include <mutex>
#include <numeric>
#include <string>
#include <thread>
#include <tuple>
#include <vector>

#include "../../include/cas.h"
#include "cas_host.h"
#include "cas_internal.h"

using namespace cas;

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
std::string str(int64_t x) { return std::to_string(x); }

// No exception leaves a C entry (host memory for the plan's tables may run out).
template <typename F>
cas_status_t guarded(F &&f) {
  try {
    return f();
  } catch (const std::exception &e) {
    return set_error(CAS_ERR_UNSUPPORTED, std::string("host memory: ") + e.what());
  }
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
cas_status_t check_rope(const cas_rope_t *r, int head_dim) {
  if (!r) return set_error(CAS_ERR_INVALID_ARGUMENT, "rope is NULL");
  if (r->layout != CAS_ROPE_HALF && r->layout != CAS_ROPE_INTERLEAVED)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "unknown rope layout");
  if (r->rotary_dim < 16 || r->rotary_dim > head_dim || r->rotary_dim % 16)
    return set_error(CAS_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in [16, head_dim]");
  if (!std::isfinite(r->scale) || !(r->scale > 0.0f)) return set_error(CAS_ERR_INVALID_ARGUMENT, "rope scale must be finite and > 0");
  if (!r->turns) return set_error(CAS_ERR_INVALID_ARGUMENT, "rope turns is NULL");
  if ((uintptr_t)r->turns & 7u) return set_error(CAS_ERR_ALIGNMENT, "rope turns must be 8-byte aligned");
  return CAS_OK;
}

DevRope dev_rope(const cas_rope_t *r, bool inverse) {
  return DevRope{r->turns, r->rotary_dim, r->scale, r->layout == CAS_ROPE_INTERLEAVED, inverse};
}

// What a strided [tokens, heads, head_dim] tensor covers, in bytes: rows of
// `ext` bytes (of one or several heads or tokens), `stride` apart, made of pieces of
// `width` bytes (a head), `inner` apart (0: one piece).
struct Footprint {
  uintptr_t base, end;
  uint64_t stride, ext, inner, width;
  bool distinct;   // no two elements share an address
};

Footprint footprint(const void *x, int64_t tokens, int64_t heads, int64_t st, int64_t sh, int D, int es) {
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
Footprint span_of(const void *x, uint64_t bytes) {
  return Footprint{(uintptr_t)x, (uintptr_t)x + bytes, 0, bytes, 0, bytes, true};
}

// Two tensors that share a range of addresses are still apart when their rows
// interleave (slices of one projection's output, [tokens, Hq + 2 Hkv, d]), or their
// heads do ([tokens, heads, 3, d]): counted modulo a step that divides all their
// strides, every row (or head) of a tensor lies in the same place.
bool apart(const Footprint &a, const Footprint &b) {
  if (a.end <= b.base || b.end <= a.base) return true;
  auto modulo = [&](uint64_t step, uint64_t wa, uint64_t wb) {
    if (step == 0) return false;
    const uint64_t delta = b.base >= a.base ? (b.base - a.base) % step : (step - (a.base - b.base) % step) % step;
    return delta >= wa && delta + wb <= step;
  };
  const uint64_t rows = std::gcd(a.stride, b.stride);
  return modulo(rows, a.ext, b.ext) || modulo(std::gcd(rows, std::gcd(a.inner, b.inner)), a.width, b.width);
}

constexpr int64_t kMaxStride = (int64_t)1 << 31;   // (with the limits on tokens and heads, spans fit 64 bits)
constexpr int64_t kMaxRopeTokens = (int64_t)1 << 24;   // (two or more to a workgroup of 256: under 2^32 threads)

cas_status_t check_strides(const char *what, int64_t st, int64_t sh, int es) {
  if (st < 0 || sh < 0 || st > kMaxStride || sh > kMaxStride)
    return set_error(CAS_ERR_INVALID_ARGUMENT, std::string(what) + ": strides must be in [0, 2^31]");
  if (((st | sh) * es) % 16) return set_error(CAS_ERR_ALIGNMENT, std::string(what) + ": strides must be multiples of 16 bytes");
  return CAS_OK;
}

// Heads of one token that the threads of a workgroup take at a time, no more
// than its tensor has (rounded up). Every thread computes its angles, so few
// slots save arithmetic and many spread a few tokens over more threads. us with
// 32 / 16 / 8 / 4 slots, 32 query and 8 key heads of 128 in one call: bf16 2.7 /
// 3.0 / 3.1 / 3.9 at 64 tokens, 3.4 / 3.3 / 3.4 / 4.1 at 256, 4.5 / 4.3 / 3.7 / 5.2
// at 512, 38.3 / 34.4 / 32.9 / 33.7 at 8192; fp32, whose threads have twice the
// bytes for their angles, 3.1 / 3.4 / 3.9 / 5.2, 4.5 / 4.3 / 5.4 / 7.0, 6.8 / 6.7 /
// 7.0 / 7.9 and 61.4 / 61.6 / 64.3 / 68.2.
int head_slots(int64_t tokens, int D, int es, int heads) {
  int slots = tokens < 512 ? 256 / (D / 16) : 4 * es;
  while (slots > 1 && slots / 2 >= heads) slots /= 2;
  return slots;
}

cas_status_t rope_call(const cas_rope_t *rope, int32_t dtype, int32_t D, int64_t tokens, const int32_t *positions,
                       const cas_rope_tensor_t *ts, int32_t n, int32_t inverse, hipStream_t stream) {
  if (dtype != CAS_DTYPE_BF16 && dtype != CAS_DTYPE_FP32) return set_error(CAS_ERR_UNSUPPORTED, "dtype must be bf16 or fp32");
  if (D != 64 && D != 128) return set_error(CAS_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  cas_status_t s = check_rope(rope, D);
  if (s != CAS_OK) return s;
  if (tokens < 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "tokens must be >= 0");
  if (tokens > kMaxRopeTokens) return set_error(CAS_ERR_UNSUPPORTED, "more than 2^24 tokens");
  if (n < 1 || n > 4 || !ts) return set_error(CAS_ERR_INVALID_ARGUMENT, "1 to 4 tensors");
  if (tokens == 0) return CAS_OK;
  if (!positions) return set_error(CAS_ERR_INVALID_ARGUMENT, "positions is NULL");
  if ((uintptr_t)positions & 3u) return set_error(CAS_ERR_ALIGNMENT, "positions must be 4-byte aligned");
  const int es = dtype == CAS_DTYPE_BF16 ? 2 : 4;
  RopeParams p{};
  Footprint in[4], out[4];
  for (int i = 0; i < n; ++i) {
    const cas_rope_tensor_t &t = ts[i];
    auto refuse = [&](cas_status_t code, const char *why) { return set_error(code, "tensor " + str(i) + ": " + why); };
    if (!t.x || !t.y) return refuse(CAS_ERR_INVALID_ARGUMENT, "x and y must be non-NULL");
    if (t.heads < 1 || t.heads > (1 << 16)) return refuse(CAS_ERR_INVALID_ARGUMENT, "heads must be in [1, 2^16]");
    if (!aligned16(t.x) || !aligned16(t.y)) return refuse(CAS_ERR_ALIGNMENT, "x and y must be 16-byte aligned");
    if ((s = check_strides("x", t.x_stride_tok, t.x_stride_head, es)) != CAS_OK) return s;
    if ((s = check_strides("y", t.y_stride_tok, t.y_stride_head, es)) != CAS_OK) return s;
    in[i] = footprint(t.x, tokens, t.heads, t.x_stride_tok, t.x_stride_head, D, es);
    out[i] = footprint(t.y, tokens, t.heads, t.y_stride_tok, t.y_stride_head, D, es);
    if (!out[i].distinct) return refuse(CAS_ERR_INVALID_ARGUMENT, "y overlaps itself");
    p.t[i] = DevRopeTensor{t.x, t.y, t.x_stride_tok, t.x_stride_head, t.y_stride_tok, t.y_stride_head, t.heads,
                            head_slots(tokens, D, es, t.heads)};
  }
  const Footprint pos = span_of(positions, (uint64_t)tokens * 4), turns = span_of(rope->turns, (uint64_t)rope->rotary_dim * 4);
  for (int i = 0; i < n; ++i) {
    auto refuse = [&](const std::string &what) {
      return set_error(CAS_ERR_INVALID_ARGUMENT, "tensor " + str(i) + ": y overlaps " + what);
    };
    if (!apart(out[i], pos) || !apart(out[i], turns)) return refuse("positions or turns");
    for (int j = 0; j < n; ++j) {
      const bool in_place = i == j && ts[i].x == ts[i].y && (tokens == 1 || ts[i].x_stride_tok == ts[i].y_stride_tok) &&
                            (ts[i].heads == 1 || ts[i].x_stride_head == ts[i].y_stride_head);
      if (!in_place && !apart(out[i], in[j])) return refuse("the x of tensor " + str(j));
      if (i != j && !apart(out[i], out[j])) return refuse("the y of tensor " + str(j));
    }
  }
  p.rope = dev_rope(rope, inverse != 0);
  p.positions = positions;
  p.tokens = tokens;
  const hipError_t e = timed_launch("rope", stream, [&] { return launch_rope(p, dtype == CAS_DTYPE_BF16 ? kBF16 : kFP32, D, n, stream); });
  return e == hipSuccess ? CAS_OK : set_hip_error("rope launch", e);
}

// ---------------------------------------------------------------------------
// Tables of paged requests
// ---------------------------------------------------------------------------
// As the paged decode checks them, except that requests without new tokens (and
// without keys) are allowed: a padded batch has some.
cas_status_t check_paged(const cas_decode_problem_t *p) {
  if (!p) return set_error(CAS_ERR_INVALID_ARGUMENT, "problem is NULL");
  if (p->batch < 1 || p->num_kv_heads < 1 || p->group_size < 1)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "batch, num_kv_heads and group_size must be >= 1");
  if (p->head_dim != 64 && p->head_dim != 128) return set_error(CAS_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  const int P = p->page_size;
  if (P != 16 && P != 32 && P != 64 && P != 128) return set_error(CAS_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  const int64_t Hq = (int64_t)p->num_kv_heads * p->group_size;
  if (Hq > (1 << 16)) return set_error(CAS_ERR_UNSUPPORTED, "num_kv_heads*group_size above 2^16");
  if ((int64_t)P * p->num_kv_heads * p->head_dim * 2 >= ((int64_t)1 << 31))
    return set_error(CAS_ERR_UNSUPPORTED, "page larger than 2 GiB");
  if (p->num_pages < 1) return set_error(CAS_ERR_INVALID_ARGUMENT, "num_pages must be >= 1");
  if (!p->q_offsets || !p->kv_lens || !p->page_offsets || !p->page_ids)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "q_offsets, kv_lens, page_offsets and page_ids must be non-NULL");
  if (p->q_offsets[0] != 0 || p->page_offsets[0] != 0)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "q_offsets[0] and page_offsets[0] must be 0");
  for (int b = 0; b < p->batch; ++b) {
    const int64_t n = (int64_t)p->q_offsets[b + 1] - p->q_offsets[b], L = p->kv_lens[b];
    const std::string name = "request " + str(b);
    if (n < 0) return set_error(CAS_ERR_INVALID_ARGUMENT, name + ": q_offsets decrease");
    if (L < n) return set_error(CAS_ERR_INVALID_ARGUMENT, name + ": kv_len below its new tokens");
    if (L > (1 << 30)) return set_error(CAS_ERR_UNSUPPORTED, name + ": more than 2^30 keys");
    if ((int64_t)p->page_offsets[b + 1] - p->page_offsets[b] != ceil_div(L, P))
      return set_error(CAS_ERR_INVALID_ARGUMENT, name + ": page count must be ceil(kv_len / page_size)");
  }
  if ((int64_t)p->q_offsets[p->batch] * Hq > INT32_MAX) return set_error(CAS_ERR_UNSUPPORTED, "new tokens * heads above 2^31");
  for (int32_t i = 0; i < p->page_offsets[p->batch]; ++i)
    if (p->page_ids[i] < 0 || p->page_ids[i] >= p->num_pages)
      return set_error(CAS_ERR_INVALID_ARGUMENT, "page id " + str(i) + " out of range");
  return CAS_OK;
}

// A problem with copies of its tables.
struct OwnedProblem {
  cas_decode_problem_t p;
  std::vector<int32_t> tables;   // q_offsets, kv_lens, page_offsets, page_ids

  void assign(const cas_decode_problem_t &o) {
    const size_t B = (size_t)o.batch, ids = (size_t)o.page_offsets[B];
    tables.clear();
    tables.reserve(3 * B + 2 + ids);
    auto copy = [&](const int32_t *src, size_t n) {
      const int32_t *at = tables.data() + tables.size();
      tables.insert(tables.end(), src, src + n);
      return at;
    };
    p = o;
    p.q_offsets = copy(o.q_offsets, B + 1);
    p.kv_lens = copy(o.kv_lens, B);
    p.page_offsets = copy(o.page_offsets, B + 1);
    p.page_ids = copy(o.page_ids, ids);
  }
  bool matches(const cas_decode_problem_t *q) const {
    if (!q || !q->q_offsets || !q->kv_lens || !q->page_offsets || !q->page_ids) return false;
    if (q->batch != p.batch || q->num_kv_heads != p.num_kv_heads || q->group_size != p.group_size || q->head_dim != p.head_dim ||
        q->softmax_scale != p.softmax_scale || q->page_size != p.page_size || q->num_pages != p.num_pages)
      return false;
    auto same = [](const int32_t *a, const int32_t *b, size_t n) { return std::memcmp(a, b, n * sizeof(int32_t)) == 0; };
    const size_t B = (size_t)p.batch;
    return same(q->q_offsets, p.q_offsets, B + 1) && same(q->kv_lens, p.kv_lens, B) &&
           same(q->page_offsets, p.page_offsets, B + 1) && same(q->page_ids, p.page_ids, (size_t)p.page_offsets[B]);
  }
};

// ---------------------------------------------------------------------------
// Appending to the paged cache
// ---------------------------------------------------------------------------
// Refuses tables whose new tokens would be written to a row which is someone
// else's key, or a key twice.
cas_status_t check_append(const cas_decode_problem_t *p) {
  cas_status_t s = check_paged(p);
  if (s != CAS_OK) return s;
  const int P = p->page_size, B = p->batch;
  struct Write {
    int32_t page, lo, hi, entry;   // rows [lo, hi) of a page, named by page_ids[entry]
  };
  std::vector<Write> w;
  for (int b = 0; b < B; ++b) {
    const int32_t n = p->q_offsets[b + 1] - p->q_offsets[b], L = p->kv_lens[b], e0 = p->page_offsets[b];
    for (int32_t k = L - n; k < L;) {
      const int32_t j = k / P, lo = k % P, hi = (int32_t)std::min<int64_t>(P, lo + (int64_t)(L - k));
      w.push_back({p->page_ids[e0 + j], lo, hi, e0 + j});
      k += hi - lo;
    }
  }
  if (w.empty()) return CAS_OK;
  std::sort(w.begin(), w.end(), [](const Write &a, const Write &b) { return a.page != b.page ? a.page < b.page : a.lo < b.lo; });
  auto refuse = [&](int32_t page) {
    return set_error(CAS_ERR_INVALID_ARGUMENT, "page " + str(page) + ": new tokens would overwrite a key that the tables name elsewhere");
  };
  for (size_t i = 1; i < w.size(); ++i)
    if (w[i].page == w[i - 1].page && w[i].lo < w[i - 1].hi) return refuse(w[i].page);
  // Every other place that names a written page. A bit for the low 16 bits of
  // each written id passes over nearly all entries at once.
  std::vector<uint64_t> bits(1024, 0);
  for (const Write &x : w) bits[(x.page & 0xffff) >> 6] |= 1ull << (x.page & 63);
  for (int b = 0; b < B; ++b)
    for (int32_t e = p->page_offsets[b]; e < p->page_offsets[b + 1]; ++e) {
      const int32_t id = p->page_ids[e];
      if (!(bits[(id & 0xffff) >> 6] >> (id & 63) & 1)) continue;
      const int64_t seen = std::min<int64_t>(P, (int64_t)p->kv_lens[b] - (int64_t)(e - p->page_offsets[b]) * P);
      auto it = std::lower_bound(w.begin(), w.end(), id, [](const Write &a, int32_t v) { return a.page < v; });
      for (; it != w.end() && it->page == id; ++it)
        if (it->entry != e && it->lo < seen) return refuse(id);
    }
  return CAS_OK;
}

// New tokens of a workgroup. Few tokens are spread over as many threads as their
// heads fill; many share their angles between heads, and their page ids between
// tokens. 64 requests of one token take 2.9 us with 1, 3.1 with 4 and 3.6 with 16
// tokens to a workgroup; 800 tokens 7.1, 6.0 and 6.1 us; 8,100 tokens 64, 49 and
// 45 us (32/8 heads, d = 128).
int append_tokens_per_wg(int64_t tokens) { return tokens >= 1024 ? kAppendMaxPerWg : tokens >= 256 ? 4 : 1; }

cas_status_t run_append(const cas_decode_problem_t *p, const cas_rope_t *rope, const cas_append_t *t, void *k_pages,
                        void *v_pages, hipStream_t stream) {
  if (!t) return set_error(CAS_ERR_INVALID_ARGUMENT, "append tensors are NULL");
  const int D = p->head_dim, Hkv = p->num_kv_heads, Hq = Hkv * p->group_size;
  const int64_t Tq = p->q_offsets[p->batch];
  cas_status_t s;
  if (rope && (s = check_rope(rope, D)) != CAS_OK) return s;
  if (!rope && t->q) return set_error(CAS_ERR_INVALID_ARGUMENT, "q without a rope");
  if (Tq == 0) return CAS_OK;
  if (!t->k || !t->v || !k_pages || !v_pages) return set_error(CAS_ERR_INVALID_ARGUMENT, "k, v, k_pages and v_pages must be non-NULL");
  if (t->q && !t->q_out) return set_error(CAS_ERR_INVALID_ARGUMENT, "q without q_out");
  if (!aligned16(t->k) || !aligned16(t->v) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(t->q) ||
      (t->q && !aligned16(t->q_out)))
    return set_error(CAS_ERR_ALIGNMENT, "tensors must be 16-byte aligned");
  if ((s = check_strides("k", t->k_stride_tok, t->k_stride_head, 2)) != CAS_OK) return s;
  if ((s = check_strides("v", t->v_stride_tok, t->v_stride_head, 2)) != CAS_OK) return s;
  if (t->q && (s = check_strides("q", t->q_stride_tok, t->q_stride_head, 2)) != CAS_OK) return s;
  auto span = [&](const void *x, int64_t heads, int64_t st, int64_t sh) {
    return (uintptr_t)x + (uintptr_t)((Tq - 1) * st + (heads - 1) * sh + D) * 2;
  };
  const uintptr_t pool = (uintptr_t)p->num_pages * p->page_size * Hkv * D * 2;
  std::vector<Interval> iv;
  iv.push_back({(uintptr_t)t->k, span(t->k, Hkv, t->k_stride_tok, t->k_stride_head), false, 0, "k"});
  iv.push_back({(uintptr_t)t->v, span(t->v, Hkv, t->v_stride_tok, t->v_stride_head), false, 0, "v"});
  iv.push_back({(uintptr_t)k_pages, (uintptr_t)k_pages + pool, true, 1, "k_pages"});
  iv.push_back({(uintptr_t)v_pages, (uintptr_t)v_pages + pool, true, 2, "v_pages"});
  if (t->q) {
    const bool in_place = t->q == t->q_out && (Hq == 1 || t->q_stride_head == D) && (Tq == 1 || t->q_stride_tok == (int64_t)Hq * D);
    if (!in_place) iv.push_back({(uintptr_t)t->q, span(t->q, Hq, t->q_stride_tok, t->q_stride_head), false, 0, "q"});
    iv.push_back({(uintptr_t)t->q_out, (uintptr_t)t->q_out + (uintptr_t)Tq * Hq * D * 2, true, 3, "q_out"});
  }
  if (rope) iv.push_back({(uintptr_t)rope->turns, (uintptr_t)rope->turns + (uintptr_t)rope->rotary_dim * 4, false, 0, "turns"});
  std::string msg;
  if (!overlap_free(iv, msg)) return set_error(CAS_ERR_INVALID_ARGUMENT, msg);
  for (int b = 0; b < p->batch && t->starts; ++b) {
    const int64_t n = p->q_offsets[b + 1] - p->q_offsets[b];
    if ((int64_t)t->starts[b] + n > INT32_MAX) return set_error(CAS_ERR_INVALID_ARGUMENT, "request " + str(b) + ": position above 2^31");
  }
  AppendParams a;
  a.rope = rope ? dev_rope(rope, false) : DevRope{};
  a.k = t->k;
  a.v = t->v;
  a.q = t->q;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.q_out = t->q_out;
  a.k_tok = t->k_stride_tok;
  a.k_head = t->k_stride_head;
  a.v_tok = t->v_stride_tok;
  a.v_head = t->v_stride_head;
  a.q_tok = t->q_stride_tok;
  a.q_head = t->q_stride_head;
  a.Hkv = Hkv;
  a.g = p->group_size;
  const int ps = a.page_shift = __builtin_ctz((unsigned)p->page_size);
  const int rows = 256 / (D / 16), per_wg = append_tokens_per_wg(Tq);
  a.slots = rows / per_wg;
  const int head_groups = (int)std::min<int64_t>(64, ceil_div(t->q ? Hq : Hkv, 4 * a.slots));
  // Launches of as many requests (the last one perhaps in part) as the words hold.
  constexpr int kReq = sizeof(DevAppendRequest) / 4;
  std::vector<DevAppendRequest> reqs;
  std::vector<uint16_t> map;
  std::vector<int32_t> ids;
  auto flush = [&]() -> hipError_t {
    if (reqs.empty()) return hipSuccess;
    a.map0 = (int32_t)reqs.size() * kReq;
    a.page0 = a.map0 + (int32_t)(map.size() + 1) / 2;
    std::memcpy(a.words, reqs.data(), reqs.size() * sizeof(DevAppendRequest));
    std::memcpy(a.words + a.map0, map.data(), map.size() * sizeof(uint16_t));
    std::memcpy(a.words + a.page0, ids.data(), ids.size() * sizeof(int32_t));
    const int units = (int)map.size();
    reqs.clear();
    map.clear();
    ids.clear();
    return timed_launch("append", stream, [&] { return launch_append(a, D, units, head_groups, stream); });
  };
  for (int b = 0; b < p->batch; ++b) {
    const int32_t n_all = p->q_offsets[b + 1] - p->q_offsets[b], first = p->kv_lens[b] - n_all;
    for (int32_t off = 0; off < n_all;) {
      // Words left behind a further request's own, and how many of its tokens they hold: half a word for every
      // workgroup and one for every page, of which there is one more than the tokens fill.
      const int64_t left = kAppendWords - (int64_t)(reqs.size() + 1) * kReq - (int64_t)(map.size() + 2) / 2 - (int64_t)ids.size();
      const int64_t n_fit = (left - 3) * 2 * per_wg * p->page_size / (p->page_size + 2 * per_wg);
      if (left < 8 || n_fit < std::min<int64_t>(n_all - off, 2 * per_wg)) {
        const hipError_t e = flush();
        if (e != hipSuccess) return set_hip_error("append launch", e);
        continue;
      }
      const int32_t n = (int32_t)std::min<int64_t>(n_all - off, n_fit / per_wg * per_wg > 0 ? n_fit / per_wg * per_wg : n_fit);
      const int32_t key = first + off, row0 = key & (p->page_size - 1), pages = ((row0 + n - 1) >> ps) + 1;
      const int32_t start = t->starts ? t->starts[b] : first;
      reqs.push_back({(int32_t)map.size(), p->q_offsets[b] + off, n, row0, (int32_t)ids.size(), start + off});
      map.insert(map.end(), (size_t)ceil_div(n, per_wg), (uint16_t)(reqs.size() - 1));
      const int32_t *pg = p->page_ids + p->page_offsets[b] + (key >> ps);
      ids.insert(ids.end(), pg, pg + pages);
      off += n;
    }
  }
  const hipError_t e = flush();
  return e == hipSuccess ? CAS_OK : set_hip_error("append launch", e);
}

// ---------------------------------------------------------------------------
// Chunk attention over the paged cache
// ---------------------------------------------------------------------------
constexpr int kChunkRows = 256;     // packed rows of a workgroup
constexpr int kChunkTile = 64;

// Consecutive requests of one new token each whose shared pages the decode kernels
// stream once for all of them.
struct DecodePart {
  std::unique_ptr<cas_decode_plan_t, cas_status_t (*)(cas_decode_plan_t *)> plan{nullptr, cas_paged_decode_plan_destroy};
  int32_t tok0 = 0, tokens = 0;
  size_t off = 0, bytes = 0;   // in the workspace
};

struct ChunkPlan {
  std::vector<DecodePart> decode;
  std::vector<DevChunkItem> items;   // the first ones of the workgroups, in dispatch order, then the others
  int32_t wgs = 0;
  std::vector<uint32_t> granules;
  std::vector<DevChunkMerge> merges;   // the blocks of few rows first
  int32_t parts = 0, max_parts = 1, few = 0, part_rows = 0;
  std::vector<ChunkDirectRequest> direct;   // not empty: the plan goes as kernel arguments
  int64_t tiles = 0;
  size_t off_merges = 0, off_granules = 0, table_bytes = 0, off_plse = 0, off_po = 0, bytes = 0;
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Costs, in 64-key tiles of 256 rows with d = 128 (1.75 us). Fewer rows cost
// more than their share (a phase waits for its copies and barriers): measured 1.20 us
// for 96 and 1.25 for 128, with d = 64 0.87, 0.89 and 1.22 for 256; the lines through
// them here give 1.28, 1.37, 0.93, 1.00 and 1.26. Up to kChunkNarrowRows of
// them the kernel's waves divide the keys: 0.47 us for 32 rows and 0.92 for 64
// (d = 64: 0.26 and 0.52) where the keys are in the L2, as those of a request with
// several blocks are, `shared`; else most come from HBM and are priced at what that
// takes where every unit asks for some, 0.79 us for 32 rows and 1.05 for 64 (0.44 and
// 0.58): with 0.47 a batch of 16 single tokens beside a chunk took 106 us, with 0.79
// 93. kWgCost: what a workgroup costs beside its tiles (dispatch,
// first loads, pipeline fill and drain, epilogue), kItemCost: a further item of a
// workgroup; kMergeCost: a merge's launch; the partials' bytes, written and read, at
// kBytesPerTile. (Over 30 mixes, each of them 20-50 % higher or lower changes the
// time by 1 %.)
double tile_cost(int D, int rows, bool shared) {
  if (rows <= kChunkNarrowRows) {
    if (shared) return D == 128 ? (rows <= 32 ? 0.27 : 0.53) : rows <= 32 ? 0.15 : 0.30;
    return D == 128 ? (rows <= 32 ? 0.45 : 0.60) : rows <= 32 ? 0.25 : 0.33;
  }
  return D == 128 ? 0.57 + 0.43 * rows / 256 : 0.42 + 0.30 * rows / 256;
}
constexpr double kWgCost = 5.0, kItemCost = 3.0, kMergeCost = 3.0, kBytesPerTile = 5e6;
constexpr double kWorthIt = 0.97;   // of the cost without cuts: below it, blocks are cut
int min_piece(int rows) { return rows <= kChunkNarrowRows ? 4 : 2; }   // tiles (narrow: a piece for every wave)
constexpr int kManyRounds = 8;

struct ChunkBlock {
  int32_t b, row0, rows, tiles, kvh;
  double cost;   // of a tile
};
struct ChunkPiece {
  int32_t block, t0, t1;
};

// Cuts the blocks for n_bins workgroups that all cost about the same: whole
// blocks, longest first, to the workgroup with the least so far while they fit,
// then the other blocks in pieces into what is left. Returns the largest cost.
double fill_bins(const std::vector<ChunkBlock> &blocks, int n_bins, std::vector<std::vector<ChunkPiece>> &bins) {
  bins.assign(n_bins, {});
  std::vector<double> load(n_bins, kWgCost - kItemCost);
  std::vector<int32_t> order(blocks.size());
  double sum = 0.0;
  for (size_t i = 0; i < blocks.size(); ++i) {
    order[i] = (int32_t)i;
    sum += blocks[i].tiles * blocks[i].cost;
  }
  auto whole = [&](int32_t i) { return blocks[i].tiles * blocks[i].cost + kItemCost; };
  std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return whole(x) > whole(y); });
  // An equal share of all blocks, and a piece beside whole ones; at least a piece.
  double target = kWgCost + (sum + kItemCost * (double)blocks.size()) / n_bins;
  for (const ChunkBlock &x : blocks) target = std::max(target, kWgCost + std::min<int>(min_piece(x.rows), x.tiles) * x.cost);
  std::vector<int32_t> left;
  auto later = [&](int x, int y) { return load[x] != load[y] ? load[x] > load[y] : x > y; };
  std::vector<int> heap(n_bins);
  for (int i = 0; i < n_bins; ++i) heap[i] = i;
  std::make_heap(heap.begin(), heap.end(), later);
  for (int32_t i : order) {
    const int x = heap.front();
    if (load[x] + whole(i) > target) {
      left.push_back(i);
      continue;
    }
    std::pop_heap(heap.begin(), heap.end(), later);
    bins[x].push_back({i, 0, blocks[i].tiles});
    load[x] += whole(i);
    std::push_heap(heap.begin(), heap.end(), later);
  }
  std::vector<int> by_room(n_bins);
  for (int i = 0; i < n_bins; ++i) by_room[i] = i;
  std::stable_sort(by_room.begin(), by_room.end(), [&](int x, int y) { return load[x] < load[y]; });
  size_t k = 0;
  for (int32_t i : left) {
    for (int32_t t = 0; t < blocks[i].tiles;) {
      const int32_t rest = blocks[i].tiles - t;
      int32_t take = rest;
      if (k < by_room.size()) {
        take = (int32_t)std::max(0.0, std::min((double)rest, (target - load[by_room[k]] - kItemCost) / blocks[i].cost + 0.5));
        if (take < std::min(min_piece(blocks[i].rows), rest)) {
          ++k;
          continue;
        }
        if (rest - take < min_piece(blocks[i].rows)) take = rest;
      }
      const int x = k < by_room.size() ? by_room[k] : (int)(std::min_element(load.begin(), load.end()) - load.begin());
      bins[x].push_back({i, t, t + take});
      load[x] += kItemCost + take * blocks[i].cost;
      t += take;
      if (t < blocks[i].tiles) ++k;   // (the workgroup is full)
    }
  }
  return *std::max_element(load.begin(), load.end());
}

// Whether the requests b0 .. b1 - 1 (of one or no new token each) are better off
// with the decode kernels, which stream a run of pages once for all requests that
// read it: 32 requests over 8 of 16 cartridges of 1,024 tokens take 51 us there
// and 88 us here, over 4 of 256 (nothing shared) 100 us on either side; 30 requests
// over 4 of 64 beside two chunks 159 and 136 us, 30 over 8 of 16 194 and 229. In
// us, with launches and merge: 12 + 2.7 ns a 32-key tile that is streamed there; here
// 1.55 ns a 64-key tile and 1.75 ns a streamed one, for what comes from HBM, and 13,
// but not beside chunks, with which they fill the compute units. With d = 64: 14, 1.2,
// 0.8 and 0.75. (Of 12 batches of each size one is on the slower side, by 4 %.)
bool plan_decode_part(const cas_decode_problem_t *p, int b0, int b1, bool beside_chunks, std::vector<DecodePart> &out) {
  std::vector<int32_t> qo{0}, kv, po{0}, ids;
  int64_t tiles = 0;
  for (int b = b0; b < b1; ++b) {
    if (p->q_offsets[b + 1] == p->q_offsets[b]) continue;
    qo.push_back(qo.back() + 1);
    kv.push_back(p->kv_lens[b]);
    ids.insert(ids.end(), p->page_ids + p->page_offsets[b], p->page_ids + p->page_offsets[b + 1]);
    po.push_back((int32_t)ids.size());
    tiles += ceil_div(p->kv_lens[b], kChunkTile) * p->num_kv_heads;
  }
  if (kv.size() < 2) return false;
  cas_decode_problem_t sub = *p;
  sub.batch = (int32_t)kv.size();
  sub.q_offsets = qo.data();
  sub.kv_lens = kv.data();
  sub.page_offsets = po.data();
  sub.page_ids = ids.data();
  cas_decode_plan_t *plan = nullptr;
  DecodePart part;
  if (cas_paged_decode_plan_create(&sub, &plan, &part.bytes) != CAS_OK) return false;   // (too large for those kernels)
  part.plan.reset(plan);
  int64_t decode_tiles = 0;
  int32_t shared = 0;
  decode_plan_counts(plan, &decode_tiles, &shared);
  const bool d64 = p->head_dim == 64;
  const double there = d64 ? 14.0 + 1.2e-3 * (double)decode_tiles : 12.0 + 2.7e-3 * (double)decode_tiles;
  const double here = (beside_chunks ? 0.0 : 13.0) + (d64 ? 0.8e-3 : 1.55e-3) * (double)tiles +
                      (d64 ? 0.75e-3 : 1.75e-3) * (double)decode_tiles;
  if (shared == 0 || there > here) return false;
  part.tok0 = p->q_offsets[b0];
  part.tokens = sub.batch;
  out.push_back(std::move(part));
  return true;
}

// The launch plan. Either a workgroup per block, longest first, which the
// hardware hands out as compute units become free; or, where that leaves some
// idle, one workgroup per compute unit with an equal share, blocks cut along the
// key axis as that needs and merged afterwards. Blocks have 256 rows, fewer where
// the costs say so: one request of 64 tokens over 1,074 keys (d = 128, 8 KV heads of
// 4) takes 26.4 us in blocks of 256 rows, 22.2 of 128, 22.2 of 64 and 19.3 of 32, over
// 4,146 keys 43.4, 38.6, 32.6 and 25.5, 512 tokens over 1,536 keys 38.5, 40.8, 32.4 and
// 37.6. Over 64 problems the choice is 0.5 % slower than the best of the four, at most
// 7 %, and blocks of 256 alone 18 %, at most 71.
//
// Workgroup i goes to XCD i mod X, each with its own L2, so a KV head's workgroups
// stay on one XCD (or on X / Hkv of them) where the heads divide evenly.
cas_status_t build_chunk(const cas_decode_problem_t *p, ChunkPlan &pl) {
  cas_status_t s = check_paged(p);
  if (s != CAS_OK) return s;
  if (!std::isfinite(p->softmax_scale) || !(p->softmax_scale > 0.0f))
    return set_error(CAS_ERR_INVALID_ARGUMENT, "softmax_scale must be finite and > 0");
  const int64_t granule = (int64_t)16 * p->num_kv_heads * p->head_dim * 2 / 2048;   // in 2 KiB
  if (p->num_pages > (int64_t)UINT32_MAX / (granule * (p->page_size / 16))) return set_error(CAS_ERR_UNSUPPORTED, "page pool above 8 TiB");
  const int B = p->batch, g = p->group_size, Hkv = p->num_kv_heads, D = p->head_dim;
  std::vector<uint8_t> elsewhere(B, 0);   // requests that the decode kernels take
  bool chunks = false;
  for (int b = 0; b < B; ++b) chunks |= p->q_offsets[b + 1] - p->q_offsets[b] > 1;
  for (int b = 0; b < B && g <= 2 * kDecRows;) {
    int e = b;
    while (e < B && p->q_offsets[e + 1] - p->q_offsets[e] <= 1) ++e;
    if (e > b && plan_decode_part(p, b, e, chunks, pl.decode)) std::fill(elsewhere.begin() + b, elsewhere.begin() + e, 1);
    b = std::max(e, b + 1);
  }
  const Topology topo = device_topology();
  const int X = std::max(1, topo.xcds), cus = std::max(X, topo.cus);
  // KV heads kvh with kvh mod groups == i share the XCDs x with x mod groups == i.
  const int groups = Hkv % X == 0 ? X : X % Hkv == 0 ? Hkv : 1;
  const int bins = cus / groups, heads = Hkv / groups;   // of a group
  // In blocks of `rows` rows: those of the first group's heads, the group's
  // workgroups in order, and what they cost.
  struct Split {
    std::vector<ChunkBlock> blocks;
    std::vector<std::vector<ChunkPiece>> wgs;
    double cost;
    bool whole = true;   // no block is cut
  };
  auto split = [&](int rows) {
    Split x;
    std::vector<ChunkBlock> &blocks = x.blocks;
    double sum = 0.0;
    for (int h = 0; h < heads; ++h)
      for (int b = 0; b < B; ++b) {
        const int64_t n = p->q_offsets[b + 1] - p->q_offsets[b], nrows = n * g, before = p->kv_lens[b] - n;
        for (int64_t r = 0; r < nrows && !elsewhere[b]; r += rows) {
          const int64_t r1 = std::min<int64_t>(nrows, r + rows);
          const int32_t nt = (int32_t)((before + (r1 - 1) / g) / kChunkTile + 1);   // up to its last query's own key
          blocks.push_back({b, (int32_t)r, (int32_t)(r1 - r), nt, h * groups, tile_cost(D, (int)(r1 - r), nrows > rows)});
          sum += blocks.back().tiles * blocks.back().cost + kWgCost;
        }
      }
    // First a block each.
    std::stable_sort(blocks.begin(), blocks.end(), [](const ChunkBlock &x, const ChunkBlock &y) { return x.tiles * x.cost > y.tiles * y.cost; });
    auto whole = [&](size_t i) { return blocks[i].tiles * blocks[i].cost + kWgCost; };
    x.cost = sum / bins;
    // (Of the k * bins + 1 longest blocks, one unit gets k + 1.)
    for (size_t k = 0; k < 4 && k * bins < blocks.size(); ++k) {
      double c = 0.0;
      for (size_t i = k * bins - k; i <= k * bins; ++i) c += whole(i);
      x.cost = std::max(x.cost, c);
    }
    for (size_t i = 0; i < blocks.size(); ++i) x.wgs.push_back({{(int32_t)i, 0, blocks[i].tiles}});
    // Units differ in speed by a few per cent, which evens out where each gets
    // several blocks from the hardware: with kManyRounds of them nothing is cut.
    if (!blocks.empty() && blocks.size() < (size_t)(kManyRounds * bins)) {
      std::vector<std::vector<ChunkPiece>> equal;
      double even = fill_bins(blocks, bins, equal) + kMergeCost;
      std::vector<int32_t> n_pieces(blocks.size(), 0);
      for (const auto &w : equal)
        for (const ChunkPiece &y : w) ++n_pieces[y.block];
      double bytes = 0.0;
      for (size_t i = 0; i < blocks.size(); ++i)
        if (n_pieces[i] > 1) bytes += (double)n_pieces[i] * blocks[i].rows * D * 4;
      even += bytes * groups / kBytesPerTile;
      if (even < kWorthIt * x.cost) {
        x.wgs.swap(equal);
        x.cost = even;
        x.whole = false;
      }
    }
    return x;
  };
  Split best = split(kChunkRows);
  pl.part_rows = kChunkRows;
  // Smaller blocks cost more a row and are done sooner; not where every unit has one.
  for (int rows = kChunkRows / 2; rows >= kChunkFewRows && best.blocks.size() < (size_t)bins; rows /= 2) {
    Split x = split(rows);
    if (x.cost < best.cost) {
      best = std::move(x);
      pl.part_rows = rows;
    }
  }
  auto &blocks = best.blocks;
  auto &wgs = best.wgs;
  // Few whole blocks, one for a unit (so that their order is no matter), need no
  // tables in the workspace, whose upload is a launch of its own: a request of 33
  // tokens over 1,107 keys takes 19.7 us with them and 16.4 without.
  size_t words = 0;
  for (int b = 0; b < B; ++b)
    if (p->q_offsets[b + 1] > p->q_offsets[b] && !elsewhere[b])
      words += sizeof(ChunkDirectRequest) / 4 + (((size_t)(p->page_offsets[b + 1] - p->page_offsets[b]) * (p->page_size / 16) + 3) & ~(size_t)3);
  const bool direct = best.whole && !blocks.empty() && blocks.size() <= (size_t)bins && words <= (size_t)kChunkDirectWords;
  if (direct) {
    std::sort(blocks.begin(), blocks.end(), [](const ChunkBlock &x, const ChunkBlock &y) {
      return std::make_tuple(x.b, x.row0, x.kvh) < std::make_tuple(y.b, y.row0, y.kvh);
    });
    for (size_t i = 0; i < blocks.size(); ++i) wgs[i] = {{(int32_t)i, 0, blocks[i].tiles}};
  }
  if ((int64_t)blocks.size() * groups > INT32_MAX / 256) return set_error(CAS_ERR_UNSUPPORTED, "too many workgroups");
  wgs.erase(std::remove_if(wgs.begin(), wgs.end(), [](const std::vector<ChunkPiece> &w) { return w.empty(); }), wgs.end());
  // Partials: a block's lie together, in the order of its keys.
  std::vector<std::vector<int32_t>> cut(blocks.size());
  for (const auto &w : wgs)
    for (const ChunkPiece &x : w) cut[x.block].push_back(x.t0);
  std::vector<int32_t> part0(blocks.size(), -1);
  int32_t parts = 0;   // of a group
  for (size_t i = 0; i < blocks.size(); ++i) {
    std::sort(cut[i].begin(), cut[i].end());
    pl.max_parts = std::max(pl.max_parts, (int32_t)cut[i].size());
    if (cut[i].size() < 2) continue;
    part0[i] = parts;
    parts += (int32_t)cut[i].size();
  }
  if ((int64_t)parts * groups > INT32_MAX / kChunkRows) return set_error(CAS_ERR_UNSUPPORTED, "too many partials");
  pl.parts = parts * groups;
  for (int few = 1; few >= 0; --few) {
    for (int gr = 0; gr < groups; ++gr)
      for (size_t i = 0; i < blocks.size(); ++i) {
        const ChunkBlock &x = blocks[i];
        if (part0[i] < 0 || (x.rows <= kChunkFewRows) != (few == 1)) continue;
        pl.merges.push_back({p->q_offsets[x.b], x.row0, x.row0 + x.rows, x.kvh + gr, gr * parts + part0[i], (int32_t)cut[i].size()});
      }
    if (few) pl.few = (int32_t)pl.merges.size();
  }
  // The granules of the requests, whole tiles of them.
  std::vector<int32_t> granule0(B, 0);
  const int per_page = p->page_size / 16;
  for (int b = 0; b < B; ++b) {
    if (p->q_offsets[b + 1] == p->q_offsets[b] || elsewhere[b]) continue;
    if (pl.granules.size() > (size_t)INT32_MAX / 2) return set_error(CAS_ERR_UNSUPPORTED, "too many pages");
    granule0[b] = (int32_t)pl.granules.size();
    for (int32_t e = p->page_offsets[b]; e < p->page_offsets[b + 1]; ++e)
      for (int j = 0; j < per_page; ++j) pl.granules.push_back((uint32_t)(((int64_t)p->page_ids[e] * per_page + j) * granule));
    pl.granules.resize((pl.granules.size() + 3) & ~(size_t)3, 0);
  }
  // Groups in turn, so that workgroup i belongs to group i mod groups.
  auto item = [&](const ChunkPiece &y, int gr) {
    const ChunkBlock &x = blocks[y.block];
    const int32_t tok0 = p->q_offsets[x.b], len = p->q_offsets[x.b + 1] - tok0;
    const auto &c = cut[y.block];
    const int32_t part = part0[y.block] < 0 ? -1 : gr * parts + part0[y.block] + (int32_t)(std::lower_bound(c.begin(), c.end(), y.t0) - c.begin());
    pl.tiles += y.t1 - y.t0;
    return DevChunkItem{tok0, len, p->kv_lens[x.b], granule0[x.b], x.row0, x.kvh + gr, y.t0, y.t1, part, -1, x.row0 + x.rows};
  };
  pl.wgs = (int32_t)wgs.size() * groups;
  for (const auto &w : wgs)
    for (int gr = 0; gr < groups; ++gr) pl.items.push_back(item(w[0], gr));
  for (size_t i = 0; i < wgs.size(); ++i)
    for (int gr = 0; gr < groups; ++gr) {
      size_t last = i * groups + gr;
      for (size_t k = 1; k < wgs[i].size(); ++k) {
        pl.items[last].next = (int32_t)pl.items.size();
        last = pl.items.size();
        pl.items.push_back(item(wgs[i][k], gr));
      }
    }
  int32_t block0 = 0;
  for (int b = 0; b < B && direct; ++b) {
    const int32_t tok0 = p->q_offsets[b], len = p->q_offsets[b + 1] - tok0;
    if (!len || elsewhere[b]) continue;
    pl.direct.push_back({block0, tok0, len, p->kv_lens[b], granule0[b]});
    block0 += (int32_t)ceil_div((int64_t)len * g, pl.part_rows);
  }
  if (!direct) {
    pl.off_merges = align256(pl.items.size() * sizeof(DevChunkItem));
    pl.off_granules = align256(pl.off_merges + pl.merges.size() * sizeof(DevChunkMerge));
    pl.table_bytes = align256(pl.off_granules + pl.granules.size() * sizeof(uint32_t));
  }
  pl.off_plse = pl.table_bytes;
  pl.off_po = align256(pl.off_plse + (size_t)pl.parts * pl.part_rows * 4);
  pl.bytes = align256(pl.off_po + (size_t)pl.parts * pl.part_rows * p->head_dim * 4);
  for (DecodePart &d : pl.decode) {
    d.off = pl.bytes;
    pl.bytes = align256(pl.bytes + d.bytes);
  }
  return CAS_OK;
}

// Pinned slots for launch tables on their way to a workspace. A slot is free once
// the kernel that read it has set its flags.
struct TableSlots {
  static constexpr int kSlots = 16, kFlags = 16;
  static constexpr size_t kFlagBytes = kSlots * kFlags * sizeof(uint32_t);
  char *host = nullptr;              // kSlots slots, then their flags
  size_t slot_bytes = 0;
  uint32_t want[kSlots] = {};        // value of the slot's flags when it is free
  int used[kSlots] = {};             // flags of the slot's last upload
  bool taken[kSlots] = {};           // a thread is filling it
  int next = 0;
  uint32_t *flags(int i) const { return (uint32_t *)(host + kSlots * slot_bytes) + i * kFlags; }
  bool free(int i) const {
    if (taken[i]) return false;
    for (int f = 0; f < used[i]; ++f)
      if (__atomic_load_n(flags(i) + f, __ATOMIC_ACQUIRE) != want[i]) return false;
    return true;
  }
};

// The slots of a device, of its largest tables so far; those of smaller tables
// stay (less memory together than the current ones), since kernels may not have
// read them yet and freeing pinned memory waits for them.
struct TableRing {
  std::mutex mu;
  std::vector<std::unique_ptr<TableSlots>> slots;
};

TableRing &table_ring(int dev) {
  static std::mutex mu;
  static std::map<int, TableRing> rings;
  std::lock_guard<std::mutex> lk(mu);
  return rings[dev];
}

// A free slot of at least `bytes`, taken for the caller, or -1.
cas_status_t take_slot(TableRing &r, size_t bytes, TableSlots *&s, int &slot) {
  std::lock_guard<std::mutex> lk(r.mu);
  slot = -1;
  if (r.slots.empty() || bytes > r.slots.back()->slot_bytes) {
    auto fresh = std::make_unique<TableSlots>();
    fresh->slot_bytes = r.slots.empty() ? 64 << 10 : 2 * r.slots.back()->slot_bytes;
    while (fresh->slot_bytes < bytes) fresh->slot_bytes *= 2;
    r.slots.reserve(r.slots.size() + 1);
    // Coherent: the kernel reads slots that the host has just rewritten, and the
    // host the flags that it writes.
    const size_t all = fresh->slot_bytes * TableSlots::kSlots;
    const hipError_t e = hipHostMalloc((void **)&fresh->host, all + TableSlots::kFlagBytes, hipHostMallocCoherent);
    if (e != hipSuccess) return set_hip_error("hipHostMalloc", e);
    std::memset(fresh->host + all, 0, TableSlots::kFlagBytes);
    r.slots.push_back(std::move(fresh));
  }
  s = r.slots.back().get();
  for (int k = 0; k < TableSlots::kSlots && slot < 0; ++k) {
    const int i = (s->next + k) % TableSlots::kSlots;
    if (s->free(i)) slot = i;
  }
  if (slot >= 0) {
    s->taken[slot] = true;
    s->next = (slot + 1) % TableSlots::kSlots;
  }
  return CAS_OK;
}

// Tables as kernel arguments, 3.9 KiB to a launch.
template <typename Fill>
cas_status_t upload_as_arguments(size_t bytes, void *ws, hipStream_t stream, Fill &&fill) {
  std::vector<char> h((bytes + 15) & ~(size_t)15, 0);
  fill(h.data());
  const hipError_t e = launch_table_args_upload(h.data(), h.size(), ws, stream);
  return e == hipSuccess ? CAS_OK : set_hip_error("table upload launch", e);
}

// Copies launch tables through a pinned slot. With all slots on their way the host
// is 16 tables ahead of the GPU and waits for the first of them, without the lock,
// but no longer than until its call's deadline, kSlotWait: what they wait for may be work that this thread, or
// one that waits with it, has yet to enqueue, and after a device error they never
// end. Then the tables go as kernel arguments, whose launches (28 us more for 57 KB,
// 12 us for 14 KB) are little beside a GPU that took that long for a call.
constexpr std::chrono::microseconds kSlotWait{10000}, kSlotSpin{100}, kSlotSleep{50};

using Clock = std::chrono::steady_clock;

template <typename Fill>
cas_status_t upload_tables(size_t bytes, void *ws, hipStream_t stream, Clock::time_point deadline, Fill &&fill) {
  int dev = 0, slot = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return set_hip_error("hipGetDevice", e);
  TableRing &r = table_ring(dev);
  TableSlots *s = nullptr;
  cas_status_t st = take_slot(r, bytes, s, slot);
  for (const auto t0 = Clock::now(); st == CAS_OK && slot < 0; st = take_slot(r, bytes, s, slot)) {
    const auto now = Clock::now();
    if (now >= deadline) return upload_as_arguments(bytes, ws, stream, fill);
    if (now - t0 < kSlotSpin) std::this_thread::yield();
    else std::this_thread::sleep_for(kSlotSleep);
  }
  if (st != CAS_OK) return st;
  char *h = s->host + (size_t)slot * s->slot_bytes;
  fill(h);
  const int n = (int)std::min<size_t>(TableSlots::kFlags, (bytes + 4095) / 4096);
  const uint32_t value = s->want[slot] + 1;
  e = launch_table_flags(ws, h, bytes, s->flags(slot), n, value, stream);
  std::lock_guard<std::mutex> lk(r.mu);
  s->taken[slot] = false;
  if (e != hipSuccess) return set_hip_error("table upload launch", e);
  s->want[slot] = value;
  s->used[slot] = n;
  return CAS_OK;
}

cas_status_t run_chunk(const cas_decode_problem_t *p, const ChunkPlan &pl, const void *q, const void *k_pages, const void *v_pages,
                       void *o, float *lse, void *workspace, size_t ws_bytes, hipStream_t stream) {
  if (pl.items.empty() && pl.decode.empty()) return CAS_OK;
  if (!q || !k_pages || !v_pages || !o) return set_error(CAS_ERR_INVALID_ARGUMENT, "q, k_pages, v_pages and o must be non-NULL");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(o) || ((uintptr_t)lse & 3u))
    return set_error(CAS_ERR_ALIGNMENT, "tensors must be 16-byte aligned (lse 4-byte)");
  const uintptr_t rows = (uintptr_t)p->q_offsets[p->batch] * p->num_kv_heads * p->group_size, qbytes = rows * p->head_dim * 2;
  const uintptr_t pool = (uintptr_t)p->num_pages * p->page_size * p->num_kv_heads * p->head_dim * 2;
  cas_status_t s = check_workspace(workspace, ws_bytes, pl.bytes);
  if (s != CAS_OK) return s;
  std::vector<Interval> iv;
  iv.push_back({(uintptr_t)q, (uintptr_t)q + qbytes, false, 0, "q"});
  iv.push_back({(uintptr_t)k_pages, (uintptr_t)k_pages + pool, false, 0, "k_pages"});
  iv.push_back({(uintptr_t)v_pages, (uintptr_t)v_pages + pool, false, 0, "v_pages"});
  iv.push_back({(uintptr_t)o, (uintptr_t)o + qbytes, true, 1, "o"});
  iv.push_back({(uintptr_t)workspace, (uintptr_t)workspace + pl.bytes, true, 2, "workspace"});
  if (lse) iv.push_back({(uintptr_t)lse, (uintptr_t)lse + rows * 4, true, 3, "lse"});
  std::string msg;
  if (!overlap_free(iv, msg)) return set_error(CAS_ERR_INVALID_ARGUMENT, msg);
  char *ws = (char *)workspace;
  auto fill = [&](char *h) {
    std::memcpy(h, pl.items.data(), pl.items.size() * sizeof(DevChunkItem));
    if (!pl.merges.empty()) std::memcpy(h + pl.off_merges, pl.merges.data(), pl.merges.size() * sizeof(DevChunkMerge));
    std::memcpy(h + pl.off_granules, pl.granules.data(), pl.granules.size() * sizeof(uint32_t));
  };
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (stream && hipStreamIsCapturing(stream, &capture) != hipSuccess) (void)hipGetLastError();
  const bool capturing = capture == hipStreamCaptureStatusActive;
  const Clock::time_point deadline = Clock::now() + kSlotWait;
  const TableUpload upload = [&](size_t bytes, void *dst, hipStream_t st, const std::function<void(char *)> &write) {
    // A graph keeps kernel arguments, but not what the pinned slots hold now.
    return capturing ? upload_as_arguments(bytes, dst, st, write) : upload_tables(bytes, dst, st, deadline, write);
  };
  const int64_t row = (int64_t)p->num_kv_heads * p->group_size * p->head_dim * 2, Tq = p->q_offsets[p->batch];
  for (const DecodePart &d : pl.decode) {
    s = decode_run_part(d.plan.get(), (const char *)q + d.tok0 * row, k_pages, v_pages, (char *)o + d.tok0 * row,
                        lse ? lse + d.tok0 : nullptr, (int)Tq, ws + d.off, d.bytes, upload, stream);
    if (s != CAS_OK) return s;
  }
  if (pl.items.empty()) return CAS_OK;
  const bool direct = !pl.direct.empty();
  if (!direct && (s = upload(pl.table_bytes, workspace, stream, fill)) != CAS_OK) return s;
  ChunkParams c{};
  c.q = q;
  c.k_pages = k_pages;
  c.v_pages = v_pages;
  c.o = o;
  c.lse = lse;
  c.items = (const DevChunkItem *)ws;
  c.merges = (const DevChunkMerge *)(ws + pl.off_merges);
  c.granules = (const uint32_t *)(ws + pl.off_granules);
  c.part_lse = (float *)(ws + pl.off_plse);
  c.part_o = (float *)(ws + pl.off_po);
  c.Hkv = p->num_kv_heads;
  c.g = p->group_size;
  c.Tq = p->q_offsets[p->batch];
  c.part_rows = pl.part_rows;
  c.scale_log2 = p->softmax_scale * 1.4426950408889634f;
  ChunkDirect d;
  if (direct) {
    d.n = (int32_t)pl.direct.size();
    d.rows = pl.part_rows;
    std::memcpy(d.words, pl.direct.data(), pl.direct.size() * sizeof(ChunkDirectRequest));
    std::memcpy(d.words + pl.direct.size() * (sizeof(ChunkDirectRequest) / 4), pl.granules.data(), pl.granules.size() * sizeof(uint32_t));
  }
  hipError_t e = timed_launch("chunk", stream, [&] { return launch_chunk_bf16(c, direct ? &d : nullptr, p->head_dim, pl.wgs, stream); });
  if (e != hipSuccess) return set_hip_error("chunk launch", e);
  if (!pl.merges.empty()) {
    e = timed_launch("chunk_merge", stream, [&] {
      return launch_chunk_merge_bf16(c, p->head_dim, pl.few, (int)pl.merges.size(), pl.max_parts, stream);
    });
    if (e != hipSuccess) return set_hip_error("chunk_merge launch", e);
  }
  return CAS_OK;
}

}  // namespace

struct cas_append_plan {
  OwnedProblem own;
};

struct cas_chunk_plan {
  OwnedProblem own;
  ChunkPlan plan;
};

extern "C" {

cas_status_t cas_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_len,
                                  double low, double high, double *turns) {
  if (!turns) return set_error(CAS_ERR_INVALID_ARGUMENT, "turns is NULL");
  if (rotary_dim < 16 || rotary_dim > 128 || rotary_dim % 16)
    return set_error(CAS_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in [16, 128]");
  if (!std::isfinite(base) || !(base > 0.0)) return set_error(CAS_ERR_INVALID_ARGUMENT, "base must be finite and > 0");
  if (scaling < CAS_ROPE_NONE || scaling > CAS_ROPE_BY_PARTS) return set_error(CAS_ERR_INVALID_ARGUMENT, "unknown scaling");
  if (scaling != CAS_ROPE_NONE && (!std::isfinite(factor) || !(factor > 0.0)))
    return set_error(CAS_ERR_INVALID_ARGUMENT, "factor must be finite and > 0");
  if (scaling == CAS_ROPE_BY_PARTS &&
      (!std::isfinite(original_len) || !(original_len > 0.0) || !std::isfinite(low) || !std::isfinite(high) || !(low < high)))
    return set_error(CAS_ERR_INVALID_ARGUMENT, "by parts: original_len must be > 0 and low < high");
  const double R = rotary_dim, two_pi = 6.283185307179586477;
  if (scaling == CAS_ROPE_NTK) base *= std::pow(factor, R / (R - 2.0));
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / R) / two_pi;   // turns per position
    if (scaling == CAS_ROPE_LINEAR) f /= factor;
    if (scaling == CAS_ROPE_BY_PARTS) {
      const double w = std::min(1.0, std::max(0.0, (original_len * f - low) / (high - low)));
      f = (1.0 - w) * f / factor + w * f;
    }
    turns[i] = f;
  }
  return CAS_OK;
}

cas_status_t cas_rope(const cas_rope_t *rope, int32_t dtype, int32_t head_dim, int64_t tokens, const int32_t *positions,
                      const cas_rope_tensor_t *tensors, int32_t n, int32_t inverse, void *hip_stream) {
  return guarded([&] { return rope_call(rope, dtype, head_dim, tokens, positions, tensors, n, inverse, (hipStream_t)hip_stream); });
}

cas_status_t cas_paged_append(const cas_decode_problem_t *p, const cas_rope_t *rope, const cas_append_t *t, void *k_pages,
                              void *v_pages, void *hip_stream) {
  return guarded([&] {
    const cas_status_t s = check_append(p);
    return s == CAS_OK ? run_append(p, rope, t, k_pages, v_pages, (hipStream_t)hip_stream) : s;
  });
}

cas_status_t cas_paged_append_plan_create(const cas_decode_problem_t *p, cas_append_plan_t **plan) {
  if (!plan) return set_error(CAS_ERR_INVALID_ARGUMENT, "plan is NULL");
  *plan = nullptr;
  return guarded([&] {
    auto pl = std::make_unique<cas_append_plan>();
    const cas_status_t s = check_append(p);
    if (s != CAS_OK) return s;
    pl->own.assign(*p);
    *plan = pl.release();
    return CAS_OK;
  });
}

cas_status_t cas_paged_append_run(const cas_append_plan_t *plan, const cas_rope_t *rope, const cas_append_t *t, void *k_pages,
                                  void *v_pages, void *hip_stream) {
  if (!plan) return set_error(CAS_ERR_INVALID_ARGUMENT, "plan is NULL");
  return guarded([&] { return run_append(&plan->own.p, rope, t, k_pages, v_pages, (hipStream_t)hip_stream); });
}

int32_t cas_paged_append_plan_matches(const cas_append_plan_t *plan, const cas_decode_problem_t *p) {
  return plan && p && plan->own.matches(p);
}

cas_status_t cas_paged_append_plan_destroy(cas_append_plan_t *plan) {
  delete plan;
  return CAS_OK;
}

cas_status_t cas_paged_chunk_workspace_size(const cas_decode_problem_t *p, size_t *bytes) {
  if (!bytes) return set_error(CAS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  return guarded([&] {
    ChunkPlan pl;
    const cas_status_t s = build_chunk(p, pl);
    if (s == CAS_OK) *bytes = pl.bytes;
    return s;
  });
}

cas_status_t cas_paged_chunk_fwd(const cas_decode_problem_t *p, const void *q, const void *k_pages, const void *v_pages,
                                 void *o, float *lse, void *workspace, size_t ws_bytes, void *hip_stream) {
  return guarded([&] {
    ChunkPlan pl;
    const cas_status_t s = build_chunk(p, pl);
    return s == CAS_OK ? run_chunk(p, pl, q, k_pages, v_pages, o, lse, workspace, ws_bytes, (hipStream_t)hip_stream) : s;
  });
}

cas_status_t cas_paged_chunk_plan_create(const cas_decode_problem_t *p, cas_chunk_plan_t **plan, size_t *ws_bytes) {
  if (!plan || !ws_bytes) return set_error(CAS_ERR_INVALID_ARGUMENT, "plan or ws_bytes is NULL");
  *plan = nullptr;
  return guarded([&] {
    auto pl = std::make_unique<cas_chunk_plan>();
    const cas_status_t s = build_chunk(p, pl->plan);
    if (s != CAS_OK) return s;
    pl->own.assign(*p);
    *ws_bytes = pl->plan.bytes;
    *plan = pl.release();
    return CAS_OK;
  });
}

cas_status_t cas_paged_chunk_run(const cas_chunk_plan_t *plan, const void *q, const void *k_pages, const void *v_pages,
                                 void *o, float *lse, void *workspace, size_t ws_bytes, void *hip_stream) {
  if (!plan) return set_error(CAS_ERR_INVALID_ARGUMENT, "plan is NULL");
  return guarded([&] {
    return run_chunk(&plan->own.p, plan->plan, q, k_pages, v_pages, o, lse, workspace, ws_bytes, (hipStream_t)hip_stream);
  });
}

int32_t cas_paged_chunk_plan_matches(const cas_chunk_plan_t *plan, const cas_decode_problem_t *p) {
  return plan && p && plan->own.matches(p);
}

cas_status_t cas_paged_chunk_plan_destroy(cas_chunk_plan_t *plan) {
  delete plan;
  return CAS_OK;
}

cas_status_t cas_paged_chunk_plan_info(const cas_chunk_plan_t *plan, cas_chunk_plan_info_t *info, int32_t *items) {
  if (!plan || !info) return set_error(CAS_ERR_INVALID_ARGUMENT, "plan or info is NULL");
  const ChunkPlan &pl = plan->plan;
  *info = cas_chunk_plan_info_t{};
  info->workgroups = pl.wgs;
  info->items = (int32_t)pl.items.size();
  info->partials = pl.parts;
  info->max_partials = pl.max_parts;
  info->key_tiles = pl.tiles;
  info->decode_parts = (int32_t)pl.decode.size();
  for (const DecodePart &d : pl.decode) info->decode_tokens += d.tokens;
  info->ws_bytes = pl.bytes;
  static_assert(sizeof(DevChunkItem) == 44, "a table of 32-bit values");
  if (items && !pl.items.empty()) std::memcpy(items, pl.items.data(), pl.items.size() * sizeof(DevChunkItem));
  return CAS_OK;
}

}  // extern "C"
