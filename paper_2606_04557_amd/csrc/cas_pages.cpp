// Pages of the paged cache: the page table (which sequence has which pages; host
// only) and the host side of the copies between pages.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <exception>
#include <functional>
#include <memory>
#include <string>
#include <unordered_map>
#include <unordered_set>
#include <vector>

#include "../../include/cas.h"
#include "cas_host.h"
#include "cas_internal.h"

using namespace cas;

namespace {

constexpr int64_t kMaxKeys = (int64_t)1 << 30;   // of a sequence, as the paged calls have it

std::string str(int64_t x) { return std::to_string(x); }

// No exception leaves a C entry (host memory may run out).
template <typename F>
cas_status_t guarded(F &&f) {
  try {
    return f();
  } catch (const std::exception &e) {
    return set_error(CAS_ERR_UNSUPPORTED, std::string("host memory: ") + e.what());
  }
}

struct Sequence {
  int64_t len = 0;
  std::vector<int32_t> pages;   // ceil(len / page size)
};

}  // namespace

struct cas_page_table {
  int64_t num_pages;
  int32_t page;                 // tokens of a page
  std::vector<int64_t> refs;    // per page ever used, how often sequences' lists name it
  std::vector<int32_t> spare;   // free pages below refs.size(), a heap with the lowest on top
  std::unordered_map<int64_t, Sequence> seqs;
  int64_t next_id = 0;
  int64_t used = 0;

  int64_t free_pages() const { return num_pages - used; }
  Sequence *find(int64_t id) {
    const auto it = seqs.find(id);
    return it == seqs.end() ? nullptr : &it->second;
  }
  // A page with one reference.
  int32_t take() {
    int32_t id;
    if (!spare.empty()) {
      std::pop_heap(spare.begin(), spare.end(), std::greater<int32_t>());
      id = spare.back();
      spare.pop_back();
      refs[(size_t)id] = 1;
    } else {
      id = (int32_t)refs.size();
      refs.push_back(1);
    }
    ++used;
    return id;
  }
  void drop(int32_t id) {
    if (--refs[(size_t)id] == 0) {
      spare.push_back(id);
      std::push_heap(spare.begin(), spare.end(), std::greater<int32_t>());
      --used;
    }
  }
};

namespace {

// Memory for `more` pages that will be taken and for whatever will be dropped, so
// that neither can fail half-way.
void reserve_pages(cas_page_table &t, int64_t more) {
  const size_t need = t.refs.size() + (size_t)std::max<int64_t>(more - (int64_t)t.spare.size(), 0);
  if (need > t.refs.capacity()) t.refs.reserve(std::max(need, 2 * t.refs.capacity()));
  if (t.refs.capacity() > t.spare.capacity()) t.spare.reserve(t.refs.capacity());
}

cas_status_t unknown(int64_t id) { return set_error(CAS_ERR_INVALID_ARGUMENT, "no sequence " + str(id)); }

// The named sequences, all different.
cas_status_t look_up(cas_page_table &t, const int64_t *ids, int32_t n, std::vector<Sequence *> &out, bool distinct = true) {
  if (n < 0 || (n > 0 && !ids)) return set_error(CAS_ERR_INVALID_ARGUMENT, "n must be >= 0 and the sequences non-NULL");
  out.resize((size_t)n);
  std::unordered_set<int64_t> seen;
  for (int32_t i = 0; i < n; ++i) {
    if (!(out[(size_t)i] = t.find(ids[i]))) return unknown(ids[i]);
    if (distinct && n > 1 && !seen.insert(ids[i]).second)
      return set_error(CAS_ERR_INVALID_ARGUMENT, "sequence " + str(ids[i]) + " is named twice");
  }
  return CAS_OK;
}

int64_t pages_for(const cas_page_table &t, int64_t len) { return (len + t.page - 1) / t.page; }

cas_status_t add(cas_page_table &t, const int64_t *parts, int32_t n, int64_t *seq) {
  std::vector<Sequence *> from;
  cas_status_t s = look_up(t, parts, n, from, false);
  if (s != CAS_OK) return s;
  Sequence q;
  for (int32_t i = 0; i < n; ++i) {
    if (i + 1 < n && from[(size_t)i]->len % t.page)
      return set_error(CAS_ERR_INVALID_ARGUMENT, "sequence " + str(parts[i]) + " ends inside a page: only the last part may");
    q.len += from[(size_t)i]->len;
    if (q.len > kMaxKeys) return set_error(CAS_ERR_UNSUPPORTED, "more than 2^30 keys");
    // (A page twice in one sequence, as the same cartridge twice, counts twice.)
    q.pages.insert(q.pages.end(), from[(size_t)i]->pages.begin(), from[(size_t)i]->pages.end());
  }
  const int64_t id = t.next_id;
  Sequence &kept = t.seqs[id];
  kept = std::move(q);
  for (const int32_t p : kept.pages) ++t.refs[(size_t)p];
  t.next_id = id + 1;
  *seq = id;
  return CAS_OK;
}

cas_status_t extend(cas_page_table &t, const int64_t *ids, int32_t n, const int32_t *counts, cas_page_copy_t *copies,
                    int32_t *n_copies) {
  std::vector<Sequence *> q;
  cas_status_t s = look_up(t, ids, n, q);
  if (s != CAS_OK) return s;
  if (n > 0 && (!counts || !copies)) return set_error(CAS_ERR_INVALID_ARGUMENT, "counts and copies must be non-NULL");
  // What every sequence needs, in order: of those that share their last page, the last one to be extended keeps it.
  std::unordered_map<int32_t, int64_t> left;   // references of a shared last page that remain
  std::vector<uint8_t> copy((size_t)n, 0);
  int64_t need = 0;
  for (int32_t i = 0; i < n; ++i) {
    const Sequence &x = *q[(size_t)i];
    if (counts[i] < 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "counts must be >= 0");
    if (x.len + counts[i] > kMaxKeys) return set_error(CAS_ERR_UNSUPPORTED, "sequence " + str(ids[i]) + ": more than 2^30 keys");
    if (counts[i] == 0) continue;
    need += pages_for(t, x.len + counts[i]) - (int64_t)x.pages.size();
    if (x.len % t.page == 0) continue;
    const int32_t last = x.pages.back();
    int64_t &refs = left.emplace(last, t.refs[(size_t)last]).first->second;
    if (refs > 1) {
      --refs;
      copy[(size_t)i] = 1;
      ++need;
    }
  }
  if (need > t.free_pages())
    return set_error(CAS_ERR_PAGES, "needs " + str(need) + " free pages, has " + str(t.free_pages()));
  // From here on nothing allocates.
  for (int32_t i = 0; i < n; ++i)
    if (counts[i]) q[(size_t)i]->pages.reserve((size_t)pages_for(t, q[(size_t)i]->len + counts[i]));
  reserve_pages(t, need);
  int32_t done = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] == 0) continue;
    Sequence &x = *q[(size_t)i];
    if (copy[(size_t)i]) {
      const int32_t old = x.pages.back(), fresh = t.take();
      copies[done++] = {old, fresh, (int32_t)(x.len % t.page)};
      x.pages.back() = fresh;
      t.drop(old);
    }
    x.len += counts[i];
    while ((int64_t)x.pages.size() < pages_for(t, x.len)) x.pages.push_back(t.take());
  }
  *n_copies = done;
  return CAS_OK;
}

cas_status_t reorder(cas_page_table &t, const int64_t *ids, int32_t n, const int32_t *parents) {
  std::vector<Sequence *> q;
  cas_status_t s = look_up(t, ids, n, q);
  if (s != CAS_OK) return s;
  if (n > 0 && !parents) return set_error(CAS_ERR_INVALID_ARGUMENT, "parents is NULL");
  for (int32_t i = 0; i < n; ++i)
    if (parents[i] < 0 || parents[i] >= n) return set_error(CAS_ERR_INVALID_ARGUMENT, "parents must be in [0, n)");
  // Beams have long prefixes in common: only from where a parent's list and the own one part do references change.
  std::vector<Sequence> next((size_t)n);
  std::vector<size_t> same((size_t)n, 0);
  for (int32_t i = 0; i < n; ++i) {
    if (parents[i] == i) continue;
    const Sequence &from = *q[(size_t)parents[i]];
    next[(size_t)i] = from;
    const auto &a = q[(size_t)i]->pages, &b = from.pages;
    same[(size_t)i] = (size_t)(std::mismatch(a.begin(), a.begin() + (ptrdiff_t)std::min(a.size(), b.size()), b.begin()).first - a.begin());
  }
  reserve_pages(t, 0);
  for (int32_t i = 0; i < n; ++i)
    if (parents[i] != i)
      for (size_t j = same[(size_t)i]; j < next[(size_t)i].pages.size(); ++j) ++t.refs[(size_t)next[(size_t)i].pages[j]];
  for (int32_t i = 0; i < n; ++i) {
    if (parents[i] == i) continue;
    Sequence &x = *q[(size_t)i];
    for (size_t j = same[(size_t)i]; j < x.pages.size(); ++j) t.drop(x.pages[j]);
    x = std::move(next[(size_t)i]);
  }
  return CAS_OK;
}

cas_status_t compact(cas_page_table &t, int32_t most, cas_page_copy_t *copies, int32_t *n_copies) {
  if (most < 0 || (most > 0 && !copies)) return set_error(CAS_ERR_INVALID_ARGUMENT, "most must be >= 0 and copies non-NULL");
  // The highest pages in use against the lowest free ones.
  std::vector<int32_t> to((size_t)t.refs.size(), -1);
  std::vector<cas_page_copy_t> moves;
  int64_t lo = 0, hi = (int64_t)t.refs.size() - 1;
  while ((int64_t)moves.size() < most) {
    while (lo < hi && t.refs[(size_t)lo] > 0) ++lo;
    while (hi > lo && t.refs[(size_t)hi] == 0) --hi;
    if (lo >= hi) break;
    to[(size_t)hi] = (int32_t)lo;
    moves.push_back({(int32_t)hi--, (int32_t)lo++, 0});
  }
  // The rows that hold keys: a shared page has as many as the longest of its sequences put there.
  std::vector<int32_t> rows((size_t)t.refs.size(), 0);
  for (const auto &e : t.seqs) {
    const Sequence &x = e.second;
    for (size_t j = 0; j < x.pages.size(); ++j) {
      int32_t &r = rows[(size_t)x.pages[j]];
      r = std::max(r, (int32_t)std::min<int64_t>(t.page, x.len - (int64_t)j * t.page));
    }
  }
  // The free list anew: what is below the end and has no reference.
  std::vector<int64_t> refs = t.refs;
  for (const cas_page_copy_t &m : moves) std::swap(refs[(size_t)m.src], refs[(size_t)m.dst]);
  while (!refs.empty() && refs.back() == 0) refs.pop_back();
  std::vector<int32_t> spare;
  spare.reserve(refs.size());
  for (size_t i = 0; i < refs.size(); ++i)
    if (refs[i] == 0) spare.push_back((int32_t)i);
  // (Ascending ids are a heap.)
  // From here on nothing allocates.
  for (auto &e : t.seqs)
    for (int32_t &p : e.second.pages)
      if (to[(size_t)p] >= 0) p = to[(size_t)p];
  for (size_t i = 0; i < moves.size(); ++i) copies[i] = {moves[i].src, moves[i].dst, rows[(size_t)moves[i].src]};
  t.refs.swap(refs);
  t.spare.swap(spare);
  *n_copies = (int32_t)moves.size();
  return CAS_OK;
}

// ---------------------------------------------------------------------------
// Copies between pages
// ---------------------------------------------------------------------------
// Whether the pages of the list are in range, none is written twice, and none is
// both written and read.
cas_status_t check_copies(const cas_page_copy_t *c, int32_t n, int64_t num_pages, int32_t page_size) {
  // A small open-addressed set of the written pages.
  size_t slots = 16;
  while (slots < 2 * (size_t)n) slots *= 2;
  std::vector<int32_t> set(slots, -1);
  auto slot = [&](int32_t id) {
    size_t i = ((uint32_t)id * 2654435761u) & (slots - 1);
    while (set[i] >= 0 && set[i] != id) i = (i + 1) & (slots - 1);
    return i;
  };
  for (int32_t i = 0; i < n; ++i) {
    if (c[i].src < 0 || c[i].src >= num_pages || c[i].dst < 0 || c[i].dst >= num_pages)
      return set_error(CAS_ERR_INVALID_ARGUMENT, "copy " + str(i) + ": page out of range");
    if (c[i].rows < 0 || c[i].rows > page_size)
      return set_error(CAS_ERR_INVALID_ARGUMENT, "copy " + str(i) + ": rows must be in [0, page_size]");
    const size_t at = slot(c[i].dst);
    if (set[at] >= 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "page " + str(c[i].dst) + " is written twice");
    set[at] = c[i].dst;
  }
  for (int32_t i = 0; i < n; ++i)
    if (set[slot(c[i].src)] >= 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "page " + str(c[i].src) + " is read and written");
  return CAS_OK;
}

constexpr int32_t kTableCopies = 1 << 16;   // of a list at a time (786 KB)

size_t table_bytes(int32_t n) {
  return n <= kPageCopyArgs ? 0 : ((size_t)std::min(n, kTableCopies) * sizeof(cas_page_copy_t) + 15) / 16 * 16;
}

// Bytes of a workgroup's piece. Whole pages go fastest with one 16-byte load to a
// thread (8,192 of 32 KB in two pools: 172 us; with two 187, four 194). Where copies are of
// few rows, most pieces of the longest one's count are empty, and starting their
// waves takes longer than the bytes of the others: 200 tails in 64 pools take 104 us
// with pieces of 8 KiB, 88 with 16 and 82 with 32 (a workgroup of 1,024 threads); 37
// tails of 48 KB in 10 pools 4.8, 4.3 and 5.8.
int32_t piece_bytes(int64_t all_rows, int32_t most_rows, int32_t n, int64_t row_bytes, int32_t n_pools) {
  if (all_rows * 4 >= (int64_t)most_rows * n * 3) return kPagePiece;
  return all_rows * row_bytes * n_pools < ((int64_t)64 << 20) ? 2 * kPagePiece : 4 * kPagePiece;
}

cas_status_t copy_pages(void *const *pools, int32_t n_pools, int64_t num_pages, int32_t page_size, int64_t row_bytes,
                        const cas_page_copy_t *c, int32_t n, void *workspace, size_t ws_bytes, hipStream_t stream) {
  if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
    return set_error(CAS_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  if (num_pages < 1 || num_pages > INT32_MAX) return set_error(CAS_ERR_INVALID_ARGUMENT, "num_pages must be in [1, 2^31)");
  if (row_bytes < 16) return set_error(CAS_ERR_INVALID_ARGUMENT, "row_bytes must be >= 16");
  if (row_bytes % 16) return set_error(CAS_ERR_ALIGNMENT, "row_bytes must be a multiple of 16");
  if (row_bytes > (1 << 24)) return set_error(CAS_ERR_UNSUPPORTED, "page larger than 2 GiB");
  if (n_pools < 0 || n_pools > (1 << 16) || (n_pools > 0 && !pools))
    return set_error(CAS_ERR_INVALID_ARGUMENT, "n_pools must be in [0, 2^16] and pools non-NULL");
  if (n < 0 || (n > 0 && !c)) return set_error(CAS_ERR_INVALID_ARGUMENT, "n must be >= 0 and copies non-NULL");
  cas_status_t s = check_copies(c, n, num_pages, page_size);
  if (s != CAS_OK) return s;
  int32_t rows = 0;
  int64_t all_rows = 0;
  for (int32_t i = 0; i < n; ++i) {
    rows = std::max(rows, c[i].rows);
    all_rows += c[i].rows;
  }
  if (rows == 0 || n_pools == 0) return CAS_OK;
  const size_t need = table_bytes(n);
  if ((s = check_workspace(workspace, ws_bytes, need)) != CAS_OK) return s;
  const uintptr_t pool = (uintptr_t)num_pages * (uintptr_t)page_size * (uintptr_t)row_bytes;
  std::vector<Interval> iv;
  iv.reserve((size_t)n_pools + 1);
  for (int32_t i = 0; i < n_pools; ++i) {
    if (!pools[i]) return set_error(CAS_ERR_INVALID_ARGUMENT, "pool " + str(i) + " is NULL");
    if ((uintptr_t)pools[i] & 15u) return set_error(CAS_ERR_ALIGNMENT, "pools must be 16-byte aligned");
    iv.push_back({(uintptr_t)pools[i], (uintptr_t)pools[i] + pool, true, (uintptr_t)i + 1, "a pool"});
  }
  if (need) iv.push_back({(uintptr_t)workspace, (uintptr_t)workspace + need, true, 0, "the workspace"});
  std::string msg;
  if (!overlap_free(iv, msg)) return set_error(CAS_ERR_INVALID_ARGUMENT, msg);
  PageCopyParams p;
  p.row_bytes = row_bytes;
  p.page_bytes = row_bytes * page_size;
  p.table = need ? (const cas_page_copy_t *)workspace : nullptr;
  p.piece = piece_bytes(all_rows, rows, n, row_bytes, n_pools);
  p.pieces = (int32_t)((rows * row_bytes + p.piece - 1) / p.piece);
  const int32_t most = std::max(1, (1 << 21) / p.pieces);   // copies of a launch, of at most 2^31 threads
  for (int32_t from = 0; from < n; from += kTableCopies) {
    const int32_t listed = std::min(kTableCopies, n - from);
    PageCopyList list;
    if (need) {
      // (The stream has read the copies before these by then.)
      const size_t bytes = ((size_t)listed * sizeof(cas_page_copy_t) + 15) / 16 * 16;
      s = upload_call_tables(bytes, workspace, stream, [&](char *h) { std::memcpy(h, c + from, (size_t)listed * sizeof(cas_page_copy_t)); });
      if (s != CAS_OK) return s;
    } else {
      std::memcpy(list.copies, c, (size_t)n * sizeof(cas_page_copy_t));
    }
    for (int32_t pool0 = 0; pool0 < n_pools; pool0 += kPageCopyPools) {
      const int32_t m = std::min(kPageCopyPools, n_pools - pool0);
      for (int32_t i = 0; i < m; ++i) p.pools[i] = (char *)pools[pool0 + i];
      for (p.first = 0; p.first < listed; p.first += most) {
        const int32_t k = std::min(most, listed - p.first);
        const hipError_t e = timed_launch("page_copy", stream, [&] { return launch_page_copy(p, need ? nullptr : &list, k, m, stream); });
        if (e != hipSuccess) return set_hip_error("page_copy launch", e);
      }
    }
  }
  return CAS_OK;
}

}  // namespace

extern "C" {

cas_status_t cas_page_table_create(int64_t num_pages, int32_t page_size, cas_page_table_t **table) {
  if (!table) return set_error(CAS_ERR_INVALID_ARGUMENT, "table is NULL");
  *table = nullptr;
  if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
    return set_error(CAS_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  if (num_pages < 1 || num_pages > INT32_MAX) return set_error(CAS_ERR_INVALID_ARGUMENT, "num_pages must be in [1, 2^31)");
  return guarded([&] {
    auto t = std::make_unique<cas_page_table>();
    t->num_pages = num_pages;
    t->page = page_size;
    *table = t.release();
    return CAS_OK;
  });
}

cas_status_t cas_page_table_destroy(cas_page_table_t *table) {
  delete table;
  return CAS_OK;
}

cas_status_t cas_page_table_info(const cas_page_table_t *table, cas_page_table_info_t *info) {
  if (!table || !info) return set_error(CAS_ERR_INVALID_ARGUMENT, "table or info is NULL");
  int64_t end = (int64_t)table->refs.size();
  while (end > 0 && table->refs[(size_t)end - 1] == 0) --end;
  *info = cas_page_table_info_t{(int64_t)table->seqs.size(), table->used, table->free_pages(), end};
  return CAS_OK;
}

cas_status_t cas_page_table_add(cas_page_table_t *table, const int64_t *parts, int32_t n, int64_t *seq) {
  if (!table || !seq) return set_error(CAS_ERR_INVALID_ARGUMENT, "table or seq is NULL");
  return guarded([&] { return add(*table, parts, n, seq); });
}

cas_status_t cas_page_table_extend(cas_page_table_t *table, const int64_t *seqs, int32_t n, const int32_t *counts,
                                   cas_page_copy_t *copies, int32_t *n_copies) {
  if (!table || !n_copies) return set_error(CAS_ERR_INVALID_ARGUMENT, "table or n_copies is NULL");
  return guarded([&] { return extend(*table, seqs, n, counts, copies, n_copies); });
}

cas_status_t cas_page_table_reorder(cas_page_table_t *table, const int64_t *seqs, int32_t n, const int32_t *parents) {
  if (!table) return set_error(CAS_ERR_INVALID_ARGUMENT, "table is NULL");
  return guarded([&] { return reorder(*table, seqs, n, parents); });
}

cas_status_t cas_page_table_truncate(cas_page_table_t *table, int64_t seq, int64_t len) {
  if (!table) return set_error(CAS_ERR_INVALID_ARGUMENT, "table is NULL");
  return guarded([&] {
    Sequence *x = table->find(seq);
    if (!x) return unknown(seq);
    if (len < 0 || len > x->len) return set_error(CAS_ERR_INVALID_ARGUMENT, "len must be in [0, the sequence's length]");
    reserve_pages(*table, 0);
    while ((int64_t)x->pages.size() > pages_for(*table, len)) {
      table->drop(x->pages.back());
      x->pages.pop_back();
    }
    x->len = len;
    return CAS_OK;
  });
}

cas_status_t cas_page_table_free(cas_page_table_t *table, const int64_t *seqs, int32_t n) {
  if (!table) return set_error(CAS_ERR_INVALID_ARGUMENT, "table is NULL");
  return guarded([&] {
    std::vector<Sequence *> q;
    const cas_status_t s = look_up(*table, seqs, n, q);
    if (s != CAS_OK) return s;
    reserve_pages(*table, 0);
    for (int32_t i = 0; i < n; ++i) {
      for (const int32_t p : q[(size_t)i]->pages) table->drop(p);
      table->seqs.erase(seqs[i]);
    }
    return CAS_OK;
  });
}

cas_status_t cas_page_table_compact(cas_page_table_t *table, int32_t most, cas_page_copy_t *copies, int32_t *n_copies) {
  if (!table || !n_copies) return set_error(CAS_ERR_INVALID_ARGUMENT, "table or n_copies is NULL");
  return guarded([&] { return compact(*table, most, copies, n_copies); });
}

cas_status_t cas_page_table_lists(const cas_page_table_t *table, const int64_t *seqs, int32_t n, int32_t *kv_lens,
                                  int32_t *page_offsets, int32_t *page_ids, int64_t cap) {
  if (!table || !page_offsets) return set_error(CAS_ERR_INVALID_ARGUMENT, "table or page_offsets is NULL");
  return guarded([&] {
    std::vector<Sequence *> q;
    const cas_status_t s = look_up(*const_cast<cas_page_table_t *>(table), seqs, n, q, false);
    if (s != CAS_OK) return s;
    if (n > 0 && !kv_lens) return set_error(CAS_ERR_INVALID_ARGUMENT, "kv_lens is NULL");
    int64_t total = 0;
    for (const Sequence *x : q) total += (int64_t)x->pages.size();
    if (total > INT32_MAX) return set_error(CAS_ERR_UNSUPPORTED, "more than 2^31 page ids");
    if (page_ids && cap < total) return set_error(CAS_ERR_INVALID_ARGUMENT, "room for " + str(cap) + " page ids, has " + str(total));
    int32_t at = 0;
    page_offsets[0] = 0;
    for (int32_t i = 0; i < n; ++i) {
      const Sequence &x = *q[(size_t)i];
      kv_lens[i] = (int32_t)x.len;
      if (page_ids && !x.pages.empty()) std::memcpy(page_ids + at, x.pages.data(), x.pages.size() * sizeof(int32_t));
      at += (int32_t)x.pages.size();
      page_offsets[i + 1] = at;
    }
    return CAS_OK;
  });
}

cas_status_t cas_pages_copy_workspace_size(int32_t n, size_t *bytes) {
  if (!bytes) return set_error(CAS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  if (n < 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "n must be >= 0");
  *bytes = table_bytes(n);
  return CAS_OK;
}

cas_status_t cas_pages_copy(void *const *pools, int32_t n_pools, int64_t num_pages, int32_t page_size, int64_t row_bytes,
                            const cas_page_copy_t *copies, int32_t n, void *workspace, size_t ws_bytes, void *hip_stream) {
  return guarded([&] {
    return copy_pages(pools, n_pools, num_pages, page_size, row_bytes, copies, n, workspace, ws_bytes, (hipStream_t)hip_stream);
  });
}

}  // extern "C"
