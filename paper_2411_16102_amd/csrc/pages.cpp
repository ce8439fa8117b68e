// Book-keeping of a cache's pages (host only): tables, references, the free numbers, forks and compaction.
#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <exception>
#include <limits>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/blendstep_stream.h"
#include "pages.hpp"

namespace {

constexpr int PAGE = 16;
constexpr int32_t MAX_TOKENS = 1 << 30;
thread_local std::string g_error;

// A set of small numbers that hands out the smallest; nothing but reserve() allocates.
class Numbers {
  std::vector<uint64_t> words_;
  size_t first_ = 0;  // no word before this one has a bit
  int64_t count_ = 0;

 public:
  void reserve(int64_t n) { if ((size_t)(n + 63) / 64 > words_.size()) words_.resize((size_t)(n + 63) / 64, 0); }
  int64_t size() const { return count_; }
  void insert(int32_t i) {
    words_[(size_t)i / 64] |= (uint64_t)1 << (i % 64);
    first_ = std::min(first_, (size_t)i / 64);
    ++count_;
  }
  int32_t take() {  // the set must not be empty
    while (!words_[first_]) ++first_;
    const int bit = __builtin_ctzll(words_[first_]);
    words_[first_] &= words_[first_] - 1;
    --count_;
    return (int32_t)(first_ * 64) + bit;
  }
  void clear() {
    std::fill(words_.begin(), words_.end(), 0);
    first_ = words_.size();
    count_ = 0;
  }
};

struct Sequence {
  bool live = false;
  int32_t tokens = 0;
  std::vector<int32_t> table;
};

}  // namespace

struct bs_pages {
  std::vector<int32_t> refs;   // references to each page
  int64_t most_refs = 1;       // no page has more
  Numbers free;                // pages without one
  std::vector<Sequence> seqs;
  Numbers free_ids;            // of seqs
  mutable std::string err;
};

namespace {

int fail(const bs_pages *p, int code, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    (p ? p->err : g_error) = buf;
  } catch (...) {
  }
  return code;
}

template <class F>
int guarded(const bs_pages *p, F &&body) {
  try {
    return body();
  } catch (const std::bad_alloc &) {
    return fail(p, BS_ENOMEM, "out of host memory");
  } catch (const std::exception &e) {
    return fail(p, BS_EINVAL, "unexpected exception: %s", e.what());
  } catch (...) {
    return fail(p, BS_EINVAL, "unexpected exception");
  }
}

int check_ids(const bs_pages *p, const int32_t *ids, int32_t n, bool once) {
  if (n < 0 || (n > 0 && !ids)) return fail(p, BS_EINVAL, "bad list of %d sequences", n);
  std::vector<char> seen(once ? p->seqs.size() : 0, 0);
  for (int32_t i = 0; i < n; ++i) {
    if (ids[i] < 0 || (size_t)ids[i] >= p->seqs.size() || !p->seqs[ids[i]].live) return fail(p, BS_EINVAL, "%d is no sequence", ids[i]);
    if (once && seen[ids[i]]++) return fail(p, BS_EINVAL, "sequence %d comes twice", ids[i]);
  }
  return BS_OK;
}

// room for n further sequences; nothing else changes
void reserve_ids(bs_pages *p, int64_t n) {
  const int64_t more = n - p->free_ids.size();
  if (more <= 0) return;
  const size_t before = p->seqs.size();
  p->free_ids.reserve((int64_t)before + more);
  p->seqs.resize(before + (size_t)more);
  for (size_t i = before; i < p->seqs.size(); ++i) p->free_ids.insert((int32_t)i);
}

void drop(bs_pages *p, int32_t page) {
  if (--p->refs[page] == 0) p->free.insert(page);
}

}  // namespace

namespace bs {

int32_t plan_compaction(const std::vector<char> &named, std::vector<int32_t> &to, std::vector<int32_t> &src, std::vector<int32_t> &dst) {
  const int32_t n_pages = (int32_t)named.size();
  const int32_t n_live = (int32_t)std::count(named.begin(), named.end(), 1);
  to.resize((size_t)n_pages);
  src.clear();
  dst.clear();
  int32_t hole = 0;
  for (int32_t i = 0; i < n_pages; ++i) {
    to[i] = i;
    if (!named[i] || i < n_live) continue;
    while (named[hole]) ++hole;  // (as many holes below n_live as live pages from it on)
    to[i] = hole;
    src.push_back(i);
    dst.push_back(hole++);
  }
  return n_live;
}

}  // namespace bs

extern "C" {

int bs_pages_create(int32_t n_pages, bs_pages **out) {
  if (!out) return fail(nullptr, BS_EINVAL, "out is NULL");
  *out = nullptr;
  return guarded(nullptr, [&]() -> int {
    if (n_pages < 0) return fail(nullptr, BS_EINVAL, "n_pages=%d", n_pages);
    bs_pages *p = new bs_pages();
    try {
      p->refs.assign((size_t)n_pages, 0);
      p->free.reserve(n_pages);
      for (int32_t i = 0; i < n_pages; ++i) p->free.insert(i);
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return BS_OK;
  });
}

void bs_pages_destroy(bs_pages *p) { delete p; }

const char *bs_pages_last_error(const bs_pages *p) { return p ? p->err.c_str() : g_error.c_str(); }

int bs_pages_open(bs_pages *p, int32_t n, int32_t *ids) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (n < 0 || (n > 0 && !ids)) return fail(p, BS_EINVAL, "bs_pages_open: bad argument");
    if ((int64_t)p->seqs.size() + n > 0x7fffffff) return fail(p, BS_EINVAL, "too many sequences");
    reserve_ids(p, n);
    for (int32_t i = 0; i < n; ++i) {
      ids[i] = p->free_ids.take();
      p->seqs[ids[i]].live = true;
    }
    return BS_OK;
  });
}

int bs_pages_fork(bs_pages *p, const int32_t *parents, int32_t n, int32_t children, int32_t *out) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (const int rc = check_ids(p, parents, n, false)) return rc;
    if (children < 0 || (int64_t)n * children > 0x7fffffff || (int64_t)p->seqs.size() + (int64_t)n * children > 0x7fffffff)
      return fail(p, BS_EINVAL, "bs_pages_fork: %d children of %d parents", children, n);
    if (n > 0 && children > 0 && !out) return fail(p, BS_EINVAL, "bs_pages_fork: out is NULL");
    const int64_t more = (int64_t)n * children;
    if (p->most_refs + more > std::numeric_limits<int32_t>::max()) {
      p->most_refs = 0;
      for (const int32_t r : p->refs) p->most_refs = std::max<int64_t>(p->most_refs, r);
      if (p->most_refs + more > std::numeric_limits<int32_t>::max()) return fail(p, BS_EINVAL, "too many references to a page");
    }
    reserve_ids(p, more);
    p->most_refs += more;
    std::vector<std::vector<int32_t>> tables((size_t)more);  // every allocation comes before the first change
    for (size_t i = 0; i < tables.size(); ++i) tables[i] = p->seqs[parents[i / (size_t)children]].table;
    for (size_t i = 0; i < tables.size(); ++i) {
      out[i] = p->free_ids.take();
      Sequence &s = p->seqs[out[i]];
      s.live = true;
      s.tokens = p->seqs[parents[i / (size_t)children]].tokens;
      s.table = std::move(tables[i]);
      for (const int32_t page : s.table)
        if (page >= 0) ++p->refs[page];
    }
    return BS_OK;
  });
}

int bs_pages_extend(bs_pages *p, const int32_t *ids, const int32_t *tokens, int32_t n, int32_t *src, int32_t *dst, int32_t *n_copies) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (const int rc = check_ids(p, ids, n, true)) return rc;
    if (!n_copies || (n > 0 && (!tokens || !src || !dst))) return fail(p, BS_EINVAL, "bs_pages_extend: NULL argument");
    // which open pages are shared goes by the references as they fall one by one; nothing is changed before there is room for all
    int64_t need = 0;
    std::vector<char> copied((size_t)n, 0);
    std::vector<std::pair<int32_t, int32_t>> left;  // (open page, sequences of this call that have left it), by page
    for (int32_t i = 0; i < n; ++i) {
      Sequence &s = p->seqs[ids[i]];
      if (tokens[i] < 0 || (int64_t)s.tokens + tokens[i] > MAX_TOKENS) return fail(p, BS_EINVAL, "sequence %d: %d further tokens", ids[i], tokens[i]);
      if (tokens[i] == 0) continue;
      if (s.tokens % PAGE) left.push_back({s.table.back(), i});
      need += (s.tokens + tokens[i] + PAGE - 1) / PAGE - (int64_t)s.table.size();
    }
    std::sort(left.begin(), left.end());
    for (size_t i = 0, at = 0; i < left.size(); ++i) {
      if (i == 0 || left[i].first != left[i - 1].first) at = i;
      copied[left[i].second] = p->refs[left[i].first] - (int32_t)(i - at) > 1;  // all but the last reference are copied
      need += copied[left[i].second];
    }
    if (need > p->free.size()) return fail(p, BS_ENOMEM, "%lld pages are needed, %lld are free", (long long)need, (long long)p->free.size());
    for (int32_t i = 0; i < n; ++i) {
      Sequence &s = p->seqs[ids[i]];
      if (tokens[i] > 0) s.table.reserve((size_t)(s.tokens + tokens[i] + PAGE - 1) / PAGE);
    }
    int32_t copies = 0;
    const auto take = [&]() {
      const int32_t page = p->free.take();
      p->refs[page] = 1;
      return page;
    };
    for (int32_t i = 0; i < n; ++i) {
      Sequence &s = p->seqs[ids[i]];
      if (tokens[i] == 0) continue;
      if (copied[i]) {
        src[copies] = s.table.back();
        --p->refs[s.table.back()];
        s.table.back() = dst[copies++] = take();
      }
      s.tokens += tokens[i];
      while ((int64_t)s.table.size() * PAGE < s.tokens) s.table.push_back(take());
    }
    *n_copies = copies;
    return BS_OK;
  });
}

int bs_pages_trim(bs_pages *p, const int32_t *ids, int32_t n, int32_t window, int32_t sinks) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (const int rc = check_ids(p, ids, n, false)) return rc;
    if (window < 1 || sinks < 0) return fail(p, BS_EINVAL, "window %d must be at least 1 and sinks %d at least 0", window, sinks);
    for (int32_t i = 0; i < n; ++i) {
      Sequence &s = p->seqs[ids[i]];
      // the next row stands at `tokens` and sees tokens above tokens - window
      const int64_t first = ((int64_t)sinks + PAGE - 1) / PAGE, end = std::max<int64_t>(0, (int64_t)s.tokens - window + 1) / PAGE;
      for (int64_t k = first; k < std::min<int64_t>(end, (int64_t)s.table.size()); ++k)
        if (s.table[k] >= 0) {
          drop(p, s.table[k]);
          s.table[k] = BS_PAGE_NONE;
        }
    }
    return BS_OK;
  });
}

int bs_pages_free(bs_pages *p, const int32_t *ids, int32_t n) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (const int rc = check_ids(p, ids, n, true)) return rc;
    for (int32_t i = 0; i < n; ++i) {
      Sequence &s = p->seqs[ids[i]];
      p->free_ids.insert(ids[i]);
      for (const int32_t page : s.table)
        if (page >= 0) drop(p, page);
      s = Sequence();
    }
    return BS_OK;
  });
}

int bs_pages_compact(bs_pages *p, int32_t *src, int32_t *dst, int32_t *n_moves, int32_t *n_live) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (!n_moves || !n_live || (!p->refs.empty() && (!src || !dst))) return fail(p, BS_EINVAL, "bs_pages_compact: NULL argument");
    std::vector<char> named(p->refs.size());
    for (size_t i = 0; i < named.size(); ++i) named[i] = p->refs[i] > 0;
    std::vector<int32_t> to, from, into;
    const int32_t live = bs::plan_compaction(named, to, from, into);
    for (size_t i = 0; i < from.size(); ++i) {
      src[i] = from[i];
      dst[i] = into[i];
      p->refs[into[i]] = p->refs[from[i]];
      p->refs[from[i]] = 0;
    }
    for (Sequence &s : p->seqs)
      for (int32_t &page : s.table)
        if (page >= 0) page = to[page];
    p->free.clear();
    for (int32_t i = live; i < (int32_t)named.size(); ++i) p->free.insert(i);
    *n_moves = (int32_t)from.size();
    *n_live = live;
    return BS_OK;
  });
}

int bs_pages_tables(const bs_pages *p, const int32_t *ids, int32_t n, int32_t *tokens, int32_t *page_start, int32_t *page_ids, int64_t room) {
  if (!p) return BS_EINVAL;
  return guarded(p, [&]() -> int {
    if (const int rc = check_ids(p, ids, n, false)) return rc;
    if (!page_start || (n > 0 && !tokens)) return fail(p, BS_EINVAL, "bs_pages_tables: NULL argument");
    int64_t at = 0;
    for (int32_t i = 0; i < n; ++i) at += (int64_t)p->seqs[ids[i]].table.size();
    if (at > 0x7fffffff) return fail(p, BS_EINVAL, "tables of %lld pages", (long long)at);
    if (at > room) page_ids = nullptr;
    page_start[0] = 0;
    for (int32_t i = 0; i < n; ++i) {
      const Sequence &s = p->seqs[ids[i]];
      tokens[i] = s.tokens;
      page_start[i + 1] = page_start[i] + (int32_t)s.table.size();
      if (page_ids && !s.table.empty()) std::memcpy(page_ids + page_start[i], s.table.data(), sizeof(int32_t) * s.table.size());
    }
    return BS_OK;
  });
}

int bs_pages_stats(const bs_pages *p, int32_t *n_free, int32_t *n_sequences) {
  if (!p) return BS_EINVAL;
  if (n_free) *n_free = (int32_t)p->free.size();
  if (n_sequences) *n_sequences = (int32_t)(p->seqs.size() - p->free_ids.size());
  return BS_OK;
}

}  // extern "C"
