// Bookkeeping of a paged cache whose sequences share pages: which pages a sequence
// lists, how many sequences list a page, which are free.  Host only.
#include <algorithm>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "horizon.h"
#include "plan.h"

using hs::fail;

struct hs_pages {
  struct Sequence {
    std::vector<int32_t> pages;
    int32_t len = 0;
  };
  int32_t n_pages = 0, positions = 0, per_seq = 0, used = 0;
  std::vector<int32_t> users;  // sequences that list a page
  std::vector<Sequence> seqs;
  // Free pages, the lowest first.
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free;

  int32_t take() {
    const int32_t p = free.top();
    free.pop();
    users[p] = 1;
    ++used;
    return p;
  }
  void drop(int32_t p) {
    if (--users[p] == 0) {
      free.push(p);  // the queue has held every page before: no allocation
      --used;
    }
  }
};

namespace {

constexpr int32_t kMaxPages = 1 << 28, kMaxSequences = 1 << 24;

hs_status check_seqs(const hs_pages* p, const int32_t* seqs, int32_t n, bool distinct) {
  if (!p) return fail(HS_ERR_INVALID_ARG, "pages is null");
  if (n < 0 || (n > 0 && !seqs)) return fail(HS_ERR_INVALID_ARG, "%d sequences, or their list is null", n);
  for (int32_t i = 0; i < n; ++i)
    if (seqs[i] < 0 || seqs[i] >= int32_t(p->seqs.size()))
      return fail(HS_ERR_INVALID_ARG, "sequence %d outside [0, %zu)", seqs[i], p->seqs.size());
  if (distinct) {
    std::vector<int32_t> sorted(seqs, seqs + n);
    std::sort(sorted.begin(), sorted.end());
    const auto twice = std::adjacent_find(sorted.begin(), sorted.end());
    if (twice != sorted.end()) return fail(HS_ERR_INVALID_ARG, "sequence %d is listed twice", *twice);
  }
  return HS_OK;
}

int32_t pages_for(const hs_pages* p, int64_t len) { return int32_t((len + p->positions - 1) / p->positions); }

// Runs f, which allocates before it changes anything.
template <typename F>
hs_status guarded(F f) {
  hs::clear_error();
  try {
    return f();
  } catch (const std::exception&) {
    return fail(HS_ERR_INTERNAL, "out of host memory");
  }
}

}  // namespace

extern "C" {

hs_status hs_pages_create(int32_t n_pages, int32_t page_positions, int32_t max_seqs, int32_t pages_per_seq,
                          hs_pages** out) {
  return guarded([&] {
    if (!out) return fail(HS_ERR_INVALID_ARG, "output pointer is null");
    *out = nullptr;
    if (n_pages < 1 || max_seqs < 1 || pages_per_seq < 1)
      return fail(HS_ERR_INVALID_ARG, "%d pages, %d sequences of %d", n_pages, max_seqs, pages_per_seq);
    if (page_positions < 64 || page_positions % 64 != 0)
      return fail(HS_ERR_INVALID_ARG, "page size %d must be a positive multiple of 64", page_positions);
    if (n_pages > kMaxPages || max_seqs > kMaxSequences)
      return fail(HS_ERR_UNSUPPORTED, "%d pages, %d sequences: at most %d and %d", n_pages, max_seqs, kMaxPages,
                  kMaxSequences);
    if (int64_t(pages_per_seq) * page_positions > (int64_t(1) << 30))
      return fail(HS_ERR_UNSUPPORTED, "%lld positions a sequence", (long long)pages_per_seq * page_positions);
    auto* p = new hs_pages();
    try {
      p->n_pages = n_pages;
      p->positions = page_positions;
      p->per_seq = pages_per_seq;
      p->users.assign(size_t(n_pages), 0);
      p->seqs.resize(size_t(max_seqs));
      std::vector<int32_t> all(static_cast<size_t>(n_pages));
      for (int32_t i = 0; i < n_pages; ++i) all[i] = i;
      p->free = decltype(p->free)(std::greater<int32_t>(), std::move(all));
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return HS_OK;
  });
}

hs_status hs_pages_destroy(hs_pages* pages) {
  delete pages;
  return HS_OK;
}

hs_status hs_pages_reserve(hs_pages* p, const int32_t* seqs, const int32_t* add, int32_t n, int32_t* src, int32_t* dst,
                           int32_t* positions, int32_t* n_copies) {
  return guarded([&] {
    if (n_copies) *n_copies = 0;
    hs_status st = check_seqs(p, seqs, n, true);
    if (st != HS_OK) return st;
    if (n > 0 && (!add || !src || !dst || !positions)) return fail(HS_ERR_INVALID_ARG, "an array is null");
    if (!n_copies) return fail(HS_ERR_INVALID_ARG, "n_copies is null");
    // What the call takes, before it takes any.  A shared last page costs all but
    // the last of its users that write to it a page, and that one too while others
    // still list it.
    int64_t need = 0;
    std::vector<int32_t> left;  // pages that a sequence of the call would leave
    left.reserve(size_t(n));
    st = [&] {
      for (int32_t i = 0; i < n; ++i) {
        const hs_pages::Sequence& s = p->seqs[seqs[i]];
        if (add[i] < 0) return fail(HS_ERR_INVALID_ARG, "add[%d] = %d", i, add[i]);
        const int64_t len = int64_t(s.len) + add[i];
        if (len > int64_t(p->per_seq) * p->positions)
          return fail(HS_ERR_INVALID_ARG, "sequence %d would hold %lld positions, beyond its %d pages of %d", seqs[i],
                      (long long)len, p->per_seq, p->positions);
        if (add[i] == 0) continue;
        need += pages_for(p, len) - int32_t(s.pages.size());
        if (s.len % p->positions != 0 && p->users[s.pages.back()] > 1) {
          --p->users[s.pages.back()];
          left.push_back(s.pages.back());
          ++need;
        }
      }
      return HS_OK;
    }();
    for (int32_t page : left) ++p->users[page];  // as it was
    if (st != HS_OK) return st;
    if (need > int64_t(p->free.size()))
      return fail(HS_ERR_WORKSPACE, "%lld pages needed, %zu are free", (long long)need, p->free.size());
    for (int32_t i = 0; i < n; ++i) p->seqs[seqs[i]].pages.reserve(size_t(p->per_seq));
    for (int32_t i = 0; i < n; ++i) {
      hs_pages::Sequence& s = p->seqs[seqs[i]];
      if (add[i] == 0) continue;
      if (s.len % p->positions != 0 && p->users[s.pages.back()] > 1) {
        const int32_t own = p->take();
        src[*n_copies] = s.pages.back();
        dst[*n_copies] = own;
        positions[(*n_copies)++] = s.len % p->positions;
        --p->users[s.pages.back()];
        s.pages.back() = own;
      }
      s.len += add[i];
      while (int32_t(s.pages.size()) < pages_for(p, s.len)) s.pages.push_back(p->take());
    }
    return HS_OK;
  });
}

hs_status hs_pages_fork(hs_pages* p, const int32_t* seqs, const int32_t* parents, int32_t n) {
  return guarded([&] {
    hs_status st = check_seqs(p, seqs, n, true);
    if (st != HS_OK) return st;
    if (n > 0 && !parents) return fail(HS_ERR_INVALID_ARG, "parents is null");
    for (int32_t i = 0; i < n; ++i)
      if (parents[i] < -1 || parents[i] >= int32_t(p->seqs.size()))
        return fail(HS_ERR_INVALID_ARG, "parent %d outside [-1, %zu)", parents[i], p->seqs.size());
    std::vector<hs_pages::Sequence> next(static_cast<size_t>(n));
    for (int32_t i = 0; i < n; ++i)
      if (parents[i] >= 0) next[i] = p->seqs[parents[i]];
    for (const hs_pages::Sequence& s : next)
      for (int32_t page : s.pages) ++p->users[page];
    for (int32_t i = 0; i < n; ++i) {
      for (int32_t page : p->seqs[seqs[i]].pages) p->drop(page);
      p->seqs[seqs[i]] = std::move(next[i]);
    }
    return HS_OK;
  });
}

hs_status hs_pages_compact(hs_pages* p, int32_t room, int32_t* src, int32_t* dst, int32_t* positions,
                           int32_t* n_copies) {
  return guarded([&] {
    if (n_copies) *n_copies = 0;
    if (!p) return fail(HS_ERR_INVALID_ARG, "pages is null");
    if (room < 0 || (room > 0 && (!src || !dst || !positions)) || !n_copies)
      return fail(HS_ERR_INVALID_ARG, "room %d, or an array is null", room);
    std::vector<int32_t> to(size_t(p->n_pages), -1), filled(size_t(p->n_pages), 0);
    for (const hs_pages::Sequence& s : p->seqs)
      for (size_t j = 0; j < s.pages.size(); ++j)
        filled[s.pages[j]] = std::max(filled[s.pages[j]], std::min(p->positions, s.len - int32_t(j) * p->positions));
    int32_t high = p->n_pages - 1, count = 0;
    std::vector<int32_t> rest;  // free pages after the call; drop() needs room for all
    rest.reserve(size_t(p->n_pages));
    for (int32_t low = 0; low < p->used && count < room; ++low) {
      if (p->users[low] != 0) continue;
      while (p->users[high] == 0) --high;
      if (high < p->used) break;
      to[high] = low;
      src[count] = high;
      dst[count] = low;
      positions[count++] = filled[high];
      --high;
    }
    for (int32_t i = 0; i < count; ++i) {
      p->users[dst[i]] = p->users[src[i]];
      p->users[src[i]] = 0;
    }
    for (hs_pages::Sequence& s : p->seqs)
      for (int32_t& page : s.pages)
        if (to[page] >= 0) page = to[page];
    for (int32_t i = 0; i < p->n_pages; ++i)
      if (p->users[i] == 0) rest.push_back(i);
    p->free = decltype(p->free)(std::greater<int32_t>(), std::move(rest));
    *n_copies = count;
    return HS_OK;
  });
}

hs_status hs_pages_table(const hs_pages* p, const int32_t* seqs, int32_t n, int32_t* table, int32_t* lens) {
  return guarded([&] {
    hs_status st = check_seqs(p, seqs, n, false);
    if (st != HS_OK) return st;
    for (int32_t i = 0; i < n; ++i) {
      const hs_pages::Sequence& s = p->seqs[seqs[i]];
      if (lens) lens[i] = s.len;
      if (!table) continue;
      int32_t* row = table + int64_t(i) * p->per_seq;
      std::copy(s.pages.begin(), s.pages.end(), row);
      std::fill(row + s.pages.size(), row + p->per_seq, 0);
    }
    return HS_OK;
  });
}

hs_status hs_pages_shared(const hs_pages* p, const int32_t* seqs, int32_t n, int32_t* positions) {
  return guarded([&] {
    hs_status st = check_seqs(p, seqs, n, false);
    if (st != HS_OK) return st;
    if (n < 1 || !positions) return fail(HS_ERR_INVALID_ARG, "no sequences, or positions is null");
    const hs_pages::Sequence& first = p->seqs[seqs[0]];
    int32_t pages = first.len / p->positions;
    for (int32_t i = 1; i < n; ++i) {
      const hs_pages::Sequence& s = p->seqs[seqs[i]];
      pages = std::min(pages, s.len / p->positions);
      const auto end = std::mismatch(first.pages.begin(), first.pages.begin() + pages, s.pages.begin()).first;
      pages = int32_t(end - first.pages.begin());
    }
    *positions = pages * p->positions;
    return HS_OK;
  });
}

hs_status hs_pages_free_count(const hs_pages* p, int32_t* n_free) {
  return guarded([&] {
    if (!p || !n_free) return fail(HS_ERR_INVALID_ARG, "null argument");
    *n_free = p->n_pages - p->used;
    return HS_OK;
  });
}

}  // extern "C"
