// Page bookkeeping of the paged cache (speccache.h): sequences, the pages they
// hold, how many sequences share each page.  Host code only.  Free pages are
// bits, so that the lowest id is handed out first (used pages stay near the
// front of the pool) and giving pages back takes no memory.
#include "../../include/speccache.h"

#include <algorithm>
#include <cstdint>
#include <vector>

namespace {

struct Sequence {
  bool open = false;
  int32_t tokens = 0;
  std::vector<int32_t> pages;
};

template <typename F>
spec_status_t guarded(F&& f) noexcept {
  try {
    return f();
  } catch (...) {
    return SPEC_ERR_WORKSPACE;         // memory that the host does not have
  }
}

}  // namespace

struct spec_pages {
  int32_t page_tokens = 0;
  int32_t free_count = 0;
  std::vector<int32_t> holders;        // sequences that hold each page
  std::vector<uint64_t> free_bits;
  size_t low = 0;                      // no word before this one has a free page
  std::vector<Sequence> seqs;

  bool has(int32_t s) const { return s >= 0 && s < (int32_t)seqs.size() && seqs[s].open; }

  // Room for one more open sequence: its id (not opened yet).
  int32_t vacant() {
    for (size_t i = 0; i < seqs.size(); ++i)
      if (!seqs[i].open) return (int32_t)i;
    seqs.emplace_back();
    return (int32_t)seqs.size() - 1;
  }
  bool is_free(int32_t p) const { return (free_bits[p / 64] >> (p % 64)) & 1; }
  // The free page with the lowest id (there is one).
  int32_t take() {
    while (free_bits[low] == 0) ++low;
    const int32_t p = (int32_t)(low * 64) + __builtin_ctzll(free_bits[low]);
    free_bits[low] &= free_bits[low] - 1;
    holders[p] = 1;
    --free_count;
    return p;
  }
  void set_free(int32_t p) {
    free_bits[p / 64] |= 1ull << (p % 64);
    low = std::min(low, (size_t)(p / 64));
    ++free_count;
  }
  void give_back(int32_t p) {
    if (--holders[p] == 0) set_free(p);
  }
};

extern "C" {

spec_status_t spec_pages_create(int32_t num_pages, int32_t page_tokens, spec_pages_t** out) {
  if (!out || num_pages < 1 || page_tokens < 32 || page_tokens % 32) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    spec_pages* p = new spec_pages;
    try {
      p->page_tokens = page_tokens;
      p->holders.assign(num_pages, 0);
      p->free_bits.assign(((size_t)num_pages + 63) / 64, 0);
      for (int32_t i = 0; i < num_pages; ++i) p->set_free(i);
    } catch (...) {
      delete p;
      throw;
    }
    *out = p;
    return SPEC_OK;
  });
}

void spec_pages_destroy(spec_pages_t* pages) { delete pages; }

spec_status_t spec_pages_open(spec_pages_t* p, int32_t* sequence) {
  if (!p || !sequence) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    const int32_t s = p->vacant();
    p->seqs[s].open = true;
    *sequence = s;
    return SPEC_OK;
  });
}

spec_status_t spec_pages_resize(spec_pages_t* p, int32_t sequence, int32_t tokens, spec_page_copy_t* copy) {
  if (!p || !copy || tokens < 0 || !p->has(sequence)) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    Sequence& q = p->seqs[sequence];
    const int32_t P = p->page_tokens;
    const size_t want = ((size_t)tokens + P - 1) / P;
    spec_page_copy_t c = {0, 0, 0};
    if (tokens > q.tokens) {
      // rows are added: behind a shared, partly filled page on a copy of it
      const int32_t tail = q.tokens % P;
      const bool apart = tail != 0 && p->holders[q.pages.back()] > 1;
      const size_t need = want - q.pages.size() + (apart ? 1 : 0);
      if (need > (size_t)p->free_count) return SPEC_ERR_NO_PAGES;
      q.pages.reserve(want);
      if (apart) {
        c.src = q.pages.back();
        c.dst = p->take();
        c.tokens = tail;
        p->give_back(c.src);
        q.pages.back() = c.dst;
      }
      while (q.pages.size() < want) q.pages.push_back(p->take());
    } else {
      while (q.pages.size() > want) {
        p->give_back(q.pages.back());
        q.pages.pop_back();
      }
    }
    q.tokens = tokens;
    *copy = c;
    return SPEC_OK;
  });
}

spec_status_t spec_pages_fork(spec_pages_t* p, int32_t sequence, int32_t* child) {
  if (!p || !child || !p->has(sequence)) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    const int32_t s = p->vacant();
    p->seqs[s].pages = p->seqs[sequence].pages;
    p->seqs[s].tokens = p->seqs[sequence].tokens;
    p->seqs[s].open = true;
    for (int32_t x : p->seqs[s].pages) ++p->holders[x];
    *child = s;
    return SPEC_OK;
  });
}

spec_status_t spec_pages_close(spec_pages_t* p, int32_t sequence) {
  if (!p || !p->has(sequence)) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    Sequence& q = p->seqs[sequence];
    while (!q.pages.empty()) {
      p->give_back(q.pages.back());
      q.pages.pop_back();
    }
    q.tokens = 0;
    q.open = false;
    return SPEC_OK;
  });
}

spec_status_t spec_pages_table(const spec_pages_t* p, int32_t sequence, int32_t* out, int32_t max, int32_t* count) {
  if (!p || !count || max < 0 || (max > 0 && !out) || !p->has(sequence)) return SPEC_ERR_INVALID_ARG;
  const std::vector<int32_t>& pages = p->seqs[sequence].pages;
  *count = (int32_t)pages.size();
  if (max < *count) return SPEC_ERR_WORKSPACE;
  std::copy(pages.begin(), pages.end(), out);
  return SPEC_OK;
}

spec_status_t spec_pages_compact(spec_pages_t* p, spec_page_copy_t* copies, int32_t max, int32_t* count) {
  if (!p || !count || max < 0 || (max > 0 && !copies)) return SPEC_ERR_INVALID_ARG;
  return guarded([&]() -> spec_status_t {
    const int32_t n = (int32_t)p->holders.size();
    const int32_t used = n - p->free_count;
    // the free pages in front, and as many used ones behind
    std::vector<int32_t> to, from;
    for (int32_t x = 0; x < used; ++x)
      if (p->is_free(x)) to.push_back(x);
    if (max < (int32_t)to.size()) {
      *count = (int32_t)to.size();
      return SPEC_ERR_WORKSPACE;
    }
    for (int32_t x = n - 1; x >= used && !to.empty(); --x)
      if (!p->is_free(x)) from.push_back(x);             // highest first
    std::vector<int32_t> now(n), rows(n, 0);
    for (int32_t x = 0; x < n; ++x) now[x] = x;
    for (const Sequence& q : p->seqs)
      for (size_t j = 0; j < q.pages.size(); ++j) {
        const int64_t left = q.tokens - (int64_t)j * p->page_tokens;
        rows[q.pages[j]] = std::max(rows[q.pages[j]], (int32_t)std::min<int64_t>(left, p->page_tokens));
      }
    // nothing below takes memory
    for (size_t i = 0; i < to.size(); ++i) {
      copies[i] = {from[i], to[i], rows[from[i]]};
      now[from[i]] = to[i];
      p->holders[to[i]] = p->holders[from[i]];
      p->holders[from[i]] = 0;
      p->free_bits[to[i] / 64] &= ~(1ull << (to[i] % 64));
      p->free_bits[from[i] / 64] |= 1ull << (from[i] % 64);
    }
    for (Sequence& q : p->seqs)
      for (int32_t& x : q.pages) x = now[x];
    p->low = 0;
    *count = (int32_t)to.size();
    return SPEC_OK;
  });
}

int32_t spec_pages_free_count(const spec_pages_t* p) { return p ? p->free_count : 0; }

}  // extern "C"
