// Which sequence owns which page of a cache (pbz_cache.h): host code only.
#include <algorithm>
#include <cstring>
#include <mutex>
#include <new>
#include <unordered_map>
#include <vector>

#include "pbz_cache.h"

namespace {

struct Sequence {
  int64_t length = 0;
  std::vector<int32_t> pages;
};

bool is_pow2(int64_t v) { return v >= 1 && (v & (v - 1)) == 0; }

}  // namespace

struct pbz_pages {
  int32_t page_size;
  std::vector<int32_t> owners;      // [n_pages] sequences that hold the page
  std::vector<int32_t> free_pages;  // a stack; room for every page is reserved, so that letting go never allocates
  std::unordered_map<int64_t, Sequence> sequences;
  int64_t next = 1;
  mutable std::mutex mu;

  void let_go(int32_t page) {
    if (--owners[size_t(page)] == 0) free_pages.push_back(page);
  }
};

// nothing throws across the boundary: the standard containers' only exception here is a failed allocation
template <typename F>
static int guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return PBZ_ERR_ALLOC;
  }
}

extern "C" {

int pbz_pages_create(pbz_pages** out, int64_t n_pages, int32_t page_size) {
  if (!out) return PBZ_ERR_NULL;
  *out = nullptr;
  if (n_pages < 1 || n_pages > INT32_MAX || page_size < 16 || page_size > 1024 || !is_pow2(page_size)) return PBZ_ERR_SHAPE;
  pbz_pages* p = new (std::nothrow) pbz_pages();
  if (!p) return PBZ_ERR_ALLOC;
  const int st = guarded([&] {
    p->page_size = page_size;
    p->owners.assign(size_t(n_pages), 0);
    p->free_pages.resize(size_t(n_pages));
    for (int64_t i = 0; i < n_pages; ++i) p->free_pages[size_t(i)] = int32_t(n_pages - 1 - i);   // page 0 goes first
    return PBZ_OK;
  });
  if (st != PBZ_OK) {
    delete p;
    return st;
  }
  *out = p;
  return PBZ_OK;
}

void pbz_pages_destroy(pbz_pages* p) { delete p; }

int pbz_pages_open(pbz_pages* p, int64_t* sequence) {
  if (!p || !sequence) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  return guarded([&] {
    p->sequences.emplace(p->next, Sequence());
    *sequence = p->next++;
    return PBZ_OK;
  });
}

int pbz_pages_fork(pbz_pages* p, int64_t sequence, int64_t* child) {
  if (!p || !child) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  return guarded([&] {
    Sequence copy = it->second;
    const auto made = p->sequences.emplace(p->next, std::move(copy));
    for (int32_t page : made.first->second.pages) ++p->owners[size_t(page)];
    *child = p->next++;
    return PBZ_OK;
  });
}

int pbz_pages_close(pbz_pages* p, int64_t sequence) {
  if (!p) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  for (auto page = it->second.pages.rbegin(); page != it->second.pages.rend(); ++page) p->let_go(*page);
  p->sequences.erase(it);
  return PBZ_OK;
}

int pbz_pages_extend(pbz_pages* p, int64_t sequence, int64_t tokens, int64_t* slots, int32_t copy[2], int32_t* n_copies) {
  if (!p || !slots || !copy || !n_copies) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  Sequence& s = it->second;
  const int64_t size = p->page_size;
  if (tokens < 1 || tokens > int64_t(INT32_MAX) - s.length) return PBZ_ERR_SHAPE;    // lengths are 32-bit on the device
  const int64_t have = int64_t(s.pages.size());
  const int64_t need = (s.length + tokens + size - 1) / size - have;
  const bool shared = s.length % size != 0 && p->owners[size_t(s.pages.back())] > 1;
  if (need + (shared ? 1 : 0) > int64_t(p->free_pages.size())) return PBZ_ERR_PAGES;
  return guarded([&] {
    s.pages.reserve(size_t(have + need));            // the only allocation, before anything changes
    *n_copies = 0;
    const auto take = [&] {
      const int32_t page = p->free_pages.back();
      p->free_pages.pop_back();
      p->owners[size_t(page)] = 1;
      return page;
    };
    if (shared) {
      copy[0] = s.pages.back();
      copy[1] = take();
      *n_copies = 1;
      p->let_go(copy[0]);
      s.pages.back() = copy[1];
    }
    for (int64_t i = 0; i < need; ++i) s.pages.push_back(take());
    for (int64_t i = 0; i < tokens; ++i) {
      const int64_t j = s.length + i;
      slots[i] = int64_t(s.pages[size_t(j / size)]) * size + j % size;
    }
    s.length += tokens;
    return PBZ_OK;
  });
}

int pbz_pages_truncate(pbz_pages* p, int64_t sequence, int64_t length) {
  if (!p) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  Sequence& s = it->second;
  if (length < 0 || length > s.length) return PBZ_ERR_SHAPE;
  const size_t keep = size_t((length + p->page_size - 1) / p->page_size);
  while (s.pages.size() > keep) {
    p->let_go(s.pages.back());
    s.pages.pop_back();
  }
  s.length = length;
  return PBZ_OK;
}

int pbz_pages_length(const pbz_pages* p, int64_t sequence, int64_t* length, int64_t* n_pages) {
  if (!p) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  if (length) *length = it->second.length;
  if (n_pages) *n_pages = int64_t(it->second.pages.size());
  return PBZ_OK;
}

int pbz_pages_table(const pbz_pages* p, int64_t sequence, int32_t* table, int64_t capacity) {
  if (!p || !table) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const auto it = p->sequences.find(sequence);
  if (it == p->sequences.end()) return PBZ_ERR_SEQUENCE;
  const std::vector<int32_t>& pages = it->second.pages;
  if (capacity < int64_t(pages.size())) return PBZ_ERR_CAPACITY;
  std::copy(pages.begin(), pages.end(), table);
  std::fill(table + pages.size(), table + capacity, -1);
  return PBZ_OK;
}

int pbz_pages_free_count(const pbz_pages* p, int64_t* n_free) {
  if (!p || !n_free) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  *n_free = int64_t(p->free_pages.size());
  return PBZ_OK;
}

int pbz_pages_compact(pbz_pages* p, int32_t* pairs, int64_t capacity, int64_t* n_pairs) {
  if (!p || !n_pairs || (!pairs && capacity > 0)) return PBZ_ERR_NULL;
  std::lock_guard<std::mutex> lock(p->mu);
  const int64_t total = int64_t(p->owners.size());
  const int64_t used = total - int64_t(p->free_pages.size());
  int64_t moves = 0;
  for (int64_t i = used; i < total; ++i) moves += p->owners[size_t(i)] > 0;
  if (moves > capacity) return PBZ_ERR_CAPACITY;
  return guarded([&] {
    std::vector<int32_t> moved(static_cast<size_t>(total - used), -1);       // where page used + i goes
    int64_t hole = 0, n = 0;
    for (int64_t i = used; i < total; ++i) {
      if (p->owners[size_t(i)] == 0) continue;
      while (p->owners[size_t(hole)] != 0) ++hole;              // there are as many free pages below as used ones above
      pairs[2 * n] = int32_t(i);
      pairs[2 * n + 1] = int32_t(hole);
      ++n;
      moved[size_t(i - used)] = int32_t(hole);
      p->owners[size_t(hole)] = p->owners[size_t(i)];
      p->owners[size_t(i)] = 0;
    }
    for (auto& entry : p->sequences)
      for (int32_t& page : entry.second.pages)
        if (page >= used) page = moved[size_t(page - used)];
    p->free_pages.clear();
    for (int64_t i = total - 1; i >= used; --i) p->free_pages.push_back(int32_t(i));
    *n_pairs = n;
    return PBZ_OK;
  });
}

}  // extern "C"
