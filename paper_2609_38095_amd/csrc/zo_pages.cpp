// Host-only page book of the paged cache: sequences, shared pages with their counts, free pages.
//
// Free pages are handed out lowest id first when the book is new, afterwards the last freed one
// first (its lines are the likeliest to be cached still). Every call that may need memory reserves it
// before it changes anything, so a failed call leaves the book as it was.

#include <algorithm>
#include <new>
#include <stdexcept>
#include <vector>

#include "zo_decode.h"
#include "zo_tree.h"

struct zo_pages {
  struct Seq {
    std::vector<int32_t> pages;
    int64_t tokens = -1;  // -1: the number is not in use
  };
  uint32_t page_tokens;
  std::vector<uint32_t> holders;  // of each page
  std::vector<int32_t> free_ids;  // the next one last
  std::vector<Seq> seqs;
  std::vector<uint32_t> free_seqs;

  bool has(uint32_t seq) const { return seq < seqs.size() && seqs[seq].tokens >= 0; }

  uint64_t pages_of(uint64_t tokens) const { return (tokens + page_tokens - 1) / page_tokens; }

  int32_t take() {
    const int32_t id = free_ids.back();
    free_ids.pop_back();
    holders[id] = 1;
    return id;
  }

  void leave(int32_t id) {  // free_ids has room for every page from the start
    if (--holders[id] == 0) free_ids.push_back(id);
  }

  // A number for a new sequence; its entry is empty, and stays unused until the caller sets tokens.
  uint32_t reserve_seq() {
    if (free_seqs.empty()) {
      if (seqs.size() >= 0xFFFFFFu) throw std::bad_alloc();
      if (free_seqs.capacity() <= seqs.size()) free_seqs.reserve(2 * seqs.size() + 8);  // so that dropping never allocates
      seqs.emplace_back();
      free_seqs.push_back(static_cast<uint32_t>(seqs.size() - 1));
    }
    return free_seqs.back();
  }
};

namespace {

constexpr int64_t kMaxTokens = 0x7FFFFFFF;  // lengths and positions are int32

template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return ZO_ERR_MEMORY;
  } catch (const std::length_error&) {
    return ZO_ERR_MEMORY;
  }
}

}  // namespace

extern "C" {

zo_pages* zo_pages_open(uint32_t pages, uint32_t page_tokens) {
  if (pages == 0 || page_tokens == 0 || pages > 0x7FFFFFFFu || page_tokens > 0x7FFFFFFFu) return nullptr;
  zo_pages* book = nullptr;
  const int rc = guarded([&] {
    book = new zo_pages;
    book->page_tokens = page_tokens;
    book->holders.assign(pages, 0);
    book->free_ids.resize(pages);
    for (uint32_t i = 0; i < pages; ++i) book->free_ids[i] = static_cast<int32_t>(pages - 1 - i);
    return ZO_OK;
  });
  if (rc == ZO_OK) return book;
  delete book;
  return nullptr;
}

void zo_pages_close(zo_pages* book) { delete book; }

int zo_pages_add(zo_pages* book, uint32_t tokens, uint32_t* seq) {
  if (book == nullptr || seq == nullptr) return ZO_ERR_NULL;
  if (tokens > kMaxTokens) return ZO_ERR_ARG;
  const uint64_t need = book->pages_of(tokens);
  if (need > book->free_ids.size()) return ZO_ERR_FULL;
  return guarded([&] {
    const uint32_t s = book->reserve_seq();
    zo_pages::Seq& q = book->seqs[s];
    q.pages.reserve(need);
    book->free_seqs.pop_back();
    for (uint64_t i = 0; i < need; ++i) q.pages.push_back(book->take());
    q.tokens = tokens;
    *seq = s;
    return ZO_OK;
  });
}

int zo_pages_fork(zo_pages* book, uint32_t seq, uint32_t* forked) {
  if (book == nullptr || forked == nullptr) return ZO_ERR_NULL;
  if (!book->has(seq)) return ZO_ERR_ARG;
  return guarded([&] {
    const uint32_t s = book->reserve_seq();  // may move the entries
    std::vector<int32_t> pages = book->seqs[seq].pages;
    book->free_seqs.pop_back();
    for (int32_t id : pages) ++book->holders[id];
    book->seqs[s].pages.swap(pages);
    book->seqs[s].tokens = book->seqs[seq].tokens;
    *forked = s;
    return ZO_OK;
  });
}

int zo_pages_extend(zo_pages* book, uint32_t seq, uint32_t tokens, zo_page_move* move) {
  if (book == nullptr || move == nullptr) return ZO_ERR_NULL;
  if (!book->has(seq)) return ZO_ERR_ARG;
  zo_pages::Seq& q = book->seqs[seq];
  if (tokens > kMaxTokens - q.tokens) return ZO_ERR_ARG;
  const uint32_t used = static_cast<uint32_t>(q.tokens % book->page_tokens);  // tokens of the last page, 0: it is full
  const bool own = tokens > 0 && used > 0 && book->holders[q.pages.back()] > 1;
  const uint64_t more = book->pages_of(q.tokens + tokens) - q.pages.size();
  if (more + own > book->free_ids.size()) return ZO_ERR_FULL;
  return guarded([&] {
    q.pages.reserve(q.pages.size() + more);
    *move = zo_page_move{0, 0, 0};
    if (own) {
      const int32_t shared = q.pages.back(), mine = book->take();
      book->leave(shared);
      q.pages.back() = mine;
      *move = zo_page_move{shared, mine, static_cast<int32_t>(used)};
    }
    for (uint64_t i = 0; i < more; ++i) q.pages.push_back(book->take());
    q.tokens += tokens;
    return ZO_OK;
  });
}

int zo_pages_cut(zo_pages* book, uint32_t seq, uint32_t tokens) {
  if (book == nullptr) return ZO_ERR_NULL;
  if (!book->has(seq) || tokens > book->seqs[seq].tokens) return ZO_ERR_ARG;
  zo_pages::Seq& q = book->seqs[seq];
  const uint64_t keep = book->pages_of(tokens);
  while (q.pages.size() > keep) {
    book->leave(q.pages.back());
    q.pages.pop_back();
  }
  q.tokens = tokens;
  return ZO_OK;
}

int zo_pages_drop(zo_pages* book, uint32_t seq) {
  if (book == nullptr) return ZO_ERR_NULL;
  if (!book->has(seq)) return ZO_ERR_ARG;
  zo_pages::Seq& q = book->seqs[seq];
  for (int32_t id : q.pages) book->leave(id);
  q.pages.clear();
  q.tokens = -1;
  book->free_seqs.push_back(seq);  // reserved when the number was made
  return ZO_OK;
}

uint32_t zo_pages_left(const zo_pages* book) { return book == nullptr ? 0 : static_cast<uint32_t>(book->free_ids.size()); }

int64_t zo_pages_length(const zo_pages* book, uint32_t seq) {
  return book == nullptr || !book->has(seq) ? -1 : book->seqs[seq].tokens;
}

int zo_pages_table(const zo_pages* book, const uint32_t* seqs, uint32_t n, int32_t* ids, uint64_t stride, uint32_t width,
                   int32_t* lengths) {
  if (book == nullptr) return ZO_ERR_NULL;
  if (n == 0) return ZO_OK;
  if (seqs == nullptr) return ZO_ERR_NULL;
  if (ids != nullptr && n > 1 && stride < width) return ZO_ERR_ARG;
  for (uint32_t i = 0; i < n; ++i)
    if (!book->has(seqs[i]) || (ids != nullptr && book->seqs[seqs[i]].pages.size() > width)) return ZO_ERR_ARG;
  for (uint32_t i = 0; i < n; ++i) {
    const zo_pages::Seq& q = book->seqs[seqs[i]];
    if (ids != nullptr) {
      int32_t* row = ids + static_cast<uint64_t>(i) * stride;
      std::fill(std::copy(q.pages.begin(), q.pages.end(), row), row + width, -1);
    }
    if (lengths != nullptr) lengths[i] = static_cast<int32_t>(q.tokens);
  }
  return ZO_OK;
}

int zo_pages_compact(zo_pages* book, zo_page_move* moves, uint32_t room, uint32_t* n) {
  if (book == nullptr || n == nullptr || (room > 0 && moves == nullptr)) return ZO_ERR_NULL;
  return guarded([&] {
    const uint32_t pages = static_cast<uint32_t>(book->holders.size());
    const uint32_t used = pages - static_cast<uint32_t>(book->free_ids.size());
    // the pages in use at ids >= used, highest first, go into the holes below, lowest first
    std::vector<int32_t> to(pages, -1), rows(pages, 0), left;
    left.reserve(pages);
    uint32_t hole = 0, count = 0;
    for (uint32_t id = pages; id > used && count < room;) {
      --id;
      if (book->holders[id] == 0) continue;
      while (book->holders[hole] != 0 || to[hole] == -2) ++hole;
      to[id] = static_cast<int32_t>(hole);
      to[hole] = -2;  // taken
      ++count;
    }
    // the tokens that a moved page holds: the most that any sequence has in it
    for (const zo_pages::Seq& q : book->seqs)
      for (size_t i = 0; q.tokens >= 0 && i < q.pages.size(); ++i) {
        const int64_t held = std::min<int64_t>(book->page_tokens, q.tokens - static_cast<int64_t>(i) * book->page_tokens);
        rows[q.pages[i]] = std::max(rows[q.pages[i]], static_cast<int32_t>(held));
      }
    uint32_t done = 0;
    for (uint32_t id = pages; id > used && done < count;) {
      --id;
      if (to[id] < 0) continue;
      moves[done++] = zo_page_move{static_cast<int32_t>(id), to[id], rows[id]};
    }
    for (zo_pages::Seq& q : book->seqs)
      for (int32_t& id : q.pages)
        if (to[id] >= 0) id = to[id];
    for (uint32_t i = 0; i < count; ++i) {
      book->holders[moves[i].dst] = book->holders[moves[i].src];
      book->holders[moves[i].src] = 0;
    }
    for (uint32_t id = pages; id > 0; --id)
      if (book->holders[id - 1] == 0) left.push_back(static_cast<int32_t>(id - 1));
    std::copy(left.begin(), left.end(), book->free_ids.begin());  // as many as before, so that its room stays
    *n = count;
    return ZO_OK;
  });
}

}  // extern "C"
