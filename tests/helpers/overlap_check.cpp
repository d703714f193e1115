// Argument checks of the decode-step operators, under AddressSanitizer and UBSan: overlap rules against element-by-element
// counts, the memory that checks take, the addresses of outputs that have no rows.

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <random>
#include <set>
#include <vector>

#include "zo_checks.h"
#include "zo_decode.h"

#define REQUIRE(x)                                            \
  do {                                                        \
    if (!(x)) {                                               \
      std::printf("line %d: %s\n", __LINE__, #x);             \
      std::exit(1);                                           \
    }                                                         \
  } while (0)

namespace {

void* at(int64_t v) { return reinterpret_cast<void*>(static_cast<uintptr_t>(v)); }

std::set<int64_t> elements(const zo_heads& h, uint32_t tokens, uint32_t heads, uint32_t dim) {
  std::set<int64_t> all;
  for (uint32_t t = 0; t < tokens; ++t)
    for (uint32_t g = 0; g < heads; ++g)
      for (uint32_t i = 0; i < dim; ++i)
        all.insert(static_cast<int64_t>(reinterpret_cast<uintptr_t>(h.data)) / 2 + t * h.token_stride + g * h.head_stride + i);
  return all;
}

bool meet(const std::set<int64_t>& a, const std::set<int64_t>& b) {
  for (int64_t e : a)
    if (b.count(e)) return true;
  return false;
}

// Random rows: an overlap is never missed, and none is claimed where two sets have nested strides in common.
void rows() {
  std::mt19937 rng(1);
  const auto below = [&](uint32_t n) { return static_cast<int64_t>(rng() % n); };
  uint32_t exact = 0, apart = 0;
  for (int turn = 0; turn < 60000; ++turn) {
    const uint32_t tokens = 1 + rng() % 4, dim = 1 + rng() % 5, ha = 1 + rng() % 4, hb = 1 + rng() % 4;
    const bool nested = rng() % 2;
    zo_heads a{at(2 * (1000 + below(200))), below(60), below(60)}, b{at(2 * (1000 + below(200))), below(60), below(60)};
    if (nested) {  // heads inside tokens or tokens inside heads, with room between
      const int64_t most = ha > hb ? ha : hb, inner = dim + below(3 * dim);
      if (rng() % 2) {
        a.head_stride = inner;
        a.token_stride = inner * (most - 1) + dim + below(20);
      } else {
        a.token_stride = inner;
        a.head_stride = inner * (tokens - 1) + dim + below(20);
      }
      b.token_stride = a.token_stride;
      b.head_stride = a.head_stride;
      if (tokens == 1 && rng() % 2) b.token_stride = below(60);  // a stride that counts for nothing
      if (hb == 1 && rng() % 2) b.head_stride = below(60);
    }
    const bool truth = meet(elements(a, tokens, ha, dim), elements(b, tokens, hb, dim));
    const bool got = zo::rows_overlap(a, ha, b, hb, tokens, dim, 2);
    REQUIRE(got || !truth);
    REQUIRE(got == zo::rows_overlap(b, hb, a, ha, tokens, dim, 2));
    if (nested) {
      REQUIRE(got == truth);
      ++exact;
      apart += !truth;
    }
  }
  REQUIRE(apart > exact / 10 && apart < exact);
}

// Queries and keys that alternate head by head, rotated in place.
void alternating_heads() {
  const double turns[2] = {0.1, 0.01};
  zo_rotate a;
  std::memset(&a, 0, sizeof a);
  a.q = a.q_out = zo_heads{at(0x10000), 4 * 3 * 64, 3 * 64};
  a.k = a.k_out = zo_heads{at(0x10000 + 2 * 64), 4 * 3 * 64, 3 * 64};
  a.positions = static_cast<const int32_t*>(at(0x100));
  a.turns = turns;
  a.tokens = 100;
  a.q_heads = a.k_heads = 4;
  a.dim = 64;
  a.rotary = 4;
  a.magnitude = 1.0f;
  a.dtype = ZO_BF16;
  REQUIRE(zo::check_rotate(a, true) == ZO_OK);
  a.k.data = a.k_out.data = at(0x10000 + 2 * 63);  // an element too early
  REQUIRE(zo::check_rotate(a, true) == ZO_ERR_ARG);
  // head-major, keys behind the queries of each token
  a.q = a.q_out = zo_heads{at(0x10000), 2 * 64, 100 * 2 * 64};
  a.k = a.k_out = zo_heads{at(0x10000 + 2 * 64), 2 * 64, 100 * 2 * 64};
  REQUIRE(zo::check_rotate(a, true) == ZO_OK);
  // one token, whose stride is anything
  a.tokens = 1;
  a.q.token_stride = a.k.token_stride = a.q_out.token_stride = a.k_out.token_stride = int64_t{1} << 62;
  REQUIRE(zo::check_rotate(a, true) == ZO_OK);
  a.q_heads = a.k_heads = 1;
  a.q.head_stride = a.k.head_stride = a.q_out.head_stride = a.k_out.head_stride = int64_t{1} << 62;
  REQUIRE(zo::check_rotate(a, true) == ZO_OK);
  // as an attention's output beside its queries
  zo_attend t;
  std::memset(&t, 0, sizeof t);
  t.q = zo_heads{at(0x10000), 8 * 2 * 64, 2 * 64};
  t.out = zo_heads{at(0x10000 + 2 * 64), 8 * 2 * 64, 2 * 64};
  t.cache = zo_cache{at(0x1000000), at(0x9000000), 8 * 16 * 64, 16 * 64, 64, 100, 8, 16, 64};
  t.table = zo_page_table{static_cast<const int32_t*>(at(0x400)), 7, 3, 7};
  t.lengths = static_cast<const int32_t*>(at(0x800));
  t.work = at(0x100000);
  t.work_bytes = zo_cache_attend_work(3, 8, 8, 64);
  t.q_heads = 8;
  t.scale = 0.125f;
  t.dtype = ZO_BF16;
  REQUIRE(zo::check_attend(t) == ZO_OK);
  t.out.data = at(0x10000 + 2 * 65 + 2 * 64);
  REQUIRE(zo::check_attend(t) == ZO_ERR_ARG);
}

// A put writes wherever the table says: nothing that it reads or writes besides may lie in the cache.
void put() {
  zo_rotate_put p;
  std::memset(&p, 0, sizeof p);
  p.a.q = p.a.q_out = zo_heads{at(0x10000), 6 * 64, 64};
  p.a.k = zo_heads{at(0x40000), 2 * 64, 64};
  p.v = zo_heads{at(0x50000), 2 * 64, 64};
  p.a.positions = static_cast<const int32_t*>(at(0x100));
  p.a.tokens = 10;
  p.a.q_heads = 6;
  p.a.k_heads = 2;
  p.a.dim = 64;
  p.a.magnitude = 1.0f;
  p.a.dtype = ZO_BF16;
  const int64_t page = 2 * 16 * 64, bytes = 2 * page;
  p.cache = zo_cache{at(0x1000000), at(0x9000000), page, 16 * 64, 64, 100, 2, 16, 64};
  p.table = zo_page_table{static_cast<const int32_t*>(at(0x400)), 7, 10, 7};
  REQUIRE(zo::check_put(p) == ZO_OK);
  const auto with = [&](auto change) {
    zo_rotate_put b = p;
    change(b);
    return zo::check_put(b);
  };
  // keys and values of a page, a layer or a head beside each other; the same or shifted by a row or a page
  REQUIRE(with([&](zo_rotate_put& b) { b.cache.v = at(0x1000000 + bytes); b.cache.page_stride = 2 * page; }) == ZO_OK);
  REQUIRE(with([&](zo_rotate_put& b) { b.cache.v = at(0x1000000 + 100 * bytes); }) == ZO_OK);
  REQUIRE(with([&](zo_rotate_put& b) {
            b.cache = zo_cache{at(0x1000000), at(0x1000000 + 2 * 64), 2 * page, 2 * 64, 2 * 2 * 64, 100, 2, 16, 64};
          }) == ZO_OK);
  for (int64_t shift : {int64_t{0}, int64_t{2 * 64}, int64_t{2}, bytes, 99 * bytes, -bytes})
    REQUIRE(with([&](zo_rotate_put& b) { b.cache.v = at(0x1000000 + shift); }) == ZO_ERR_ARG);
  // tokens of the call in the cache
  for (int64_t in : {int64_t{0x1000000}, 0x1000000 + 99 * bytes, int64_t{0x9000000}, 0x9000000 + 50 * bytes + 2}) {
    REQUIRE(with([&](zo_rotate_put& b) { b.v.data = at(in); }) == ZO_ERR_ARG);
    REQUIRE(with([&](zo_rotate_put& b) { b.a.k.data = at(in); }) == ZO_ERR_ARG);
    REQUIRE(with([&](zo_rotate_put& b) { b.a.q.data = at(in); }) == ZO_ERR_ARG);
    REQUIRE(with([&](zo_rotate_put& b) { b.a.q_out.data = at(in); }) == ZO_ERR_ARG);
    REQUIRE(with([&](zo_rotate_put& b) { b.a.q_out.data = b.a.q.data = at(in); b.a.q_heads = 0; }) == ZO_OK);  // not touched
  }
  const int64_t rows = 10 * 2 * 64 * 2;
  REQUIRE(with([&](zo_rotate_put& b) { b.v.data = at(0x1000000 - rows); }) == ZO_OK);
  REQUIRE(with([&](zo_rotate_put& b) { b.v.data = at(0x1000000 - rows + 2); }) == ZO_ERR_ARG);
  REQUIRE(with([&](zo_rotate_put& b) { b.v.data = at(0x1000000 + 100 * bytes); }) == ZO_OK);
}

// An attention's output is written while other waves read the cache. Its queries may lie in it, and its keys may be its values.
void attend() {
  zo_attend t;
  std::memset(&t, 0, sizeof t);
  t.q = zo_heads{at(0x10000), 8 * 64, 64};
  t.out = zo_heads{at(0x20000), 8 * 64, 64};
  t.cache = zo_cache{at(0x1000000), at(0x9000000), 8 * 16 * 64, 16 * 64, 64, 100, 8, 16, 64};
  t.table = zo_page_table{static_cast<const int32_t*>(at(0x400)), 7, 3, 7};
  t.lengths = static_cast<const int32_t*>(at(0x800));
  t.work = at(0x100000);
  t.work_bytes = zo_cache_attend_work(3, 8, 8, 64);
  t.q_heads = 8;
  t.scale = 0.125f;
  t.dtype = ZO_BF16;
  REQUIRE(zo::check_attend(t) == ZO_OK);
  const int64_t extent = 100 * 8 * 16 * 64 * 2, rows = 3 * 8 * 64 * 2;
  for (int64_t side : {int64_t{0x1000000}, int64_t{0x9000000}}) {
    for (int64_t in : {side, side + extent - 2, side + 2 - rows}) {
      t.out.data = at(in);
      REQUIRE(zo::check_attend(t) == ZO_ERR_ARG);
    }
    for (int64_t beside : {side + extent, side - rows}) {
      t.out.data = at(beside);
      REQUIRE(zo::check_attend(t) == ZO_OK);
    }
  }
  t.q.data = t.cache.v = t.cache.k;
  REQUIRE(zo::check_attend(t) == ZO_OK);
}

std::set<int64_t> elements(const zo_cache& c, int64_t from) {
  std::set<int64_t> all;
  for (uint32_t p = 0; p < c.pages; ++p)
    for (uint32_t h = 0; h < c.heads; ++h)
      for (uint32_t t = 0; t < c.page_tokens; ++t)
        for (uint32_t i = 0; i < c.dim; ++i) all.insert(from / 2 + p * c.page_stride + h * c.head_stride + t * c.token_stride + i);
  return all;
}

// Caches of a copy share nothing, whatever their order; the same one may be given twice.
void copy() {
  const zo_page_move move{0, 1, 1};
  const auto check = [&](const zo_cache& shape, std::vector<int64_t> from) {
    std::vector<void*> tensors;
    for (int64_t f : from) tensors.push_back(at(f));
    return zo::check_copy(&shape, tensors.data(), static_cast<uint32_t>(tensors.size()), &move, 1, ZO_BF16);
  };
  const int64_t head = 16 * 64, page = 8 * head;
  const zo_cache whole{nullptr, nullptr, page, head, 64, 10, 8, 16, 64};
  std::vector<int64_t> layers, inside, pairs;
  zo_cache side = whole, both = whole;
  side.page_stride = 56 * page;
  both.page_stride = 2 * page;
  for (int i = 0; i < 56; ++i) {
    layers.push_back(0x100000 + (55 - i) * 2 * 10 * page);            // [layers, 2, pages, ..], the last first
    inside.push_back(0x100000 + i * 2 * page);                        // [pages, layers, 2, ..]
    pairs.push_back(0x100000 + i / 2 * 2 * 20 * page + i % 2 * 2 * page);  // [layers, pages, 2, ..]
  }
  REQUIRE(check(whole, layers) == ZO_OK && check(side, inside) == ZO_OK && check(both, pairs) == ZO_OK);
  for (auto* list : {&layers, &inside, &pairs}) {
    list->push_back((*list)[3]);  // twice the same
    const zo_cache& shape = list == &layers ? whole : list == &inside ? side : both;
    REQUIRE(check(shape, *list) == ZO_OK);
    list->back() += 2 * 64;       // a token further
    REQUIRE(check(shape, *list) == ZO_ERR_ARG);
  }
  // random shapes and places
  std::mt19937 rng(2);
  const auto below = [&](uint32_t n) { return static_cast<int64_t>(rng() % n); };
  uint32_t meets = 0, apart = 0;
  for (int turn = 0; turn < 20000; ++turn) {
    zo_cache c{nullptr, nullptr, 0, 0, 0, static_cast<uint32_t>(2 + below(3)), static_cast<uint32_t>(1 + below(3)),
               static_cast<uint32_t>(1 + below(3)), static_cast<uint32_t>(1 + below(3))};
    struct {
      int64_t* stride;
      uint32_t n;
    } order[3] = {{&c.page_stride, c.pages}, {&c.head_stride, c.heads}, {&c.token_stride, c.page_tokens}};
    std::shuffle(order, order + 3, rng);
    int64_t extent = c.dim;
    for (auto& o : order) {
      *o.stride = extent * (1 + below(3)) + below(3);
      extent += *o.stride * (static_cast<int64_t>(o.n) - 1);
    }
    std::vector<int64_t> from;
    for (int i = 0, n = 1 + static_cast<int>(below(4)); i < n; ++i) from.push_back(2 * (1000 + below(static_cast<uint32_t>(2 * extent))));
    bool truth = false;
    for (size_t i = 0; i < from.size(); ++i)
      for (size_t j = 0; j < i; ++j) truth = truth || (from[i] != from[j] && meet(elements(c, from[i]), elements(c, from[j])));
    REQUIRE(check(c, from) == (truth ? ZO_ERR_ARG : ZO_OK));
    ++(truth ? meets : apart);
  }
  REQUIRE(meets > 2000 && apart > 2000);
}

// Gamma gradients are written for a side without rows as well, and their addresses are checked there too.
void gradients_of_nothing() {
  zo_rotate_back b;
  std::memset(&b, 0, sizeof b);
  b.a.q_gamma = b.a.k_gamma = at(0x100);
  b.a.positions = static_cast<const int32_t*>(at(0x100));
  b.a.dim = 64;
  b.a.q_heads = 4;
  b.a.dtype = ZO_BF16;
  b.dq_gamma = static_cast<float*>(at(0x1000));
  b.dk_gamma = static_cast<float*>(at(0x2000));
  REQUIRE(zo::check_back(b) == ZO_OK);
  b.dq_gamma = static_cast<float*>(at(0x1002));
  REQUIRE(zo::check_back(b) == ZO_ERR_ARG);
  b.dq_gamma = static_cast<float*>(at(0x1000));
  b.dk_gamma = static_cast<float*>(at(0x2002));
  REQUIRE(zo::check_back(b) == ZO_ERR_ARG);
  b.a.k_gamma = nullptr;  // not written then
  REQUIRE(zo::check_back(b) == ZO_OK);
}

// The largest block asked for since it was set to 0.
size_t largest_block = 0;

// A copy's checks take memory by its moves, not by the pages of the cache, and find what is wrong with them all the same.
void moves() {
  std::mt19937 rng(3);
  const auto check = [](uint32_t pages, const std::vector<zo_page_move>& list) {
    const zo_cache shape{nullptr, nullptr, 64, 64, 8, pages, 1, 8, 8};
    void* tensors[2] = {at(0x100000), at(int64_t{1} << 44)};
    return zo::check_copy(&shape, tensors, 2, list.data(), static_cast<uint32_t>(list.size()), ZO_F32);
  };
  largest_block = 0;
  REQUIRE(check(0x7FFFFFFF, {{0, 0x7FFFFFFE, 8}, {0, 5, 1}}) == ZO_OK && largest_block < 4096);
  for (int turn = 0; turn < 3000; ++turn) {
    const uint32_t pages = turn % 3 ? 20 + rng() % 20 : 50000, n = 1 + rng() % 8, ids = pages < 50000 ? pages : 20;
    std::vector<zo_page_move> list;
    for (uint32_t i = 0; i < n; ++i)
      list.push_back({static_cast<int32_t>((pages - ids) + rng() % ids), static_cast<int32_t>((pages - ids) + rng() % ids), 1});
    bool good = true;
    for (const auto& a : list)
      for (const auto& b : list) good = good && a.dst != b.src && (&a == &b || a.dst != b.dst);
    REQUIRE(check(pages, list) == (good ? ZO_OK : ZO_ERR_ARG));
  }
}

}  // namespace

void* operator new(size_t size) {
  largest_block = std::max(largest_block, size);
  if (void* p = std::malloc(size)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

int main() {
  gradients_of_nothing();
  moves();
  copy();
  attend();
  rows();
  alternating_heads();
  put();
  std::printf("overlap_check ok\n");
  return 0;
}
