// Host code of the decode-step operators under AddressSanitizer and UBSan: the page book against a
// plain model over random calls, its refusals, and the argument checks at the ends of their ranges.

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
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

// Sequences as lists of token values; the pages' contents as the moves and puts leave them.
void random_book(unsigned seed) {
  std::mt19937 rng(seed);
  const uint32_t pages = 1 + rng() % 40, page = 1 + rng() % 5;
  zo_pages* book = zo_pages_open(pages, page);
  REQUIRE(book && zo_pages_left(book) == pages);
  std::vector<std::vector<int>> held(pages, std::vector<int>(page, -1));
  std::map<uint32_t, std::vector<int>> model;
  int next = 0;
  const auto table = [&](uint32_t seq) {
    std::vector<int32_t> ids(pages + 1, 7);
    int32_t length = -9;
    REQUIRE(zo_pages_table(book, &seq, 1, ids.data(), pages, pages, &length) == ZO_OK);
    REQUIRE(ids[pages] == 7 && length == static_cast<int32_t>(model[seq].size()));
    ids.pop_back();
    return ids;
  };
  const auto put = [&](uint32_t seq, uint32_t from) {  // writes tokens from .. end
    const auto ids = table(seq);
    for (uint32_t j = from; j < model[seq].size(); ++j) held[ids[j / page]][j % page] = model[seq][j];
  };
  const auto check = [&] {
    std::set<int32_t> used;
    for (auto& s : model) {
      const auto ids = table(s.first);
      for (uint32_t j = 0; j < s.second.size(); ++j) REQUIRE(held[ids[j / page]][j % page] == s.second[j]);
      for (uint32_t i = 0; i < pages; ++i) {
        REQUIRE((ids[i] >= 0) == (i < (s.second.size() + page - 1) / page));
        if (ids[i] >= 0) used.insert(ids[i]);
      }
      REQUIRE(zo_pages_length(book, s.first) == static_cast<int64_t>(s.second.size()));
    }
    REQUIRE(zo_pages_left(book) == pages - used.size());
  };
  const auto any = [&] {
    auto it = model.begin();
    std::advance(it, rng() % model.size());
    return it->first;
  };
  for (int step = 0; step < 300; ++step) {
    const uint32_t what = rng() % 10, left = zo_pages_left(book);
    uint32_t seq = 0;
    if (what < 2 || model.empty()) {
      const uint32_t n = rng() % (3 * page);
      const int rc = zo_pages_add(book, n, &seq);
      REQUIRE((n + page - 1) / page > left ? rc == ZO_ERR_FULL : rc == ZO_OK);
      if (rc != ZO_OK) continue;
      REQUIRE(model.count(seq) == 0);
      for (uint32_t i = 0; i < n; ++i) model[seq].push_back(next++);
      model[seq];
      put(seq, 0);
    } else if (what < 4) {
      const uint32_t from = any();
      REQUIRE(zo_pages_fork(book, from, &seq) == ZO_OK && model.count(seq) == 0);
      model[seq] = model[from];
    } else if (what < 8) {
      seq = any();
      const uint32_t n = rng() % 4, before = static_cast<uint32_t>(model[seq].size());
      zo_page_move move{-1, -1, -1};
      const int rc = zo_pages_extend(book, seq, n, &move);
      if (rc != ZO_OK) {
        REQUIRE(rc == ZO_ERR_FULL && zo_pages_left(book) == left);
        continue;
      }
      if (move.rows)
        for (int r = 0; r < move.rows; ++r) held[move.dst][r] = held[move.src][r];
      for (uint32_t i = 0; i < n; ++i) model[seq].push_back(next++);
      put(seq, before);
    } else if (what < 9) {
      seq = any();
      REQUIRE(zo_pages_drop(book, seq) == ZO_OK && zo_pages_length(book, seq) == -1);
      REQUIRE(zo_pages_drop(book, seq) == ZO_ERR_ARG);
      model.erase(seq);
    } else {
      const uint32_t room = rng() % 2 ? pages : rng() % 3;
      std::vector<zo_page_move> moves(room + 1, zo_page_move{-5, -5, -5});
      uint32_t n = 99;
      REQUIRE(zo_pages_compact(book, moves.data(), room, &n) == ZO_OK && n <= room && moves[room].src == -5);
      std::set<int32_t> src, dst;
      const auto was = held;
      for (uint32_t i = 0; i < n; ++i) {
        const zo_page_move& m = moves[i];
        REQUIRE(src.insert(m.src).second && dst.insert(m.dst).second && m.rows > 0 && m.rows <= static_cast<int>(page));
        for (int r = 0; r < m.rows; ++r) held[m.dst][r] = was[m.src][r];
        std::fill(held[m.src].begin(), held[m.src].end(), -1);  // nobody may need it
      }
      for (int32_t s : src) REQUIRE(dst.count(s) == 0);
      if (room == pages)
        for (auto& s : model)
          for (int32_t id : table(s.first)) REQUIRE(id < static_cast<int32_t>(pages - zo_pages_left(book)));
      REQUIRE(zo_pages_left(book) == left);
    }
    check();
  }
  zo_pages_close(book);
}

void refusals_of_the_book() {
  REQUIRE(!zo_pages_open(0, 16) && !zo_pages_open(16, 0) && !zo_pages_open(0x80000000u, 16));
  zo_pages_close(nullptr);
  REQUIRE(zo_pages_left(nullptr) == 0 && zo_pages_length(nullptr, 0) == -1);
  zo_pages* book = zo_pages_open(4, 8);
  uint32_t seq = 5, n = 0;
  zo_page_move move;
  int32_t ids[4];
  REQUIRE(zo_pages_add(nullptr, 1, &seq) == ZO_ERR_NULL && zo_pages_add(book, 1, nullptr) == ZO_ERR_NULL);
  REQUIRE(zo_pages_add(book, 0x80000000u, &seq) == ZO_ERR_ARG && zo_pages_add(book, 0x7FFFFFFFu, &seq) == ZO_ERR_FULL);
  REQUIRE(zo_pages_add(book, 33, &seq) == ZO_ERR_FULL && zo_pages_add(book, 32, &seq) == ZO_OK && seq == 0);
  REQUIRE(zo_pages_extend(book, seq, 1, &move) == ZO_ERR_FULL && zo_pages_length(book, seq) == 32);
  REQUIRE(zo_pages_extend(book, seq, 0, &move) == ZO_OK && move.rows == 0);
  REQUIRE(zo_pages_extend(book, seq, 0xFFFFFFFFu, &move) == ZO_ERR_ARG);
  REQUIRE(zo_pages_extend(book, 1, 1, &move) == ZO_ERR_ARG && zo_pages_extend(book, seq, 1, nullptr) == ZO_ERR_NULL);
  REQUIRE(zo_pages_fork(book, 7, &seq) == ZO_ERR_ARG && zo_pages_fork(book, 0, nullptr) == ZO_ERR_NULL);
  const uint32_t seqs[2] = {0, 1};
  REQUIRE(zo_pages_table(book, seqs, 2, ids, 4, 4, nullptr) == ZO_ERR_ARG);
  REQUIRE(zo_pages_table(book, seqs, 1, ids, 3, 3, nullptr) == ZO_ERR_ARG);
  REQUIRE(zo_pages_table(book, nullptr, 1, ids, 4, 4, nullptr) == ZO_ERR_NULL);
  REQUIRE(zo_pages_table(book, seqs, 1, nullptr, 0, 0, ids) == ZO_OK && ids[0] == 32);
  REQUIRE(zo_pages_compact(book, nullptr, 1, &n) == ZO_ERR_NULL && zo_pages_compact(book, nullptr, 0, &n) == ZO_OK && n == 0);
  zo_pages_close(book);
}

void argument_checks() {
  using namespace zo;
  const auto at = [](uintptr_t v) { return reinterpret_cast<void*>(v); };
  // rows of one interleaved buffer share nothing; shifted by one element they do
  const zo_heads q{at(0x10000), 6 * 64, 64}, k{at(0x10000 + 4 * 64 * 2), 6 * 64, 64}, off{at(0x10000 + 4 * 64 * 2 - 2), 6 * 64, 64};
  REQUIRE(!rows_overlap(q, 4, k, 2, 100, 64, 2) && !rows_overlap(k, 2, q, 4, 100, 64, 2));
  REQUIRE(rows_overlap(q, 4, off, 2, 100, 64, 2) && rows_overlap(off, 2, q, 4, 100, 64, 2) && rows_overlap(q, 4, q, 4, 100, 64, 2));
  const zo_heads behind{at(0x10000 + 100 * 6 * 64 * 2), 6 * 64, 64}, other{at(0x10000 + 64), 7 * 64, 64};
  REQUIRE(!rows_overlap(q, 6, behind, 6, 100, 64, 2) && rows_overlap(q, 4, other, 2, 100, 64, 2));

  const double turns[2] = {0.1, 0.01};
  zo_rotate a;
  std::memset(&a, 0, sizeof a);
  a.q = q;
  a.k = k;
  a.q_out = zo_heads{at(0x900000), 4 * 64, 64};
  a.k_out = zo_heads{at(0xA00000), 2 * 64, 64};
  a.positions = static_cast<const int32_t*>(at(0x100));
  a.turns = turns;
  a.tokens = 100;
  a.q_heads = 4;
  a.k_heads = 2;
  a.dim = 64;
  a.rotary = 4;
  a.magnitude = 1.0f;
  a.dtype = ZO_BF16;
  REQUIRE(check_rotate(a, true) == ZO_OK);
  const auto with = [&](auto change) {
    zo_rotate b = a;
    change(b);
    return check_rotate(b, true);
  };
  REQUIRE(with([](zo_rotate& b) { b.q_out = b.q; b.k_out = b.k; }) == ZO_OK);
  REQUIRE(with([](zo_rotate& b) { b.q_out = b.k; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q_out.data = static_cast<char*>(b.q.data) + 2; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.k_out = b.q_out; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q.data = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(with([](zo_rotate& b) { b.k_out.data = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(with([](zo_rotate& b) { b.positions = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(with([](zo_rotate& b) { b.turns = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(with([](zo_rotate& b) { b.turns = nullptr; b.rotary = 0; }) == ZO_OK);
  REQUIRE(with([](zo_rotate& b) { b.rotary = 3; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.rotary = 66; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.dim = 257; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.dim = 0; b.rotary = 0; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.dtype = 2; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.magnitude = INFINITY; }) == ZO_ERR_NONFINITE);
  REQUIRE(with([](zo_rotate& b) { b.norm_eps = NAN; }) == ZO_ERR_NONFINITE);
  REQUIRE(with([](zo_rotate& b) { b.q.token_stride = -64; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q.token_stride = 0; }) == ZO_OK);       // a broadcast input
  REQUIRE(with([](zo_rotate& b) { b.q_out.token_stride = 0; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q_out.head_stride = 32; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q.head_stride = int64_t{1} << 62; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.q.data = static_cast<char*>(b.q.data) + 1; }) == ZO_ERR_ARG);
  REQUIRE(with([](zo_rotate& b) { b.tokens = 0x7FFFFFFF; }) == ZO_ERR_ARG);  // 2^33 rows
  REQUIRE(with([](zo_rotate& b) { b.tokens = 0; b.q.data = nullptr; }) == ZO_OK);
  const double bad[2] = {0.1, INFINITY};
  REQUIRE(with([&](zo_rotate& b) { b.turns = bad; }) == ZO_ERR_NONFINITE);

  zo_cache c{at(0x1000000), at(0x9000000), 8 * 16 * 64, 16 * 64, 64, 100, 8, 16, 64};
  zo_attend t;
  std::memset(&t, 0, sizeof t);
  t.q = zo_heads{at(0x10000), 32 * 64, 64};
  t.out = zo_heads{at(0x90000), 32 * 64, 64};
  t.cache = c;
  t.table = zo_page_table{static_cast<const int32_t*>(at(0x400)), 7, 3, 7};
  t.lengths = static_cast<const int32_t*>(at(0x800));
  t.work = at(0x100000);
  t.work_bytes = zo_cache_attend_work(3, 32, 8, 64);
  t.q_heads = 32;
  t.scale = 0.125f;
  t.dtype = ZO_BF16;
  REQUIRE(check_attend(t) == ZO_OK);
  const auto wit = [&](auto change) {
    zo_attend b = t;
    change(b);
    return check_attend(b);
  };
  REQUIRE(wit([](zo_attend& b) { b.q_heads = 31; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.work_bytes -= 1; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.work = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(wit([](zo_attend& b) { b.out = b.q; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.scale = NAN; }) == ZO_ERR_NONFINITE);
  REQUIRE(wit([](zo_attend& b) { b.cache.pages = 0; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.cache.heads = 0; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.cache.page_tokens = 0; }) == ZO_ERR_ARG);
  REQUIRE(wit([](zo_attend& b) { b.cache.k = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(wit([](zo_attend& b) { b.lengths = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(wit([](zo_attend& b) { b.table.ids = nullptr; }) == ZO_ERR_NULL);
  REQUIRE(wit([](zo_attend& b) { b.table.width = 0; b.table.ids = nullptr; }) == ZO_OK);
  REQUIRE(wit([](zo_attend& b) { b.table.seqs = 0; b.q.data = nullptr; }) == ZO_OK);
  REQUIRE(wit([](zo_attend& b) { b.table.seqs = 0x7FFFFFFF; }) == ZO_ERR_ARG);

  const zo_page_move moves[2] = {{1, 2, 16}, {3, 4, 1}};
  void* tensors[2] = {c.k, c.v};
  REQUIRE(check_copy(&c, tensors, 2, moves, 2, ZO_BF16) == ZO_OK && check_copy(nullptr, nullptr, 0, moves, 2, ZO_BF16) == ZO_OK);
  const auto bad_move = [&](zo_page_move m) {
    const zo_page_move list[2] = {moves[0], m};
    return check_copy(&c, tensors, 2, list, 2, ZO_BF16);
  };
  REQUIRE(bad_move({3, 100, 1}) == ZO_ERR_ARG && bad_move({-1, 5, 1}) == ZO_ERR_ARG && bad_move({3, 5, 17}) == ZO_ERR_ARG);
  REQUIRE(bad_move({3, 5, 0}) == ZO_ERR_ARG && bad_move({3, 2, 1}) == ZO_ERR_ARG && bad_move({3, 1, 1}) == ZO_ERR_ARG);
  REQUIRE(bad_move({2, 5, 1}) == ZO_ERR_ARG && bad_move({5, 5, 1}) == ZO_ERR_ARG && bad_move({1, 5, 3}) == ZO_OK);
  REQUIRE(check_copy(nullptr, tensors, 2, moves, 2, ZO_BF16) == ZO_ERR_NULL && check_copy(&c, nullptr, 2, moves, 2, ZO_BF16) == ZO_ERR_NULL);
  tensors[1] = nullptr;
  REQUIRE(check_copy(&c, tensors, 2, moves, 2, ZO_BF16) == ZO_ERR_NULL);
  tensors[1] = at(0x9000001);
  REQUIRE(check_copy(&c, tensors, 2, moves, 2, ZO_BF16) == ZO_ERR_ARG);
  c.token_stride = 32;  // tokens that overlap
  REQUIRE(check_copy(&c, tensors, 1, moves, 2, ZO_BF16) == ZO_ERR_ARG);
}

int main() {
  for (unsigned seed = 0; seed < 60; ++seed) random_book(seed);
  refusals_of_the_book();
  argument_checks();
  std::printf("decode_check ok\n");
  return 0;
}
