// Host code of the operators for several new tokens (argument checks, launch shapes, the page book's cut), for a build under
// AddressSanitizer and UBSan. Prints "tree_check ok".
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "zo_checks.h"

namespace {

#define CHECK(x)                                             \
  do {                                                       \
    if (!(x)) {                                              \
      std::printf("line %d: %s\n", __LINE__, #x);            \
      std::exit(1);                                          \
    }                                                        \
  } while (0)

template <class T>
T* at(uintptr_t address) {
  return reinterpret_cast<T*>(address);
}

zo_cache cache(uint32_t pages, uint32_t heads, uint32_t page, uint32_t dim) {
  return zo_cache{at<void>(0x100000), at<void>(0x900000000), int64_t{heads} * page * dim, int64_t{page} * dim, dim, pages, heads, page, dim};
}

zo_tree_attention attention() {
  zo_tree_attention a = {};
  a.q = zo_heads{at<void>(0x10000000000), 4 * 64, 64};
  a.out = zo_heads{at<void>(0x20000000000), 4 * 64, 64};
  a.cache = cache(8, 2, 16, 64);
  a.table = zo_page_table{at<const int32_t>(0x1000), 4, 2, 4};
  a.lengths = at<const int32_t>(0x2000);
  a.starts = at<const int32_t>(0x3000);
  a.work = at<void>(0x4000);
  a.tokens = 10;
  a.q_heads = 4;
  a.scale = 0.1f;
  a.dtype = ZO_BF16;
  a.work_bytes = zo_tree_attend_work(10, 2, 4, 2, 64, ZO_BF16);
  return a;
}

template <class A, class F>
int with(A a, F change, int (*check)(const A&)) {
  change(a);
  return check(a);
}

void attention_refusals() {
  typedef zo_tree_attention A;
  const auto rc = [](auto change) { return with(attention(), change, &zo::check_tree_attend); };
  CHECK(rc([](A&) {}) == ZO_OK);
  CHECK(rc([](A& a) { a.dtype = 7; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.q_heads = 5; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.heads = 0; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.dim = 0; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.dim = 257; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.pages = 0; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.page_tokens = 0; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.cache.k = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.q.data = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.out.data = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.lengths = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.starts = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.work = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.table.ids = nullptr; }) == ZO_ERR_NULL);
  CHECK(rc([](A& a) { a.work_bytes -= 1; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.work = at<void>(0x4008); }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.lengths = at<const int32_t>(0x2001); }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.starts = at<const int32_t>(0x3002); }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.lse = at<float>(0x3002); }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.scale = std::numeric_limits<float>::infinity(); }) == ZO_ERR_NONFINITE);
  CHECK(rc([](A& a) { a.scale = std::numeric_limits<float>::quiet_NaN(); }) == ZO_ERR_NONFINITE);
  CHECK(rc([](A& a) { a.out = a.q; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.out.data = at<void>(0x100000 + 64); }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.out.head_stride = 32; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.q.token_stride = -1; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.seen = at<const uint64_t>(0x5004); a.words = 1; a.seen_stride = 1; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.seen = at<const uint64_t>(0x5008); a.words = 1; a.seen_stride = -1; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.seen = at<const uint64_t>(0x5008); a.words = (1u << 20) + 1; a.seen_stride = 1; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.seen = at<const uint64_t>(0x5008); a.words = 1; a.seen_stride = 1; }) == ZO_OK);
  CHECK(rc([](A& a) { a.tokens = 1u << 22; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.table.width = 1u << 27; a.table.stride = 1 << 27; }) == ZO_ERR_ARG);
  CHECK(rc([](A& a) { a.tokens = 0; a.q.data = nullptr; a.work = nullptr; }) == ZO_OK);
  CHECK(rc([](A& a) { a.table.seqs = 0; a.work = nullptr; }) == ZO_OK);
}

void other_refusals() {
  zo_tree t = {};
  t.starts = t.lengths = t.parents = at<const int32_t>(0x1000);
  t.seq_of = t.positions = t.places = at<int32_t>(0x2000);
  t.seen = at<uint64_t>(0x3000);
  t.tokens = 5;
  t.seqs = 2;
  t.words = 1;
  const auto lay = [&](auto change) { return with(t, change, &zo::check_tree); };
  CHECK(lay([](zo_tree&) {}) == ZO_OK);
  CHECK(lay([](zo_tree& x) { x.words = ZO_TREE_WORDS; }) == ZO_OK);
  CHECK(lay([](zo_tree& x) { x.words = ZO_TREE_WORDS + 1; }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x.words = 0; }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x.words = 0; x.parents = nullptr; x.seen = nullptr; }) == ZO_OK);
  CHECK(lay([](zo_tree& x) { x.seen = nullptr; }) == ZO_ERR_NULL);
  CHECK(lay([](zo_tree& x) { x.starts = nullptr; }) == ZO_ERR_NULL);
  CHECK(lay([](zo_tree& x) { x.places = nullptr; }) == ZO_ERR_NULL);
  CHECK(lay([](zo_tree& x) { x.seen = at<uint64_t>(0x3004); }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x.parents = at<const int32_t>(0x1002); }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x.tokens = 1u << 24; }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x.seqs = 1u << 24; }) == ZO_ERR_ARG);
  CHECK(lay([](zo_tree& x) { x = zo_tree{}; }) == ZO_OK);

  zo_tree_walk w = {};
  w.drafted = w.drawn = w.starts = at<const int32_t>(0x1000);
  w.path = w.tokens_out = w.counts = at<int32_t>(0x2000);
  w.tokens = 5;
  w.seqs = 2;
  w.most = 4;
  const auto walk = [&](auto change) { return with(w, change, &zo::check_walk); };
  CHECK(walk([](zo_tree_walk&) {}) == ZO_OK);
  CHECK(walk([](zo_tree_walk& x) { x.most = 0; }) == ZO_ERR_ARG);
  CHECK(walk([](zo_tree_walk& x) { x.most = 1u << 23; }) == ZO_ERR_ARG);
  CHECK(walk([](zo_tree_walk& x) { x.drawn = nullptr; }) == ZO_ERR_NULL);
  CHECK(walk([](zo_tree_walk& x) { x.counts = nullptr; }) == ZO_ERR_NULL);
  CHECK(walk([](zo_tree_walk& x) { x.parents = at<const int32_t>(0x1001); }) == ZO_ERR_ARG);
  CHECK(walk([](zo_tree_walk& x) { x.drawn = x.drafted = nullptr; x.tokens = 0; }) == ZO_OK);

  void* tensors[3] = {at<void>(0x100000), at<void>(0x200000), at<void>(0x300000)};
  zo_tree_moves m = {};
  m.shape = cache(8, 2, 16, 64);
  m.tensors = tensors;
  m.n_tensors = 3;
  m.table = zo_page_table{at<const int32_t>(0x1000), 4, 2, 4};
  m.lengths = m.path = at<const int32_t>(0x2000);
  m.path_stride = 3;
  m.most = 3;
  m.dtype = ZO_F32;
  const auto moves = [&](auto change) { return with(m, change, &zo::check_moves); };
  CHECK(moves([](zo_tree_moves&) {}) == ZO_OK);
  CHECK(moves([](zo_tree_moves& x) { x.dtype = 2; }) == ZO_ERR_ARG);
  CHECK(moves([](zo_tree_moves& x) { x.shape.dim = 0; }) == ZO_ERR_ARG);
  CHECK(moves([](zo_tree_moves& x) { x.shape.token_stride = 63; }) == ZO_ERR_ARG);
  CHECK(moves([](zo_tree_moves& x) { x.path_stride = -1; }) == ZO_ERR_ARG);
  CHECK(moves([](zo_tree_moves& x) { x.path = nullptr; }) == ZO_ERR_NULL);
  CHECK(moves([](zo_tree_moves& x) { x.tensors = nullptr; }) == ZO_ERR_NULL);
  CHECK(moves([](zo_tree_moves& x) { x.table.seqs = 1u << 17; }) == ZO_ERR_ARG);
  CHECK(moves([](zo_tree_moves& x) { x.n_tensors = 0; x.tensors = nullptr; }) == ZO_OK);
  void* close[2] = {at<void>(0x100000), at<void>(0x100000 + 16 * 64 * 4)};
  CHECK(moves([&](zo_tree_moves& x) { x.tensors = close; x.n_tensors = 2; }) == ZO_ERR_ARG);
  void* none[2] = {at<void>(0x100000), nullptr};
  CHECK(moves([&](zo_tree_moves& x) { x.tensors = none; x.n_tensors = 2; }) == ZO_ERR_NULL);
}

// The workspace holds an entry and two parts of all rows for each workgroup.
void workspace() {
  std::mt19937 rng(1);
  for (int round = 0; round < 20000; ++round) {
    const uint32_t seqs = 1 + rng() % 9, heads = 1 + rng() % 4, group = 1 + rng() % 20, tokens = 1 + rng() % (rng() % 3 ? 20 : 500);
    const uint32_t dim = 1 + rng() % ZO_DIM_MAX;
    const int32_t dtype = rng() % 2 ? ZO_BF16 : ZO_F32;
    const zo::TreeShape s = zo::tree_shape(tokens, seqs, heads * group, heads, dim, dtype);
    CHECK(s.rows == 32 * s.row_waves && s.workers > 0 && s.workers % 8 == 0);
    const uint64_t row = (dim + 3) / 4 * 4 + 4;
    CHECK(zo_tree_attend_work(tokens, seqs, heads * group, heads, dim, dtype) ==
          16 + s.workers * (zo::kTreeSplitWords * 4 + 2 * uint64_t{s.rows} * row * 4));
  }
  CHECK(zo_tree_attend_work(1, 1, 3, 2, 64, ZO_F32) == 16 && zo_tree_attend_work(1, 1, 2, 2, 257, ZO_F32) == 0);
}

// Random extensions and cuts of sequences that share pages, against a plain model: which tokens a sequence has, and who holds a page.
void cuts() {
  std::mt19937 rng(2);
  for (int round = 0; round < 200; ++round) {
    const uint32_t pages = 4 + rng() % 40, page = 1 + rng() % 5;
    zo_pages* book = zo_pages_open(pages, page);
    std::vector<uint32_t> seqs;
    const auto holders = [&] {
      std::vector<int> held(pages, 0);
      for (uint32_t s : seqs) {
        const int64_t n = zo_pages_length(book, s);
        const uint32_t width = static_cast<uint32_t>((n + page - 1) / page) + 1;
        std::vector<int32_t> ids(width);
        CHECK(zo_pages_table(book, &s, 1, ids.data(), width, width, nullptr) == ZO_OK);
        for (uint32_t i = 0; i + 1 < width; ++i) {
          CHECK(ids[i] >= 0 && static_cast<uint32_t>(ids[i]) < pages);
          ++held[ids[i]];
        }
        CHECK(ids[width - 1] == -1);
      }
      return held;
    };
    for (int step = 0; step < 100; ++step) {
      uint32_t s = 0;
      zo_page_move move;
      switch (rng() % 5) {
        case 0:
          if (zo_pages_add(book, rng() % (2 * page), &s) == ZO_OK) seqs.push_back(s);
          break;
        case 1:
          if (!seqs.empty() && zo_pages_fork(book, seqs[rng() % seqs.size()], &s) == ZO_OK) seqs.push_back(s);
          break;
        case 2:
          if (!seqs.empty()) zo_pages_extend(book, seqs[rng() % seqs.size()], rng() % (3 * page), &move);
          break;
        default:
          if (seqs.empty()) break;
          s = seqs[rng() % seqs.size()];
          const int64_t n = zo_pages_length(book, s);
          CHECK(zo_pages_cut(book, s, static_cast<uint32_t>(n) + 1) == ZO_ERR_ARG && zo_pages_length(book, s) == n);
          const uint32_t keep = static_cast<uint32_t>(rng() % (n + 1));
          CHECK(zo_pages_cut(book, s, keep) == ZO_OK && zo_pages_length(book, s) == keep);
      }
      uint32_t used = 0;
      for (int h : holders()) used += h > 0;
      CHECK(zo_pages_left(book) == pages - used);
    }
    for (uint32_t s : seqs) CHECK(zo_pages_drop(book, s) == ZO_OK);
    CHECK(zo_pages_left(book) == pages && zo_pages_cut(book, 0, 0) == ZO_ERR_ARG);
    zo_pages_close(book);
  }
  CHECK(zo_pages_cut(nullptr, 0, 0) == ZO_ERR_NULL);
}

}  // namespace

int main() {
  attention_refusals();
  other_refusals();
  workspace();
  cuts();
  std::printf("tree_check ok\n");
}
