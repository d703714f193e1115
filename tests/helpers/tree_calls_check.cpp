// Checks of calls of the operators for several new tokens that are easy to forget, on the host, under AddressSanitizer and UBSan.
// Prints "tree_calls_check ok".
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "zo_checks.h"

namespace {

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      std::exit(1);                               \
    }                                             \
  } while (0)

template <class T>
T* at(uintptr_t address) {
  return reinterpret_cast<T*>(address);
}

// Layers that share a cache: each tensor once, whatever the list's order, and overlapping ones refused as before.
void tensors_listed_twice() {
  void* tensors[6] = {at<void>(0x500000), at<void>(0x100000), at<void>(0x500000), at<void>(0x300000), at<void>(0x100000), at<void>(0x500000)};
  zo_tree_moves m = {};
  m.shape = zo_cache{nullptr, nullptr, 2 * 16 * 64, 16 * 64, 64, 8, 2, 16, 64};
  m.tensors = tensors;
  m.n_tensors = 6;
  m.table = zo_page_table{at<const int32_t>(0x1000), 4, 2, 4};
  m.lengths = m.path = at<const int32_t>(0x2000);
  m.path_stride = 3;
  m.most = 3;
  m.dtype = ZO_F32;
  std::vector<int64_t> each;
  CHECK(zo::check_moves_of(m, each) == ZO_OK && (each == std::vector<int64_t>{0x100000, 0x300000, 0x500000}));
  m.n_tensors = 1;
  CHECK(zo::check_moves_of(m, each) == ZO_OK && each == std::vector<int64_t>{0x500000});
  m.n_tensors = 6;
  tensors[3] = at<void>(0x100000 + 16 * 64 * 4);
  CHECK(zo::check_moves_of(m, each) == ZO_ERR_ARG && zo::check_moves(m) == ZO_ERR_ARG);
}

void words_of_a_walk() {
  zo_tree_walk w = {};
  w.drafted = w.drawn = w.starts = at<const int32_t>(0x1000);
  w.path = w.tokens_out = w.counts = at<int32_t>(0x2000);
  w.tokens = 600;
  w.seqs = 2;
  w.most = 4;
  w.words = ZO_TREE_WORDS;
  CHECK(zo::check_walk(w) == ZO_OK);
  w.words = ZO_TREE_WORDS + 1;
  CHECK(zo::check_walk(w) == ZO_ERR_ARG);
}

}  // namespace

int main() {
  words_of_a_walk();
  tensors_listed_twice();
  std::printf("tree_calls_check ok\n");
}
