// Host-side argument checks of the decode-step operators. Plain C++ (no HIP), shared by their
// launchers and by the host test that runs this code under AddressSanitizer and UBSan.
#ifndef ZO_CHECKS_H_
#define ZO_CHECKS_H_

#include <cstddef>
#include <cstdint>
#include <vector>

#include "zo_decode.h"
#include "zo_tree.h"

namespace zo {

inline size_t elem_bytes(int32_t dtype) { return dtype == ZO_F32 ? 4 : 2; }

int check_rotate(const zo_rotate& a, bool k_out);
int check_put(const zo_rotate_put& p);
int check_back(const zo_rotate_back& b);
int check_attend(const zo_attend& a);
int check_draw(const zo_draw_args& a);
int check_draw_split(const zo_draw_args& a, const void* work, uint64_t work_bytes);
int check_copy(const zo_cache* shape, void* const* tensors, uint32_t n_tensors, const zo_page_move* moves, uint32_t n_moves, int32_t dtype);
int check_tree(const zo_tree& t);
int check_walk(const zo_tree_walk& w);
int check_moves(const zo_tree_moves& m);
// The same, and the tensors' addresses, each once: where one moved row is the next one's source, moving a tensor twice moves it further.
int check_moves_of(const zo_tree_moves& m, std::vector<int64_t>& tensors);
int check_tree_attend(const zo_tree_attention& a);

// Whether two sets of rows may share an element. Exact for rows of one interleaved buffer: equal strides, each as large as
// what lies below it, or equal token strides and the heads of each side together. Otherwise by the ranges that they span.
bool rows_overlap(const zo_heads& a, uint32_t a_heads, const zo_heads& b, uint32_t b_heads, uint32_t tokens, uint32_t dim,
                  size_t elem);

// Launch shapes of zo_norm_rotate_back: workgroups for each side, and of zo_cache_attend: workers
// (waves) among which the tiles are split.
constexpr uint32_t kBackBlocks = 512;
uint32_t back_blocks(uint32_t tokens, uint32_t heads);
uint64_t attend_items_bytes(uint32_t seqs, uint32_t q_heads, uint32_t heads);  // the parts' whereabouts
uint32_t attend_workers(uint32_t dim);  // at most

// zo_tree_attend: rows (a new token, a query head of a key head's group) of an item, waves that hold them, and workgroups among which the
// tiles are split (at most).
struct TreeShape {
  uint32_t row_waves, rows, workers;
};
TreeShape tree_shape(uint32_t tokens, uint32_t seqs, uint32_t q_heads, uint32_t heads, uint32_t dim, int32_t dtype);
constexpr uint32_t kTreeSplitWords = 8;  // of 4 bytes: where a split item's parts are

// zo_draw_split: tokens of a workgroup's part, and words of 8 bytes that a part and a row keep.
constexpr uint32_t kDrawPart = 4096, kDrawPartWords = 4074, kDrawRowWords = 2;

}  // namespace zo

#endif  // ZO_CHECKS_H_
