// Host-only part of the decode-step operators: argument checks, workspace sizes and rotation
// frequencies. Nothing here throws: the one container (the page lists of zo_cache_copy) is
// allocated under a try block.

#include "zo_checks.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace zo {

namespace {

constexpr int64_t kMaxElems = int64_t{1} << 46;  // extents of a tensor: far above any memory, far below overflow

bool dtype_ok(int32_t dtype) { return dtype == ZO_F32 || dtype == ZO_BF16; }

bool aligned(const void* p, size_t elem) { return reinterpret_cast<uintptr_t>(p) % elem == 0; }

// Strides of an axis of n entries: not negative, and the axis ends below kMaxElems.
bool axis_ok(int64_t stride, uint64_t n) {
  return stride >= 0 && (n <= 1 || stride <= kMaxElems / static_cast<int64_t>(n));
}

struct Axis {
  int64_t stride;
  uint64_t n;
};

// Whether distinct indices of the axes (runs of `run` elements innermost) never share an element.
bool distinct(Axis* axes, int count, int64_t run) {
  std::sort(axes, axes + count, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  int64_t extent = run;
  for (int i = 0; i < count; ++i) {
    if (axes[i].n <= 1) continue;
    if (axes[i].stride < extent) return false;
    extent += axes[i].stride * static_cast<int64_t>(axes[i].n - 1);
  }
  return true;
}

// Places of runs: `count` axes, largest stride first, none with a stride of 0, over runs of reach[count] bytes; reach[k] bytes
// lie from an index of the axes from k on to the end of its last run.
struct Places {
  Axis axes[3];
  int64_t reach[4];
  int count = 0;

  void add(int64_t stride, uint64_t n) {
    if (n > 1 && stride > 0) axes[count++] = Axis{stride, n};
  }
  // false: strides so small beside what lies below them that meets() would have to look at many indices.
  bool close(int64_t run) {
    std::sort(axes, axes + count, [](const Axis& a, const Axis& b) { return a.stride > b.stride; });
    reach[count] = run;
    bool few = true;
    for (int k = count - 1; k >= 0; --k) {
      few = few && reach[k + 1] <= 2 * axes[k].stride;
      reach[k] = reach[k + 1] + axes[k].stride * static_cast<int64_t>(axes[k].n - 1);
    }
    return few;
  }
  // Whether the bytes [x, x + size) meet a run, x counted from the first run's.
  bool meets(int64_t x, int64_t size, int k = 0) const {
    if (x >= reach[k] || x + size <= 0) return false;
    if (k == count || (x <= 0 && x + size >= reach[k])) return true;
    const int64_t stride = axes[k].stride, n = static_cast<int64_t>(axes[k].n);
    int64_t i = x < reach[k + 1] ? 0 : (x - reach[k + 1]) / stride + 1;  // the first that ends behind x
    for (; i < n && i * stride < x + size; ++i)
      if (meets(x - i * stride, size, k + 1)) return true;
    return false;
  }
};

// Two tensors of the same strides (bytes; of an axis that one has a single entry of, the other's), the second `gap` bytes behind the
// first: whether two of their runs meet, exact where the strides are nested.
struct Both {
  int64_t stride;
  uint64_t n, m;
};
bool same_strides_meet(const Both* axes, int count, int64_t gap, int64_t run) {
  Places steps;  // differences of two indices, as steps from the lowest
  int64_t lowest = gap;
  for (int i = 0; i < count; ++i) {
    if (axes[i].n == 0 || axes[i].m == 0) return false;
    lowest -= axes[i].stride * static_cast<int64_t>(axes[i].n - 1);
    steps.add(axes[i].stride, axes[i].n + axes[i].m - 1);
  }
  return !steps.close(1) || steps.meets(1 - run - lowest, 2 * run - 1);
}

int check_rows(const zo_heads& h, uint32_t tokens, uint32_t heads, uint32_t dim, size_t elem, bool written) {
  if (h.data == nullptr) return ZO_ERR_NULL;
  if (!aligned(h.data, elem) || !axis_ok(h.token_stride, tokens) || !axis_ok(h.head_stride, heads)) return ZO_ERR_ARG;
  if (written) {
    Axis axes[2] = {{h.token_stride, tokens}, {h.head_stride, heads}};
    if (!distinct(axes, 2, dim)) return ZO_ERR_ARG;
  }
  return ZO_OK;
}

bool same_rows(const zo_heads& a, const zo_heads& b, uint32_t tokens, uint32_t heads) {
  return a.data == b.data && (tokens <= 1 || a.token_stride == b.token_stride) &&
         (heads <= 1 || a.head_stride == b.head_stride);
}

int check_cache(const zo_cache& c, size_t elem, bool written) {
  if (c.pages == 0 || c.heads == 0 || c.page_tokens == 0 || c.dim == 0 || c.dim > ZO_DIM_MAX) return ZO_ERR_ARG;
  if (c.pages > 0x7FFFFFFFu || c.page_tokens > 0x7FFFFFFFu) return ZO_ERR_ARG;
  if (c.k == nullptr || c.v == nullptr) return ZO_ERR_NULL;
  if (!aligned(c.k, elem) || !aligned(c.v, elem)) return ZO_ERR_ARG;
  if (!axis_ok(c.page_stride, c.pages) || !axis_ok(c.head_stride, c.heads) || !axis_ok(c.token_stride, c.page_tokens))
    return ZO_ERR_ARG;
  if (written) {
    Axis axes[3] = {{c.page_stride, c.pages}, {c.head_stride, c.heads}, {c.token_stride, c.page_tokens}};
    if (!distinct(axes, 3, c.dim)) return ZO_ERR_ARG;
  }
  return ZO_OK;
}

int64_t address(const void* p) { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(p)); }

// Whether the keys and the values of a cache that is written (its strides are nested) share an element.
bool sides_overlap(const zo_cache& c, size_t elem) {
  const int64_t size = static_cast<int64_t>(elem);
  const auto axis = [&](int64_t stride, uint32_t n) { return Both{n > 1 ? stride * size : 0, n, n}; };
  const Both axes[3] = {axis(c.page_stride, c.pages), axis(c.head_stride, c.heads), axis(c.token_stride, c.page_tokens)};
  return same_strides_meet(axes, 3, address(c.v) - address(c.k), c.dim * size);
}

// Whether two tensors of a list, all of the (nested) shape of `c`, share elements. The same tensor twice does not count: its moves
// are the same. Sorted by address; layers one behind another, or side by side inside a page's stride, need no pairs.
bool tensors_overlap(const zo_cache& c, void* const* tensors, uint32_t n, size_t elem) {
  const int64_t size = static_cast<int64_t>(elem), run = c.dim * size;
  Places all;
  const auto stride = [&](int64_t s, uint32_t count) { return count > 1 ? s * size : 0; };
  const Both axes[3] = {{stride(c.page_stride, c.pages), c.pages, c.pages},
                        {stride(c.head_stride, c.heads), c.heads, c.heads},
                        {stride(c.token_stride, c.page_tokens), c.page_tokens, c.page_tokens}};
  for (const Both& a : axes) all.add(a.stride, a.n);
  all.close(run);
  std::vector<int64_t> at(n);
  for (uint32_t i = 0; i < n; ++i) at[i] = address(tensors[i]);
  std::sort(at.begin(), at.end());
  at.erase(std::unique(at.begin(), at.end()), at.end());
  int64_t least = all.reach[0];
  for (size_t i = 1; i < at.size(); ++i) least = std::min(least, at[i] - at[i - 1]);
  if (least >= all.reach[0]) return false;
  if (all.count > 0 && least >= all.reach[1] && at.back() - at.front() + all.reach[1] <= all.axes[0].stride) return false;
  for (size_t i = 0; i < at.size(); ++i)
    for (size_t j = i + 1; j < at.size() && at[j] < at[i] + all.reach[0]; ++j)
      if (same_strides_meet(axes, 3, at[j] - at[i], run)) return true;
  return false;
}

// Whether no dst of the moves is repeated or a src. A byte for each page, or, where a cache has very many for each move, the
// sorted dsts: 32 moves in 2^20 pages 1 us (a byte for each page 22), 1,024 moves in 65,536 pages 52 us (a byte for each 4).
bool moves_apart(const zo_page_move* moves, uint32_t n, uint32_t pages) {
  if (pages / 2048 <= n) {
    std::vector<unsigned char> seen(pages, 0);  // bit 0: a destination, bit 1: a source
    for (uint32_t i = 0; i < n; ++i) {
      if (seen[moves[i].dst] != 0 || (seen[moves[i].src] & 1) != 0 || moves[i].src == moves[i].dst) return false;
      seen[moves[i].dst] |= 1;
      seen[moves[i].src] |= 2;
    }
    return true;
  }
  std::vector<int32_t> to(n);
  for (uint32_t i = 0; i < n; ++i) to[i] = moves[i].dst;
  std::sort(to.begin(), to.end());
  if (std::adjacent_find(to.begin(), to.end()) != to.end()) return false;
  return std::none_of(moves, moves + n, [&](const zo_page_move& m) { return std::binary_search(to.begin(), to.end(), m.src); });
}

// Whether rows and a cache may share an element, by the ranges that they span.
bool cache_overlaps(const zo_cache& c, const zo_heads& h, uint32_t tokens, uint32_t heads, size_t elem) {
  if (tokens == 0 || heads == 0) return false;
  const auto span = [&](int64_t stride, uint32_t n) { return n > 1 ? stride * (static_cast<int64_t>(n) - 1) : 0; };
  const int64_t size = static_cast<int64_t>(elem), lo = address(h.data);
  const int64_t hi = lo + (span(h.token_stride, tokens) + span(h.head_stride, heads) + c.dim) * size;
  const int64_t extent = (span(c.page_stride, c.pages) + span(c.head_stride, c.heads) + span(c.token_stride, c.page_tokens) + c.dim) * size;
  const auto meets = [&](const void* side) { return lo < address(side) + extent && address(side) < hi; };
  return meets(c.k) || meets(c.v);
}

int check_table(const zo_page_table& t) {
  if (t.seqs == 0 || t.width == 0) return ZO_OK;
  if (t.ids == nullptr) return ZO_ERR_NULL;
  return aligned(t.ids, 4) && axis_ok(t.stride, t.seqs) ? ZO_OK : ZO_ERR_ARG;
}

#define ZO_TRY(x)                  \
  do {                             \
    const int rc_ = (x);           \
    if (rc_ != ZO_OK) return rc_;  \
  } while (0)

// What the forward, the putting and the backward call have in common; `a` only describes where
// rows are not passed.
int check_common(const zo_rotate& a) {
  if (!dtype_ok(a.dtype) || a.dim == 0 || a.dim > ZO_DIM_MAX) return ZO_ERR_ARG;
  if (a.rotary % 2 != 0 || a.rotary > a.dim) return ZO_ERR_ARG;
  if (a.tokens > 0x7FFFFFFFu || a.q_heads > 0xFFFFu || a.k_heads > 0xFFFFu) return ZO_ERR_ARG;
  // rows of a side are numbered in 32 bits, with room for a workgroup's rows behind the last
  if (static_cast<uint64_t>(a.tokens) * std::max(a.q_heads, a.k_heads) > 0xFFFF0000ull) return ZO_ERR_ARG;
  if (a.rotary > 0) {
    if (a.turns == nullptr) return ZO_ERR_NULL;
    for (uint32_t i = 0; i < a.rotary / 2; ++i)
      if (!std::isfinite(a.turns[i])) return ZO_ERR_NONFINITE;
  }
  if (!std::isfinite(a.norm_eps) || !std::isfinite(a.magnitude)) return ZO_ERR_NONFINITE;
  const size_t elem = elem_bytes(a.dtype);
  if (!aligned(a.q_gamma, elem) || !aligned(a.k_gamma, elem) || !aligned(a.positions, 4)) return ZO_ERR_ARG;
  if (a.tokens > 0 && a.q_heads + a.k_heads > 0 && a.positions == nullptr) return ZO_ERR_NULL;
  return ZO_OK;
}

// An output against an input: the same rows, or no element shared.
int check_apart(const zo_heads& out, uint32_t out_heads, const zo_heads& in, uint32_t in_heads, bool may_be_same,
                uint32_t tokens, uint32_t dim, size_t elem) {
  if (out_heads == 0 || in_heads == 0 || out.data == nullptr || in.data == nullptr) return ZO_OK;
  if (may_be_same && out_heads == in_heads && same_rows(out, in, tokens, out_heads)) return ZO_OK;
  return rows_overlap(out, out_heads, in, in_heads, tokens, dim, elem) ? ZO_ERR_ARG : ZO_OK;
}

}  // namespace

bool rows_overlap(const zo_heads& a, uint32_t a_heads, const zo_heads& b, uint32_t b_heads, uint32_t tokens, uint32_t dim,
                  size_t elem) {
  const int64_t size = static_cast<int64_t>(elem);
  const auto lo = [](const zo_heads& h) { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(h.data)); };
  const auto span = [&](const zo_heads& h, uint32_t heads) {  // bytes of one token's heads
    return (h.head_stride * (static_cast<int64_t>(heads) - 1) + dim) * size;
  };
  const auto end = [&](const zo_heads& h, uint32_t heads) {
    return lo(h) + h.token_stride * (static_cast<int64_t>(tokens) - 1) * size + span(h, heads);
  };
  if (end(a, a_heads) <= lo(b) || end(b, b_heads) <= lo(a)) return false;
  const int64_t pitch = tokens > 1 ? a.token_stride * size : 0;  // (the stride of a single token is anything)
  if (a.token_stride == b.token_stride && pitch > 0 && span(a, a_heads) <= pitch && span(b, b_heads) <= pitch) {
    const int64_t gap = (((lo(b) - lo(a)) % pitch) + pitch) % pitch;  // b's token behind a's
    if (gap >= span(a, a_heads) && gap + span(b, b_heads) <= pitch) return false;
  }
  const bool same = (tokens <= 1 || a.token_stride == b.token_stride) && (a_heads <= 1 || b_heads <= 1 || a.head_stride == b.head_stride);
  if (!same) return true;
  const int64_t head = a_heads > 1 ? a.head_stride : b_heads > 1 ? b.head_stride : 0;
  const Both axes[2] = {{pitch, tokens, tokens}, {head * size, a_heads, b_heads}};
  return same_strides_meet(axes, 2, lo(b) - lo(a), dim * size);
}

int check_rotate(const zo_rotate& a, bool k_out) {
  ZO_TRY(check_common(a));
  if (a.tokens == 0) return ZO_OK;
  const size_t elem = elem_bytes(a.dtype);
  if (a.q_heads > 0) {
    ZO_TRY(check_rows(a.q, a.tokens, a.q_heads, a.dim, elem, false));
    ZO_TRY(check_rows(a.q_out, a.tokens, a.q_heads, a.dim, elem, true));
  }
  if (a.k_heads > 0) ZO_TRY(check_rows(a.k, a.tokens, a.k_heads, a.dim, elem, false));
  if (a.k_heads > 0 && k_out) ZO_TRY(check_rows(a.k_out, a.tokens, a.k_heads, a.dim, elem, true));
  const uint32_t out_k = k_out ? a.k_heads : 0;
  ZO_TRY(check_apart(a.q_out, a.q_heads, a.q, a.q_heads, true, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(a.q_out, a.q_heads, a.k, a.k_heads, false, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(a.k_out, out_k, a.k, a.k_heads, true, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(a.k_out, out_k, a.q, a.q_heads, false, a.tokens, a.dim, elem));
  return check_apart(a.q_out, a.q_heads, a.k_out, out_k, false, a.tokens, a.dim, elem);
}

int check_put(const zo_rotate_put& p) {
  ZO_TRY(check_rotate(p.a, false));
  if (p.a.tokens == 0) return ZO_OK;
  const size_t elem = elem_bytes(p.a.dtype);
  if (!aligned(p.seqs, 4)) return ZO_ERR_ARG;
  if (p.a.k_heads == 0) return ZO_OK;
  ZO_TRY(check_rows(p.v, p.a.tokens, p.a.k_heads, p.a.dim, elem, false));
  ZO_TRY(check_cache(p.cache, elem, true));
  if (p.cache.heads != p.a.k_heads || p.cache.dim != p.a.dim) return ZO_ERR_ARG;
  ZO_TRY(check_table(p.table));
  // where the rows go is known on the device alone: nothing else of the call may lie in the cache
  if (sides_overlap(p.cache, elem) || cache_overlaps(p.cache, p.a.q, p.a.tokens, p.a.q_heads, elem) ||
      cache_overlaps(p.cache, p.a.q_out, p.a.tokens, p.a.q_heads, elem) || cache_overlaps(p.cache, p.a.k, p.a.tokens, p.a.k_heads, elem) ||
      cache_overlaps(p.cache, p.v, p.a.tokens, p.a.k_heads, elem))
    return ZO_ERR_ARG;
  return check_apart(p.a.q_out, p.a.q_heads, p.v, p.a.k_heads, false, p.a.tokens, p.a.dim, elem);
}

uint32_t back_blocks(uint32_t tokens, uint32_t heads) {
  const uint64_t rows = static_cast<uint64_t>(tokens) * heads;
  return static_cast<uint32_t>(std::min<uint64_t>(kBackBlocks, (rows + 31) / 32));
}

int check_back(const zo_rotate_back& b) {
  const zo_rotate& a = b.a;
  ZO_TRY(check_common(a));
  // gamma gradients of a side without rows are written too: zeros
  if ((a.q_gamma && !aligned(b.dq_gamma, 4)) || (a.k_gamma && !aligned(b.dk_gamma, 4))) return ZO_ERR_ARG;
  if (a.tokens == 0) return ZO_OK;
  const size_t elem = elem_bytes(a.dtype);
  const auto side = [&](const zo_heads& x, const zo_heads& dy, const zo_heads& dx, uint32_t heads, const void* gamma,
                        const float* dgamma) -> int {
    if (heads == 0) return ZO_OK;
    ZO_TRY(check_rows(dy, a.tokens, heads, a.dim, elem, false));
    ZO_TRY(check_rows(dx, a.tokens, heads, a.dim, elem, true));
    ZO_TRY(check_apart(dx, heads, dy, heads, true, a.tokens, a.dim, elem));
    if (gamma == nullptr) return ZO_OK;
    ZO_TRY(check_rows(x, a.tokens, heads, a.dim, elem, false));
    ZO_TRY(check_apart(dx, heads, x, heads, true, a.tokens, a.dim, elem));
    return dgamma == nullptr || b.work == nullptr ? ZO_ERR_NULL : ZO_OK;
  };
  ZO_TRY(side(a.q, a.q_out, b.dq, a.q_heads, a.q_gamma, b.dq_gamma));
  ZO_TRY(side(a.k, a.k_out, b.dk, a.k_heads, a.k_gamma, b.dk_gamma));
  // one side's gradients against the other side's inputs and outputs
  const uint32_t xq = a.q_gamma ? a.q_heads : 0, xk = a.k_gamma ? a.k_heads : 0;
  ZO_TRY(check_apart(b.dq, a.q_heads, a.k_out, a.k_heads, false, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(b.dq, a.q_heads, a.k, xk, false, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(b.dk, a.k_heads, a.q_out, a.q_heads, false, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(b.dk, a.k_heads, a.q, xq, false, a.tokens, a.dim, elem));
  ZO_TRY(check_apart(b.dq, a.q_heads, b.dk, a.k_heads, false, a.tokens, a.dim, elem));
  if (xq + xk > 0) {
    if (!aligned(b.work, 16)) return ZO_ERR_ARG;
    if (b.work_bytes < zo_norm_rotate_back_work(a.tokens, a.q_heads, a.k_heads, a.dim)) return ZO_ERR_ARG;
  }
  return ZO_OK;
}

// 16 bytes for each item: a sequence, a key head, up to 16 of its query heads.
uint64_t attend_items_bytes(uint32_t seqs, uint32_t q_heads, uint32_t heads) {
  return static_cast<uint64_t>(seqs) * heads * ((q_heads / heads + 15) / 16) * 16;
}

uint32_t attend_workers(uint32_t dim) { return 1024 * (dim > 128 ? 2 : dim > 64 ? 3 : 4); }

int check_attend(const zo_attend& a) {
  if (!dtype_ok(a.dtype)) return ZO_ERR_ARG;
  const size_t elem = elem_bytes(a.dtype);
  if (a.cache.heads == 0 || a.cache.heads > 0xFFFFu || a.q_heads > 0xFFFFu || a.q_heads % a.cache.heads != 0) return ZO_ERR_ARG;
  // a workgroup for each item, 2^32 threads at most in a launch
  if (static_cast<uint64_t>(a.table.seqs) * std::max(a.q_heads, 1u) >= (1u << 24)) return ZO_ERR_ARG;
  if (!std::isfinite(a.scale)) return ZO_ERR_NONFINITE;
  if (a.table.seqs == 0 || a.q_heads == 0) return ZO_OK;
  ZO_TRY(check_cache(a.cache, elem, false));
  ZO_TRY(check_table(a.table));
  ZO_TRY(check_rows(a.q, a.table.seqs, a.q_heads, a.cache.dim, elem, false));
  ZO_TRY(check_rows(a.out, a.table.seqs, a.q_heads, a.cache.dim, elem, true));
  // a worker writes a head's output while others still read their queries and the cache
  ZO_TRY(check_apart(a.out, a.q_heads, a.q, a.q_heads, false, a.table.seqs, a.cache.dim, elem));
  if (cache_overlaps(a.cache, a.out, a.table.seqs, a.q_heads, elem)) return ZO_ERR_ARG;
  // tiles of 16 tokens are numbered below 2^52 (a token that no memory of its own holds may count many times)
  if (static_cast<uint64_t>(a.table.width) * a.cache.page_tokens / 16 >= (1ull << 52) / (static_cast<uint64_t>(a.table.seqs) * a.q_heads))
    return ZO_ERR_ARG;
  if (a.lengths == nullptr || a.work == nullptr) return ZO_ERR_NULL;
  if (!aligned(a.lengths, 4) || !aligned(a.lse, 4) || !aligned(a.work, 16)) return ZO_ERR_ARG;
  if (a.work_bytes < zo_cache_attend_work(a.table.seqs, a.q_heads, a.cache.heads, a.cache.dim)) return ZO_ERR_ARG;
  return ZO_OK;
}

int check_draw(const zo_draw_args& a) {
  if (!dtype_ok(a.dtype) || a.vocab == 0 || a.vocab > (1u << 18) || !axis_ok(a.row_stride, a.rows)) return ZO_ERR_ARG;
  if (a.rows == 0) return ZO_OK;
  if (a.rows >= (1u << 22)) return ZO_ERR_ARG;  // 2^32 threads at most in a launch
  if (a.logits == nullptr || a.u == nullptr || a.tokens == nullptr) return ZO_ERR_NULL;
  if (!aligned(a.logits, elem_bytes(a.dtype)) || !aligned(a.u, 4) || !aligned(a.temperature, 4) || !aligned(a.top_k, 4) ||
      !aligned(a.top_p, 4) || !aligned(a.min_p, 4) || !aligned(a.tokens, 4) || !aligned(a.logprobs, 4))
    return ZO_ERR_ARG;
  return ZO_OK;
}

int check_draw_split(const zo_draw_args& a, const void* work, uint64_t work_bytes) {
  ZO_TRY(check_draw(a));
  const uint64_t bytes = zo_draw_work(a.rows, a.vocab, a.top_k != nullptr);
  if (bytes == 0) return ZO_OK;
  if (work == nullptr) return ZO_ERR_NULL;
  return aligned(work, 16) && work_bytes >= bytes ? ZO_OK : ZO_ERR_ARG;
}

int check_copy(const zo_cache* shape, void* const* tensors, uint32_t n_tensors, const zo_page_move* moves, uint32_t n_moves, int32_t dtype) {
  if (!dtype_ok(dtype)) return ZO_ERR_ARG;
  if (n_tensors == 0 || n_moves == 0) return ZO_OK;
  if (shape == nullptr || tensors == nullptr || moves == nullptr) return ZO_ERR_NULL;
  zo_cache first = *shape;
  first.k = first.v = tensors[0];
  const size_t elem = elem_bytes(dtype);
  ZO_TRY(check_cache(first, elem, true));
  // 2^32 threads at most in a launch
  if (first.heads > 0xFFFFu || static_cast<uint64_t>(first.page_tokens) * first.dim * first.heads > (1ull << 23)) return ZO_ERR_ARG;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    if (tensors[i] == nullptr) return ZO_ERR_NULL;
    if (!aligned(tensors[i], elem)) return ZO_ERR_ARG;
  }
  try {
    if (tensors_overlap(first, tensors, n_tensors, elem)) return ZO_ERR_ARG;
    for (uint32_t i = 0; i < n_moves; ++i) {
      const zo_page_move& m = moves[i];
      if (m.src < 0 || m.dst < 0 || static_cast<uint32_t>(m.src) >= first.pages || static_cast<uint32_t>(m.dst) >= first.pages)
        return ZO_ERR_ARG;
      if (m.rows <= 0 || static_cast<uint32_t>(m.rows) > first.page_tokens) return ZO_ERR_ARG;
    }
    return moves_apart(moves, n_moves, first.pages) ? ZO_OK : ZO_ERR_ARG;
  } catch (const std::bad_alloc&) {
    return ZO_ERR_MEMORY;
  }
}

}  // namespace zo

extern "C" {

uint64_t zo_norm_rotate_back_work(uint32_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t dim) {
  return (static_cast<uint64_t>(zo::back_blocks(tokens, q_heads)) + zo::back_blocks(tokens, k_heads)) * dim * sizeof(float);
}

// Each worker keeps at most two parts (of the items that its range begins and ends in): for every
// query head of an item a maximum, a sum and a row of fp32.
uint64_t zo_cache_attend_work(uint32_t seqs, uint32_t q_heads, uint32_t heads, uint32_t dim) {
  if (heads == 0 || q_heads % heads != 0 || dim > ZO_DIM_MAX) return 0;
  const uint64_t group = q_heads / heads < 16 ? q_heads / heads : 16;
  const uint64_t row = (dim + 3) / 4 * 4 + 4;
  return zo::attend_items_bytes(seqs, q_heads, heads) + 2ull * zo::attend_workers(dim) * group * row * sizeof(float);
}

// Rows are split from about where that is sooner. us for fp32 (bf16) rows, one workgroup each | split: with top-p alone 16,384
// logits 27 (25) | 27, 32,000 38 (33) | 28, 151,936 108 (75) | 33 for 4 rows, 43 for 16 and 57 for 32; without settings
// 14 (17) | 12 and 56 (48) | 13 for 4 rows, 21 for 32. A top-k that counts ends early in one workgroup: 16,384 logits
// 17 | 24, 151,936 25 | 23 for 4 rows, 28 for 16 and 36 for 32. What each row's top_k is lies on the device: rows whose
// top_k is 0 are as without one (108 us in one workgroup), so a call with a top_k is split as long as the rows that it
// counts for lose no more than 3 us by it (16 of them 25 | 28).
uint64_t zo_draw_work(uint32_t rows, uint32_t vocab, int top_k) {
  const uint32_t most_rows = top_k ? 16 : 32, least_vocab = top_k ? 1u << 16 : 4 * zo::kDrawPart;
  if (rows > most_rows || vocab < least_vocab || vocab > (1u << 18)) return 0;
  const uint64_t parts = (vocab + zo::kDrawPart - 1) / zo::kDrawPart;
  return rows * (parts * zo::kDrawPartWords + zo::kDrawRowWords) * 8;
}

int zo_rotary_turns(zo_rotary_kind kind, uint32_t rotary, double base, double factor, double original, double low,
                    double high, double* turns) {
  if (turns == nullptr) return ZO_ERR_NULL;
  if (kind != ZO_ROTARY_LINEAR && kind != ZO_ROTARY_BASE && kind != ZO_ROTARY_BANDS) return ZO_ERR_ARG;
  if (!std::isfinite(base) || !std::isfinite(factor)) return ZO_ERR_NONFINITE;
  const bool bands = kind == ZO_ROTARY_BANDS;
  if (bands && (!std::isfinite(original) || !std::isfinite(low) || !std::isfinite(high))) return ZO_ERR_NONFINITE;
  if (rotary < 2 || rotary % 2 != 0 || rotary > ZO_DIM_MAX || !(base > 1.0) || !(factor >= 1.0)) return ZO_ERR_ARG;
  if (bands && (!(original > 0.0) || !(low >= 0.0) || !(high > low))) return ZO_ERR_ARG;
  if (kind == ZO_ROTARY_BASE && rotary == 2) return ZO_ERR_ARG;
  const double r = static_cast<double>(rotary);
  if (kind == ZO_ROTARY_BASE) base *= std::pow(factor, r / (r - 2.0));
  for (uint32_t i = 0; i < rotary / 2; ++i) {
    double t = std::pow(base, -2.0 * i / r) / (2.0 * 3.14159265358979323846);
    if (kind == ZO_ROTARY_LINEAR) t /= factor;
    if (bands) {
      const double s = std::min(1.0, std::max(0.0, (t * original - low) / (high - low)));
      t = (1.0 - s) * (t / factor) + s * t;
    }
    turns[i] = t;
  }
  return ZO_OK;
}

}  // extern "C"
