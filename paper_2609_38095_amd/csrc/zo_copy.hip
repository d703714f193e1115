// Copies of cache pages for gfx950: forks, compactions. Bound by HBM: one read and one write of the
// rows that are copied. 1,024 pages of 16 tokens, 8 heads of 128 in bf16, in 28 layers (3.8 GB): 720 us,
// 5.2 TB/s (a plain copy with as much in flight for each wave reaches 5.6).
//
// A move copies `rows` tokens of every key head, keys and values, in every cache. One workgroup takes
// 256 vectors of 16 bytes of a head's rows, in as many heads (8, 4, 2 or 1) of one page of one tensor as
// divide their number; all are loaded before the first is stored. The moves and the tensors' addresses
// travel as kernel arguments, so the call needs no device memory and no copy of its own.

#include <algorithm>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMoves = 240;      // of a launch (kernel arguments below 4 KiB)
constexpr uint32_t kTensors = 112;

struct Copy {
  char* tensor[kTensors];  // keys and values of each cache
  zo_page_move move[kMoves];
  int64_t page_stride, head_stride, token_stride;  // bytes
  uint32_t row_vecs;                               // vectors of a row
  uint32_t vec_parts, head_parts;                  // workgroups of a page
};

// kVec: bytes of a vector (16, or the element where a row is not a whole number of vectors).
template <int kVec>
struct Piece;
template <>
struct Piece<16> {
  typedef u32x4 value;
  typedef u32x4_any place;  // at any element's address
};
template <>
struct Piece<4> {
  typedef uint32_t value, place;
};
template <>
struct Piece<2> {
  typedef uint16_t value, place;
};

template <int kVec, uint32_t kHeads>
__global__ void __launch_bounds__(kThreads) copy_kernel(const Copy c) {
  typedef typename Piece<kVec>::value T;
  typedef typename Piece<kVec>::place At;
  const uint32_t vec_part = blockIdx.x % c.vec_parts, rest = blockIdx.x / c.vec_parts;
  const uint32_t head0 = rest % c.head_parts * kHeads, m = rest / c.head_parts;
  const zo_page_move mv = c.move[m];
  char* base = c.tensor[blockIdx.y];
  const uint32_t i = vec_part * kThreads + threadIdx.x;
  const uint32_t row = i / c.row_vecs, vec = i - row * c.row_vecs;
  if (row >= static_cast<uint32_t>(mv.rows)) return;
  const int64_t at = head0 * c.head_stride + row * c.token_stride + vec * kVec;
  const char* src = base + mv.src * c.page_stride + at;
  char* dst = base + mv.dst * c.page_stride + at;
  T v[kHeads];
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h)
    v[h] = __builtin_nontemporal_load(reinterpret_cast<const At*>(src + h * c.head_stride));
#pragma unroll
  for (uint32_t h = 0; h < kHeads; ++h)
    __builtin_nontemporal_store(v[h], reinterpret_cast<At*>(dst + h * c.head_stride));
}

template <int kVec>
void launch(const Copy& c, uint32_t heads, dim3 grid, hipStream_t st) {
  const dim3 block(kThreads);
  switch (heads) {
    case 8: copy_kernel<kVec, 8><<<grid, block, 0, st>>>(c); break;
    case 4: copy_kernel<kVec, 4><<<grid, block, 0, st>>>(c); break;
    case 2: copy_kernel<kVec, 2><<<grid, block, 0, st>>>(c); break;
    default: copy_kernel<kVec, 1><<<grid, block, 0, st>>>(c);
  }
}

}  // namespace
}  // namespace zo

extern "C" int zo_cache_copy(const zo_cache* shape, void* const* tensors, uint32_t n_tensors, const zo_page_move* moves,
                             uint32_t n_moves, zo_dtype dtype, void* stream) {
  using namespace zo;
  const int rc = check_copy(shape, tensors, n_tensors, moves, n_moves, dtype);
  if (rc != ZO_OK) return rc;
  if (n_tensors == 0 || n_moves == 0) return ZO_OK;
  const int64_t elem = static_cast<int64_t>(elem_bytes(dtype));
  const zo_cache& f = *shape;
  Copy c;
  c.page_stride = f.page_stride * elem;
  c.head_stride = f.head_stride * elem;
  c.token_stride = f.token_stride * elem;
  const bool vectors = f.dim * elem % 16 == 0;
  c.row_vecs = vectors ? static_cast<uint32_t>(f.dim * elem / 16) : f.dim;
  const uint32_t together = f.heads % 8 == 0 ? 8 : f.heads % 4 == 0 ? 4 : f.heads % 2 == 0 ? 2 : 1;
  c.head_parts = f.heads / together;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  for (uint32_t m0 = 0; m0 < n_moves; m0 += kMoves) {
    const uint32_t n = std::min(kMoves, n_moves - m0);
    std::copy(moves + m0, moves + m0 + n, c.move);
    uint32_t rows = 0;
    for (uint32_t i = 0; i < n; ++i) rows = std::max(rows, static_cast<uint32_t>(c.move[i].rows));
    c.vec_parts = (rows * c.row_vecs - 1) / kThreads + 1;
    for (uint32_t t0 = 0; t0 < n_tensors; t0 += kTensors) {
      const uint32_t count = std::min(kTensors, n_tensors - t0);
      for (uint32_t i = 0; i < count; ++i) c.tensor[i] = static_cast<char*>(tensors[t0 + i]);
      const dim3 grid(c.vec_parts * c.head_parts * n, count);
      if (vectors)
        launch<16>(c, together, grid, st);
      else if (elem == 4)
        launch<4>(c, together, grid, st);
      else
        launch<2>(c, together, grid, st);
      const int rl = launched();
      if (rl != ZO_OK) return rl;
    }
  }
  return ZO_OK;
}
