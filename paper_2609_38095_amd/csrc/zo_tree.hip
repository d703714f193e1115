// Trees of new tokens for gfx950: their layout, the walk along the drafted tokens that the draws agree with, and the moves
// that bring a walked path together in the paged cache. Bound by latency at the sizes of a few answers (one launch each), the
// moves of a batch by HBM.

#include <algorithm>
#include <vector>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

// The new tokens of a sequence: rows begin .. begin + count - 1, whatever `starts` holds.
struct Span {
  uint32_t begin, count;
};
__device__ __forceinline__ Span span_of(const int32_t* starts, uint32_t seq, uint32_t tokens) {
  const int64_t most = tokens;
  int64_t a = starts[seq], b = starts[seq + 1];
  a = a < 0 ? 0 : a > most ? most : a;
  b = b < a ? a : b > most ? most : b;
  return {static_cast<uint32_t>(a), static_cast<uint32_t>(b - a)};
}

__device__ __forceinline__ int64_t cached_of(const int32_t* lengths, uint32_t seq) {
  const int64_t n = lengths[seq];
  return n < 0 ? 0 : n;
}

__device__ __forceinline__ int32_t saturated(int64_t v) { return static_cast<int32_t>(v > 0x7FFFFFFF ? 0x7FFFFFFF : v); }

__device__ __forceinline__ uint64_t lane_u64(uint64_t v, uint32_t lane) {
  const uint32_t lo = __shfl(static_cast<uint32_t>(v), lane, 64), hi = __shfl(static_cast<uint32_t>(v >> 32), lane, 64);
  return static_cast<uint64_t>(hi) << 32 | lo;
}

constexpr uint32_t kWave = 64;

// ---- layout

// A wave has a sequence, 64 new tokens at a time. Within these a mask doubles its reach in each of six steps (it
// takes in the mask of the token that it has come to); a token's index is above that of the one it comes behind, so the lowest
// bit of the finished mask is where the branch enters the 64, and what is before that is finished in LDS.
// The last workgroup has the rows of no sequence. 256 trees of up to 200 take 6.1 us, one of 12 takes 1.9; either call 6.8.
__global__ void __launch_bounds__(kWave) lay_kernel(const zo_tree t) {
  extern __shared__ uint64_t lds[];  // [64 words][words] masks, where a tree has more than 64 tokens
  const uint32_t lane = threadIdx.x, seq = blockIdx.x, words = t.words;
  const auto none = [&](uint32_t row) {
    t.seq_of[row] = t.positions[row] = t.places[row] = -1;
    for (uint32_t w = 0; w < words; ++w) t.seen[static_cast<size_t>(row) * words + w] = 0;
  };
  if (seq == t.seqs) {
    const uint32_t first = t.seqs > 0 ? span_of(t.starts, 0, t.tokens).begin : t.tokens;
    const Span last = t.seqs > 0 ? span_of(t.starts, t.seqs - 1, t.tokens) : Span{t.tokens, 0};
    for (uint32_t i = lane; i < first; i += kWave) none(i);
    for (uint32_t i = last.begin + last.count + lane; i < t.tokens; i += kWave) none(i);
    return;
  }
  const Span sp = span_of(t.starts, seq, t.tokens);
  const int64_t cached = cached_of(t.lengths, seq);
  if (t.parents == nullptr && words == 0) {
    for (uint32_t i = lane; i < sp.count; i += kWave) {
      t.seq_of[sp.begin + i] = static_cast<int32_t>(seq);
      t.positions[sp.begin + i] = t.places[sp.begin + i] = saturated(cached + i);
    }
    return;
  }
  const uint32_t count = min(sp.count, kWave * words);
  for (uint32_t block = 0; block * kWave < count; ++block) {
    const uint32_t i = block * kWave + lane, row = sp.begin + i;
    const bool there = i < count;
    int32_t parent = -1;
    if (there) parent = t.parents ? t.parents[row] : static_cast<int32_t>(i) - 1;
    if (static_cast<uint32_t>(parent) >= i) parent = -1;
    const int32_t before = static_cast<int32_t>(block * kWave);
    int32_t jump = parent >= before ? parent - before : -1;
    const int32_t outer = parent < before ? parent : -1;  // in the 64s before
    uint64_t mask = 1ull << lane;
#pragma unroll
    for (int step = 0; step < 6; ++step) {
      const uint32_t from = jump < 0 ? lane : static_cast<uint32_t>(jump);
      const uint64_t theirs = lane_u64(mask, from);
      const int32_t next = __shfl(jump, from, 64);
      if (jump >= 0) {
        mask |= theirs;
        jump = next;
      }
    }
    const int32_t entry = __shfl(outer, static_cast<uint32_t>(__builtin_ctzll(mask)), 64);
    int64_t depth = __popcll(mask) - 1;
    for (uint32_t w = 0; w < words; ++w) {
      uint64_t bits = w == block ? mask : 0;
      if (w < block && entry >= 0) bits = lds[static_cast<uint32_t>(entry) * words + w];
      if (w < block) depth += __popcll(bits);
      if (there) t.seen[static_cast<size_t>(row) * words + w] = bits;
      if (words > 1) lds[i * words + w] = bits;
    }
    if (there) {
      t.seq_of[row] = static_cast<int32_t>(seq);
      t.positions[row] = saturated(cached + depth);
      t.places[row] = saturated(cached + i);
    }
    __syncthreads();  // one wave: the masks before the next 64 read them
  }
  for (uint32_t i = count + lane; i < sp.count; i += kWave) none(sp.begin + i);
}

// ---- walk

constexpr uint32_t kWalkThreads = 256, kWindow = 1024;
constexpr uint32_t kNone = 0xFFFFFFFFu;

// A workgroup has a sequence, kWindow new tokens at a time. Every token whose drafted token is the one drawn behind its parent offers
// itself as its parent's next (the lowest index wins, in LDS), and one thread follows these from the token that the walk has come to.
// Children lie behind their parent, so one whose next is not in this window has it in a later one or nowhere. A chain needs
// no following: it ends at the first token that does not offer itself. 256 sequences take 3.8 us, four 2.8; either call 6.1.
__global__ void __launch_bounds__(kWalkThreads) accept_kernel(const zo_tree_walk w) {
  __shared__ uint32_t next[kWindow], path[kWindow], first, found, at_shared;
  const uint32_t seq = blockIdx.x;
  Span sp = span_of(w.starts, seq, w.tokens);
  if (w.words > 0) sp.count = min(sp.count, kWave * w.words);  // the tokens that the masks have room for
  int32_t* path_out = w.path + static_cast<size_t>(seq) * w.most;
  int32_t* tokens_out = w.tokens_out + static_cast<size_t>(seq) * w.most;
  uint32_t at = 0, walked = 0;  // the token that the walk has come to; tokens before those found in this window
  for (uint32_t base = 0; base < sp.count && walked < w.most; base += kWindow) {
    const uint32_t count = min(kWindow, sp.count - base), room = w.most - walked;
    for (uint32_t i = threadIdx.x; i < kWindow; i += kWalkThreads) next[i] = kNone;
    if (threadIdx.x == 0) first = kNone;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += kWalkThreads) {
      const uint32_t j = base + i, row = sp.begin + j;
      const uint32_t parent = w.parents ? static_cast<uint32_t>(w.parents[row]) : j - 1;
      const bool offers = j > 0 && parent < j && w.drafted[row] >= 0 && w.drafted[row] == w.drawn[sp.begin + parent];
      if (w.parents == nullptr) {
        if (j > 0 && !offers) atomicMin(&first, i);
      } else if (offers) {
        if (parent >= base)
          atomicMin(&next[parent - base], j);
        else if (parent == at)
          atomicMin(&first, j);
      }
    }
    __syncthreads();
    if (w.parents == nullptr) {
      const uint32_t end = min(first, count);
      for (uint32_t i = threadIdx.x; i < min(end, room); i += kWalkThreads) path[i] = base + i;
      if (threadIdx.x == 0) found = min(end, room);
      at = base + end;
    } else if (threadIdx.x == 0) {
      uint32_t n = 0;
      uint32_t j = base == 0 ? 0 : first;  // token 0 begins the walk
      while (j != kNone && n < room) {
        path[n++] = at = j;
        j = next[j - base];
      }
      found = n;
      at_shared = at;
    }
    __syncthreads();
    if (w.parents) at = at_shared;
    const uint32_t n = found;
    for (uint32_t i = threadIdx.x; i < n; i += kWalkThreads) {
      path_out[walked + i] = static_cast<int32_t>(path[i]);
      tokens_out[walked + i] = w.drawn[sp.begin + path[i]];
    }
    walked += n;
    __syncthreads();
    if (w.parents == nullptr && at < base + count) break;  // the chain ended inside this window
  }
  for (uint32_t i = walked + threadIdx.x; i < w.most; i += kWalkThreads) path_out[i] = tokens_out[i] = -1;
  if (threadIdx.x == 0) w.counts[seq] = static_cast<int32_t>(walked);
}

// ---- moves

constexpr uint32_t kKeepThreads = 256, kTensors = 112, kTogether = 8;

struct Keep {
  char* tensor[kTensors];
  const int32_t *ids, *lengths, *path;
  int64_t table_stride, path_stride, page_stride, head_stride, token_stride;  // the latter three in bytes
  uint32_t width, pages, page_tokens, most, n_tensors;
  uint32_t row_vecs, vecs;  // vectors of a row, and of all heads' rows of a token
  uint32_t tensors_each;    // of a workgroup
};

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

// Byte offset of a token's row in its page, -1 where there is none.
__device__ __forceinline__ int64_t row_at(const Keep& k, uint32_t seq, int64_t token) {
  const int64_t slot = token / k.page_tokens;
  if (slot >= k.width) return -1;
  const int32_t id = k.ids[static_cast<int64_t>(seq) * k.table_stride + slot];
  if (static_cast<uint32_t>(id) >= k.pages) return -1;
  return id * k.page_stride + (token - slot * k.page_tokens) * k.token_stride;
}

// Tensors of a workgroup: as many as give its threads a vector each, more where there are workgroups enough. 256 paths in 72 tensors:
// 32 us with up to 8,192 workgroups, 48 with 2,048.
uint32_t tensors_each(uint32_t seqs, uint32_t tensors, uint32_t vecs) {
  const uint64_t enough = (static_cast<uint64_t>(seqs) * tensors + 8191) / 8192, full = (kKeepThreads + vecs - 1) / vecs;
  return static_cast<uint32_t>(std::min<uint64_t>(tensors, std::max(enough, full)));
}

// A workgroup has one sequence in a few tensors; its first wave lists the rows that move, 64 of the path at a time, and each thread
// moves its vector of every listed row, kTogether of them loaded before the first is stored. In this order a row
// is read before it is written: the walk rises, so path[j] > path[i] >= i for j > i, and what is written for i is no later
// row's source. 256 paths in 72 tensors, three inputs in turn: 32 us, 4.8 TB/s (21 us where the last call's lines are still cached).
template <int kVec>
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const Keep k) {
  typedef typename Piece<kVec>::value T;
  typedef typename Piece<kVec>::place At;
  __shared__ int64_t src[kWave], dst[kWave];
  __shared__ uint32_t listed, ended;
  const uint32_t seq = blockIdx.x;
  const int32_t* path = k.path + static_cast<int64_t>(seq) * k.path_stride;
  const int64_t cached = cached_of(k.lengths, seq);
  const uint32_t tensor0 = blockIdx.y * k.tensors_each, tensors = min(k.tensors_each, k.n_tensors - tensor0);
  for (uint32_t base = 0; base < k.most; base += kWave) {
    if (threadIdx.x < kWave) {
      const uint32_t i = base + threadIdx.x;
      const bool in = i < k.most;
      const int32_t p = in ? path[i] : -1, before = in && i > 0 ? path[i - 1] : -1;
      const uint64_t ends = __ballot(p < 0 || p <= before);
      const bool walked = ends == 0 || threadIdx.x < static_cast<uint32_t>(__builtin_ctzll(ends));
      int64_t from = -1, to = -1;
      if (walked && p != static_cast<int32_t>(i)) {
        from = row_at(k, seq, cached + p);
        to = row_at(k, seq, cached + i);
      }
      const bool moves = from >= 0 && to >= 0;
      const uint64_t all = __ballot(moves);
      if (moves) {
        const uint32_t n = __popcll(all & ((1ull << threadIdx.x) - 1));
        src[n] = from;
        dst[n] = to;
      }
      if (threadIdx.x == 0) {
        listed = __popcll(all);
        ended = ends != 0;
      }
    }
    __syncthreads();
    const uint32_t n = listed;
    const bool last = ended != 0;
    if (n > 0) {
      for (uint32_t e = threadIdx.x; e < tensors * k.vecs; e += kKeepThreads) {
        const uint32_t tensor = e / k.vecs, v = e - tensor * k.vecs, head = v / k.row_vecs;
        char* at = k.tensor[tensor0 + tensor] + head * k.head_stride + (v - head * k.row_vecs) * kVec;
        for (uint32_t i = 0; i < n; i += kTogether) {
          T got[kTogether];
#pragma unroll
          for (uint32_t j = 0; j < kTogether; ++j)
            if (i + j < n) got[j] = *reinterpret_cast<const At*>(at + src[i + j]);
#pragma unroll
          for (uint32_t j = 0; j < kTogether; ++j)
            if (i + j < n) *reinterpret_cast<At*>(at + dst[i + j]) = got[j];
        }
      }
    }
    __syncthreads();
    if (last) return;
  }
}

}  // namespace
}  // namespace zo

extern "C" {

int zo_tree_lay(const zo_tree* t, void* stream) {
  using namespace zo;
  if (t == nullptr) return ZO_ERR_NULL;
  const int rc = check_tree(*t);
  if (rc != ZO_OK) return rc;
  if (t->tokens == 0) return ZO_OK;
  const size_t lds = t->words > 1 ? static_cast<size_t>(kWave) * t->words * t->words * sizeof(uint64_t) : 0;
  (void)hipGetLastError();
  lay_kernel<<<dim3(t->seqs + 1), dim3(kWave), lds, static_cast<hipStream_t>(stream)>>>(*t);
  return launched();
}

int zo_tree_accept(const zo_tree_walk* w, void* stream) {
  using namespace zo;
  if (w == nullptr) return ZO_ERR_NULL;
  const int rc = check_walk(*w);
  if (rc != ZO_OK) return rc;
  if (w->seqs == 0) return ZO_OK;
  (void)hipGetLastError();
  accept_kernel<<<dim3(w->seqs), dim3(kWalkThreads), 0, static_cast<hipStream_t>(stream)>>>(*w);
  return launched();
}

int zo_tree_keep(const zo_tree_moves* m, void* stream) {
  using namespace zo;
  if (m == nullptr) return ZO_ERR_NULL;
  std::vector<int64_t> tensors;  // each once
  const int rc = check_moves_of(*m, tensors);
  if (rc != ZO_OK) return rc;
  if (m->n_tensors == 0 || m->table.seqs == 0 || m->most == 0) return ZO_OK;
  const int64_t elem = static_cast<int64_t>(elem_bytes(m->dtype));
  const zo_cache& f = m->shape;
  Keep k;
  k.ids = m->table.ids;
  k.lengths = m->lengths;
  k.path = m->path;
  k.table_stride = m->table.stride;
  k.path_stride = m->path_stride;
  k.page_stride = f.page_stride * elem;
  k.head_stride = f.head_stride * elem;
  k.token_stride = f.token_stride * elem;
  k.width = m->table.width;
  k.pages = f.pages;
  k.page_tokens = f.page_tokens;
  k.most = m->most;
  const bool vectors = f.dim * elem % 16 == 0;
  k.row_vecs = vectors ? static_cast<uint32_t>(f.dim * elem / 16) : f.dim;
  k.vecs = k.row_vecs * f.heads;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const uint32_t n_tensors = static_cast<uint32_t>(tensors.size());
  for (uint32_t t0 = 0; t0 < n_tensors; t0 += kTensors) {
    k.n_tensors = std::min(kTensors, n_tensors - t0);
    for (uint32_t i = 0; i < k.n_tensors; ++i) k.tensor[i] = reinterpret_cast<char*>(tensors[t0 + i]);
    k.tensors_each = tensors_each(m->table.seqs, k.n_tensors, k.vecs);
    const dim3 grid(m->table.seqs, (k.n_tensors - 1) / k.tensors_each + 1), block(kKeepThreads);
    if (vectors)
      keep_kernel<16><<<grid, block, 0, st>>>(k);
    else if (elem == 4)
      keep_kernel<4><<<grid, block, 0, st>>>(k);
    else
      keep_kernel<2><<<grid, block, 0, st>>>(k);
    const int rl = launched();
    if (rl != ZO_OK) return rl;
  }
  return ZO_OK;
}

}  // extern "C"
