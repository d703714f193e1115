// Attention of several new tokens of each sequence over the paged cache, for gfx950: drafted trees and prompts.
//
// Mathematics. As for one token (zo_attend.hip): one pass over the keys with a running bound m of the scores and a sum l, p_j =
// 2^(x_j - m), o = sum p_j v_j; only a score above the bound raises it, to 8 above the largest. What is new are the rows: a row
// is a new token and a query head of one key head's group, so rows share keys, and each sees its own of the sequence's new tokens.
//
// Split. An item is a sequence, a key head and kRows rows; it is cut into tiles of kTile tokens up to the last one that a row of
// it can see. The tiles of all items, in order, are dealt out in equal runs to the workgroups, which find theirs from
// lengths and starts by themselves. A run that covers an item writes its output, others leave (m, l, o) in the workspace, at most
// two parts for each workgroup, and join_kernel joins them. Runs that follow each other, which read the same keys, lie on one XCD.
//
// Tile. S^T = K Q^T and O^T = V^T P^T in 32 x 32 products, a row in each lane (r = lane % 32), so a row's bound and sum stay in
// its two lanes (g = lane / 32). A wave has 32 rows. kRowWaves = 4: four waves have different rows and share a tile's keys and
// values, two buffers of them in LDS; kRowWaves = 1 (sequences of few rows): four waves have the same rows and a quarter of the
// tile's keys each, in LDS of their own, without a barrier; they join at an item's end. The next tile waits in
// registers while one is used.
//   - LDS rows are swizzled by 16-byte chunks, so that neither product's reads meet in a bank;
//   - S^T leaves in lane (r, g) the keys 8 i + 4 g .. + 3: the second product's operand as it is, if the contraction's index
//     is permuted alike; the values' operand is read by the transposing LDS read (bf16), four keys of 16 dims at a time.
//
// What a row does not see. Scores are masked, and keys that no row of the call may use are zeros in LDS. A value that is
// infinite or NaN in a tile that only some of the rows see would reach the others as 0 times itself: such rows are zeros in
// LDS too, and are added by those rows that see them one at a time.

#include <algorithm>
#include <cmath>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kThreads = 256, kWave = 64, kWaves = kThreads / kWave, kXcds = 8;
constexpr float kLazy = 8.0f;  // how far (in powers of two) the bound of the scores is set above their maximum

// Where an item's parts are, written by the workgroup of its last tile: those of workgroups first .. last, the first one's in
// slot first_slot % 2, the others' in slot 0; first = last: that workgroup wrote the output.
struct Item {
  uint32_t first_slot, last;
  uint32_t token, row, rows, head;  // the sequence's first new token; the item's first row and their number; key head
  uint32_t unused[2];
};
static_assert(sizeof(Item) == kTreeItemWords * 4, "the workspace holds items of this size");

struct Attend {
  const char *q, *k, *v;
  char* out;
  float* lse;
  uint32_t* item_count;
  Item* items;
  float* parts;
  const int32_t *ids, *lengths, *starts;
  const uint64_t* seen;
  int64_t seen_stride, q_token, q_head, out_token, out_head, page_bytes, head_bytes, token_bytes, table_stride;
  double inv_group;
  uint32_t most_items, tokens, words, seqs, width, pages, page_tokens, heads, group, dim, workers, part_row;
  int32_t page_shift;  // of a page's tokens where they are a power of two, else -1
  float scale;         // times log2(e)
};

// A value that all lanes of a wave hold, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return static_cast<uint64_t>(uniform(static_cast<uint32_t>(v >> 32))) << 32 | uniform(static_cast<uint32_t>(v));
}

// Floor of n / d for n below 2^52: exact, since quotients of neighbours are further apart than an fp64 rounding.
__device__ __forceinline__ uint64_t quotient(uint64_t n, uint64_t d) {
  return static_cast<uint64_t>(static_cast<double>(n) / static_cast<double>(d));
}

struct Seq {
  uint32_t token, count;  // its new tokens
  uint32_t cached, len;   // tokens before them, and with them: as many as the table holds
  uint32_t blocks;        // items of each key head
};

template <uint32_t kRows>
__device__ __forceinline__ Seq seq_of(const Attend& a, uint32_t seq) {
  const int64_t room = static_cast<int64_t>(a.width) * a.page_tokens, most = a.tokens;
  int64_t first = a.starts[seq], last = a.starts[seq + 1], cached = a.lengths[seq];
  first = first < 0 ? 0 : first > most ? most : first;
  last = last < first ? first : last > most ? most : last;
  cached = cached < 0 ? 0 : cached > room ? room : cached;
  Seq s;
  s.token = static_cast<uint32_t>(first);
  s.count = static_cast<uint32_t>(last - first);
  s.cached = static_cast<uint32_t>(cached);
  s.len = static_cast<uint32_t>(cached + s.count < room ? cached + s.count : room);
  s.blocks = (s.count * a.group + kRows - 1) / kRows;
  return s;
}

// The new token of a row (rows below 2^24: the product's error stays below the half's share).
__device__ __forceinline__ uint32_t node_of(const Attend& a, uint32_t row) {
  return static_cast<uint32_t>((static_cast<double>(row) + 0.5) * a.inv_group);
}

// How many tokens the rows of a sequence up to (and without) `row` can see.
__device__ __forceinline__ uint32_t visible(const Attend& a, const Seq& s, uint32_t row) {
  if (a.seen) return s.len;
  const uint32_t rows = s.count * a.group;
  return min(s.len, s.cached + node_of(a, min(row, rows) - 1) + 1);
}

// Tiles of an item; at least one, which writes the rows that see nothing.
template <uint32_t kRows, uint32_t kTile>
__device__ __forceinline__ uint32_t tiles_of(const Attend& a, const Seq& s, uint32_t block) {
  return max(1u, (visible(a, s, (block + 1) * kRows) + kTile - 1) / kTile);
}

// The sum over a wave of a value of each lane, and the sums up to each lane.
__device__ __forceinline__ uint64_t sums_upto(uint64_t v, uint32_t lane) {
#pragma unroll
  for (uint32_t m = 1; m < kWave; m *= 2) {
    const uint64_t lower = __shfl_up(v, m, 64);
    if (lane >= m) v += lower;
  }
  return v;
}

// Tiles of one key head of a sequence, by all lanes together.
template <uint32_t kRows, uint32_t kTile>
__device__ uint64_t head_tiles(const Attend& a, const Seq& s, uint32_t lane) {
  if (a.seen) return static_cast<uint64_t>(s.blocks) * tiles_of<kRows, kTile>(a, s, 0);
  uint64_t mine = 0;
  for (uint32_t b = lane; b < s.blocks; b += kWave) mine += tiles_of<kRows, kTile>(a, s, b);
  return uniform(__shfl(sums_upto(mine, lane), 63, 64));
}

// Tiles and items before each thread's sequences. Thread t counts sequences [t each, (t + 1) each).
struct Deal {
  uint64_t total;
  uint32_t items, each;
};

template <uint32_t kRows, uint32_t kTile>
__device__ Deal deal(const Attend& a, uint64_t* before, uint32_t* items_before) {
  __shared__ uint64_t wave_tiles[kWaves], wave_items[kWaves];
  const uint32_t lane = threadIdx.x % kWave;
  Deal d;
  d.each = (a.seqs + kThreads - 1) / kThreads;
  uint64_t tiles = 0, items = 0;
  for (uint32_t i = 0; i < d.each; ++i) {
    const uint32_t seq = threadIdx.x * d.each + i;
    Seq s = {};
    if (seq < a.seqs) s = seq_of<kRows>(a, seq);
    items += s.blocks;
    constexpr uint32_t kFew = 8;  // blocks that a thread counts by itself; a longer sequence's by the whole wave
    if (a.seen) {
      if (s.blocks) tiles += static_cast<uint64_t>(s.blocks) * tiles_of<kRows, kTile>(a, s, 0);
    } else {
      if (s.blocks <= kFew)
        for (uint32_t b = 0; b < s.blocks; ++b) tiles += tiles_of<kRows, kTile>(a, s, b);
      for (uint64_t left = __ballot(s.blocks > kFew); left != 0; left &= left - 1) {
        const uint32_t from = static_cast<uint32_t>(__builtin_ctzll(left));
        Seq one;
        one.token = 0;
        one.count = __builtin_amdgcn_readlane(s.count, from);
        one.cached = __builtin_amdgcn_readlane(s.cached, from);
        one.len = __builtin_amdgcn_readlane(s.len, from);
        one.blocks = __builtin_amdgcn_readlane(s.blocks, from);
        const uint64_t all = head_tiles<kRows, kTile>(a, one, lane);
        if (lane == from) tiles += all;
      }
    }
  }
  const uint64_t tiles_upto = sums_upto(tiles, lane), items_upto = sums_upto(items, lane);
  if (lane == 63) {
    wave_tiles[threadIdx.x / kWave] = tiles_upto;
    wave_items[threadIdx.x / kWave] = items_upto;
  }
  __syncthreads();
  uint64_t tiles_at = 0, tiles_all = 0, items_at = 0, items_all = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < threadIdx.x / kWave) {
      tiles_at += wave_tiles[w];
      items_at += wave_items[w];
    }
    tiles_all += wave_tiles[w];
    items_all += wave_items[w];
  }
  before[threadIdx.x] = (tiles_at + tiles_upto - tiles) * a.heads;
  const uint64_t item = (items_at + items_upto - items) * a.heads;
  items_before[threadIdx.x] = static_cast<uint32_t>(item < a.most_items ? item : a.most_items);
  d.total = uniform(tiles_all * a.heads);
  d.items = uniform(static_cast<uint32_t>(items_all * a.heads < a.most_items ? items_all * a.heads : a.most_items));
  __syncthreads();
  return d;
}

// The first tile of each worker: total tiles in equal runs, the first ones a tile longer.
struct Runs {
  uint64_t each, longer;
  uint32_t workers;
  __device__ Runs(uint64_t total, uint32_t most) {
    workers = total < most ? static_cast<uint32_t>(total) : most;
    if (workers == 0) workers = 1;
    each = uniform(quotient(total, workers));
    longer = total - each * workers;
  }
  __device__ uint64_t first(uint32_t w) const { return w * each + (w < longer ? w : longer); }
  __device__ uint32_t worker_of(uint64_t tile) const {
    const uint64_t head = longer * (each + 1);  // tiles of the longer runs
    return static_cast<uint32_t>(tile < head ? quotient(tile, each + 1) : longer + quotient(tile - head, each));
  }
};

// A part in the workspace: for each row [m, l, -, -, o[dim rounded up to 4]].
template <uint32_t kRows>
__device__ __forceinline__ float* part_at(const Attend& a, uint32_t worker, uint32_t slot) {
  return a.parts + (static_cast<size_t>(worker) * 2 + slot) * kRows * a.part_row;
}

// Four dims of a row's output from its sums, and its log-sum once.
template <class S>
__device__ __forceinline__ void write_row(const Attend& a, uint32_t token, uint32_t q_head, uint32_t dim, float m, float l, f32x4 o) {
  typedef typename S::storage T;
  const bool any = l > 0.0f || l != l;
  T* op = reinterpret_cast<T*>(a.out) + static_cast<int64_t>(token) * a.out_token + static_cast<int64_t>(q_head) * a.out_head;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    if (dim + i < a.dim) S::store1(op + dim + i, any ? o[i] / l : 0.0f);
  if (a.lse && dim == 0)
    a.lse[static_cast<size_t>(token) * a.heads * a.group + q_head] = any ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// Sixteen bytes of a row from dim `at` on; behind the row's end zeros.
template <class T>
__device__ __forceinline__ u32x4 load_chunk_of(const char* row, uint32_t at, uint32_t dim) {
  constexpr uint32_t kElems = 16 / sizeof(T);
  if (at + kElems <= dim) return *reinterpret_cast<const u32x4_any*>(row + at * sizeof(T));
  T got[kElems] = {};
#pragma unroll
  for (uint32_t e = 0; e < kElems; ++e)
    if (at + e < dim) got[e] = reinterpret_cast<const T*>(row)[at + e];
  u32x4 v;
  __builtin_memcpy(&v, got, 16);
  return v;
}

// Whether any of the values is infinite or NaN.
template <class T>
__device__ __forceinline__ bool odd_values(u32x4 v) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2)
      odd = odd || (v[i] & 0x7F800000u) == 0x7F800000u || (v[i] & 0x7F80u) == 0x7F80u;
    else
      odd = odd || (v[i] & 0x7F800000u) == 0x7F800000u;
  }
  return odd;
}

// The kernel's arguments read anew: a copy of its own for each part of the kernel, so that those of one part do not hold (and spill) the
// scalar registers of another.
__device__ __forceinline__ Attend arguments() {
  typedef const __attribute__((address_space(4))) Attend* Arguments;
  Arguments from = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(from));
  return *(const Attend*)from;
}

template <class S, uint32_t kDim, uint32_t kRowWaves, bool kAny>
struct Form {
  typedef typename S::storage T;
  static constexpr uint32_t kRowBytes = kDim * sizeof(T), kChunks = kRowBytes / 16;
  static constexpr uint32_t kRows = 32 * kRowWaves, kKeyWaves = kWaves / kRowWaves;
  static constexpr uint32_t kBlocks = kRowWaves == 4 && kRowBytes <= 256 ? 2 : 1;  // of 32 keys, of a wave in a tile
  static constexpr uint32_t kKeys = 32 * kBlocks, kTile = kKeys * kKeyWaves;
  static constexpr uint32_t kStageRows = kKeys / kRowWaves;          // rows that a wave brings
  static constexpr uint32_t kLoadRows = kWave / kChunks;             // rows of a load of all lanes
  static constexpr uint32_t kLoads = kStageRows / kLoadRows;         // of the keys, and as many of the values
  static constexpr uint32_t kBuffers = kRowWaves > 1 ? 2 : 1;
  static constexpr uint32_t kBufferBytes = 2 * kTile * kRowBytes;
  static constexpr uint32_t kLds = kBuffers * kBufferBytes;
  static constexpr uint32_t kPerCu = kRowBytes <= 256 ? 2 : 1;  // workgroups
  static_assert(kRowWaves != 1 || 2 * 32 * (kDim + 4) * 4 <= kBufferBytes, "the join at an item's end has room");
  static_assert(kLoadRows <= 8 && kStageRows % kLoadRows == 0, "a load's rows lie in one sixteen");
};

typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ uint32_t lds_address(const char* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char*)p)); }

// Sixteen bytes of each lane from base + offset straight into LDS, one lane behind another from `to` on. The compiler does not
// count these loads: loads_left() waits for them.
__device__ __forceinline__ void load_to_lds(uint32_t to, uint64_t base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
template <int kLeft>
__device__ __forceinline__ void loads_left() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLeft) : "memory");
}

// kAny: any head size (kDim: the size that it is padded to with zeros), page size and alignment; keys and values pass through
// registers. Else: heads of kDim, pages of whole sixteens of tokens, 16-byte aligned rows, straight into LDS.
template <class S, uint32_t kDim, uint32_t kRowWaves, bool kAny>
__global__ void __launch_bounds__(kThreads, (Form<S, kDim, kRowWaves, kAny>::kPerCu)) attend_kernel(const Attend) {
  typedef Form<S, kDim, kRowWaves, kAny> F;
  typedef typename S::storage T;
  constexpr bool kWide = sizeof(T) == 4;
  constexpr uint32_t kRowBytes = F::kRowBytes, kChunks = F::kChunks, kRows = F::kRows, kBlocks = F::kBlocks, kKeys = F::kKeys;
  constexpr uint32_t kTile = F::kTile, kLoads = F::kLoads, kLoadRows = F::kLoadRows, kOuts = kDim / 32, kSteps = kChunks / 2;
  constexpr uint32_t kKeyMask = kChunks < 16 ? kChunks - 1 : 15;                 // the keys' swizzle
  extern __shared__ __align__(16) char lds[];
  __shared__ uint64_t before[kThreads];
  __shared__ uint32_t items_before[kThreads];
  __shared__ uint32_t odd_there[2];  // odd values in this item's tiles, and emptied for the next item's
  __shared__ float2 merge_sums[2][32];

  const uint32_t wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 32, g = lane / 32;
  const uint32_t rw = wave % kRowWaves, kw = wave / kRowWaves;  // which rows, which keys
  Deal d;
  uint32_t workers;
  {
    const Attend a = arguments();
    d = deal<kRows, kTile>(a, before, items_before);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.item_count = d.items;
    workers = a.workers;
  }
  const Runs runs(d.total, workers);
  // neighbouring runs on one XCD: workgroup b runs on XCD b % 8
  const uint32_t per_xcd = (runs.workers + kXcds - 1) / kXcds;
  const uint32_t slot_of = blockIdx.x / kXcds, worker = blockIdx.x % kXcds * per_xcd + slot_of;
  if (slot_of >= per_xcd || worker >= runs.workers) return;
  const uint64_t begin = runs.first(worker), end = runs.first(worker + 1);
  uint64_t at = begin;
  if (at >= end) return;

  // the sequence, key head and block that tile `at` lies in
  uint32_t seq, head, block, item;
  uint64_t item_first;
  Seq s;
  {
    const Attend a = arguments();
    uint32_t chunk = 0;  // the last thread's sequences that begin at or before it
#pragma unroll
    for (uint32_t step = kThreads / 2; step > 0; step /= 2)
      if (before[chunk + step] <= at) chunk += step;
    chunk = uniform(chunk);
    seq = chunk * d.each;
    item = uniform(items_before[chunk]);
    uint64_t first = uniform(before[chunk]), tiles;
    for (;; ++seq) {  // `at` < the total: a sequence holds it
      s = seq_of<kRows>(a, seq);
      tiles = s.blocks ? head_tiles<kRows, kTile>(a, s, lane) : 0;
      if (at < first + tiles * a.heads) break;
      first += tiles * a.heads;
      item += s.blocks * a.heads;
    }
    head = uniform(static_cast<uint32_t>(quotient(at - first, tiles)));
    first += tiles * head;
    uint64_t rest = at - first;
    if (a.seen) {
      const uint32_t each = tiles_of<kRows, kTile>(a, s, 0);
      block = uniform(static_cast<uint32_t>(quotient(rest, each)));
      item_first = first + static_cast<uint64_t>(block) * each;
    } else {
      for (block = 0;; block += kWave) {
        const uint32_t mine = block + lane < s.blocks ? tiles_of<kRows, kTile>(a, s, block + lane) : 0;
        const uint64_t upto = sums_upto(mine, lane);
        const uint64_t over = __ballot(upto > rest);
        if (over != 0) {
          const uint32_t l = static_cast<uint32_t>(__builtin_ctzll(over));
          item_first = first + uniform(__shfl(upto - mine, l, 64));
          block += l;
          break;
        }
        const uint64_t all = uniform(__shfl(upto, 63, 64));
        first += all;
        rest -= all;
      }
    }
    item = min(item + head * s.blocks + block, a.most_items);
  }

  // LDS places of the lane's shares: of the rows that it brings, of the key and of the values that it uses
  const uint32_t stage_row = rw * F::kStageRows, load_row = lane / kChunks, load_chunk = lane % kChunks;
  char* own = lds + kw * 2 * kKeys * kRowBytes;  // the keys of the waves that share them, and their values behind these
  const uint32_t key_at = r * kRowBytes + ((g ^ (r & kKeyMask)) * 16);
  uint32_t value_at;
  if constexpr (kWide) {
    value_at = 4 * g * kRowBytes + r * 4;
  } else {
    const uint32_t row = 4 * g + lane % 16 / 4;
    const uint32_t chunk = (lane / 16 % 2 * 2 + lane % 4 / 2) ^ (row * 2 & (kChunks - 1));
    value_at = row * kRowBytes + chunk * 16 + lane % 2 * 8;
  }
  const auto key_swizzle = [](uint32_t row) { return row & kKeyMask; };
  const auto value_swizzle = [](uint32_t row) { return kWide ? 0u : row % 8 * 2 & (kChunks - 1); };

  if (threadIdx.x == 0) odd_there[0] = 0;
  for (uint32_t turn = 0; at < end; turn ^= 1) {
    const Attend a = arguments();
    const uint32_t rows = s.count * a.group, row0 = block * kRows, in_block = min(kRows, rows - row0);
    const uint32_t sees = visible(a, s, row0 + kRows);
    const uint32_t tiles = max(1u, (sees + kTile - 1) / kTile);
    const uint32_t t_begin = static_cast<uint32_t>(at - item_first);
    const uint32_t t_end = end - item_first < tiles ? static_cast<uint32_t>(end - item_first) : tiles;
    // the lane's row, and what all rows of the workgroup and of the wave see for certain
    const uint32_t row = row0 + rw * 32 + r;
    const bool mine = rw * 32 + r < in_block;
    const uint32_t node = mine ? node_of(a, row) : 0, q_head = head * a.group + (mine ? row - node * a.group : 0);
    const bool wave_rows = rw * 32 < in_block;
    const auto certain = [&](uint32_t first_row) -> uint32_t { return a.seen ? min(s.cached, sees) : min(sees, s.cached + node_of(a, first_row) + 1); };
    const uint32_t all_see = uniform(certain(row0)), wave_sees = uniform(wave_rows ? certain(row0 + rw * 32) : 0u);
    const uint32_t wave_end = uniform(wave_rows ? visible(a, s, row0 + rw * 32 + 32) : 0u);
    const int32_t* ids = a.ids + static_cast<int64_t>(seq) * a.table_stride;
    const char* kp = a.k + head * a.head_bytes;
    const char* vp = a.v + head * a.head_bytes;

    const auto page_of = [&](uint32_t j) { return a.page_shift >= 0 ? j >> a.page_shift : j / a.page_tokens; };
    constexpr uint64_t kAll = kKeys == 64 ? ~0ull : (1ull << (kKeys % 64)) - 1;
    // Whether values of the tile may have to be emptied: not all rows see all of its keys.
    const auto some_see = [&](uint32_t t) { return t * kTile + kTile > all_see; };
    // The lane's 16 bytes of row `row` (of the wave's keys) of the values, as they go to LDS: zeros where the row is dead, and, in a tile
    // that only some rows see, where it has an infinity or a NaN. Both are known to all lanes of a row.
    const auto kept = [&](uint32_t t, uint32_t row, uint64_t live, u32x4 v) {
      bool keep = live >> row & 1;
      if (some_see(t)) {
        const uint64_t odd = __ballot(keep && odd_values<T>(v));
        if (odd != 0) {
          if (lane == 0) odd_there[turn] = 1;
          const uint64_t row_lanes = (kChunks == 64 ? ~0ull : (1ull << (kChunks % 64)) - 1) << (lane / kChunks * kChunks);
          keep = keep && (odd & row_lanes) == 0;
        }
      }
      return keep;
    };
    const u32x4 zero = {0, 0, 0, 0};

    // kAny: the page id of the lane's key of a tile; then its row's place (bytes, -1: dead).
    const auto key_of = [&](uint32_t t) { return t * kTile + kw * kKeys + lane % kKeys; };
    const auto id_of = [&](uint32_t t) {
      const uint32_t j = key_of(t);
      return t < t_end && j < sees ? ids[page_of(j)] : -1;
    };
    const auto row_of = [&](uint32_t t, int32_t id) -> int64_t {
      const uint32_t j = key_of(t);
      if (static_cast<uint32_t>(id) >= a.pages) return -1;
      return id * a.page_bytes + static_cast<int64_t>(j - page_of(j) * a.page_tokens) * a.token_bytes;
    };
    u32x4 kr[kAny ? kLoads : 1], vr[kAny ? kLoads : 1];
    const auto fetch = [&](int64_t place) {
#pragma unroll
      for (uint32_t i = 0; i < (kAny ? kLoads : 0); ++i) {
        const uint32_t from = stage_row + load_row + i * kLoadRows;
        const int32_t lo = __shfl(static_cast<int32_t>(place), from, 64), hi = __shfl(static_cast<int32_t>(place >> 32), from, 64);
        const int64_t off = hi < 0 ? 0 : static_cast<int64_t>(hi) << 32 | static_cast<uint32_t>(lo);
        kr[i] = load_chunk_of<T>(kp + off, load_chunk * (16 / sizeof(T)), a.dim);
        vr[i] = load_chunk_of<T>(vp + off, load_chunk * (16 / sizeof(T)), a.dim);
      }
    };
    const auto put = [&](uint32_t t, uint32_t buffer, uint64_t live) {
      char* keys = own + buffer * F::kBufferBytes;
      char* values = keys + kKeys * kRowBytes;
#pragma unroll
      for (uint32_t i = 0; i < (kAny ? kLoads : 0); ++i) {
        const uint32_t to = stage_row + load_row + i * kLoadRows;
        *reinterpret_cast<u32x4*>(keys + to * kRowBytes + ((load_chunk ^ key_swizzle(to)) * 16)) = kr[i];
        *reinterpret_cast<u32x4*>(values + to * kRowBytes + ((load_chunk ^ value_swizzle(to)) * 16)) = kept(t, to, live, vr[i]) ? vr[i] : zero;
      }
    };

    // Else: the page ids of 64 sixteens of tokens at a time, one in each lane. Rows of an absent page are read from page 0,
    // those behind the last token are inside their page.
    int32_t lane_id = -1;
    uint32_t lane_ids = ~0u;  // which 64 these are
    const auto sixteen_of = [&](uint32_t t) { return t * (kTile / 16) + kw * (kKeys / 16); };
    const auto page_at = [&](uint32_t sixteen) { return __builtin_amdgcn_readlane(lane_id, sixteen % 64); };
    // Which keys of the tile are live; brings the ids along.
    const auto live_of = [&](uint32_t t) -> uint64_t {
      const uint32_t first = sixteen_of(t);
      if (first / 64 != lane_ids) {
        lane_ids = first / 64;
        const uint32_t j = (lane_ids * 64 + lane) * 16;
        lane_id = j < sees ? ids[page_of(j)] : -1;
        asm volatile("s_waitcnt vmcnt(0)" : "+v"(lane_id));  // once in 64, not at every use
      }
      uint64_t live = 0;
#pragma unroll
      for (uint32_t k = 0; k < kKeys / 16; ++k) {
        const uint32_t j = (first + k) * 16;
        const bool there = static_cast<uint32_t>(page_at(first + k)) < a.pages && j < sees;
        const uint32_t mask = !there ? 0u : sees - j >= 16 ? 0xFFFFu : (1u << (sees - j)) - 1;
        live |= static_cast<uint64_t>(mask) << (16 * k);
      }
      return live;
    };
    // Bytes from the first row of a tensor to the wave's sixteen k of a tile.
    const auto sixteen_at = [&](uint32_t t, uint32_t k) {
      const uint32_t sixteen = sixteen_of(t) + k, j = sixteen * 16;
      const uint32_t id = static_cast<uint32_t>(page_at(sixteen));
      const bool there = id < a.pages;
      const uint32_t page_row = a.page_shift >= 0 ? j & (a.page_tokens - 1) : j % a.page_tokens;
      return static_cast<uint64_t>(there ? id : 0u) * static_cast<uint64_t>(a.page_bytes) + (there ? page_row : 0u) * static_cast<uint64_t>(a.token_bytes);
    };
    constexpr uint32_t kSixteens = (F::kStageRows + 15) / 16;  // that the wave's rows lie in
    struct Places {
      uint64_t at[kSixteens];
    };
    const auto places_of = [&](uint32_t t) {
      Places p;
#pragma unroll
      for (uint32_t k = 0; k < kSixteens; ++k) p.at[k] = sixteen_at(t, stage_row / 16 + k);
      return p;
    };
    const auto bring = [&](const char* from, const Places& p, char* to, auto swizzle) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t row = stage_row + i * kLoadRows;
        const uint64_t base = reinterpret_cast<uint64_t>(from) + p.at[i * kLoadRows / 16] + (row % 16) * static_cast<uint64_t>(a.token_bytes);
        const uint32_t offset = load_row * static_cast<uint32_t>(a.token_bytes) + ((load_chunk ^ swizzle(row + load_row)) * 16);
        load_to_lds(lds_address(to) + row * kRowBytes, base, offset);
      }
    };
    const auto bring_keys = [&](const Places& p, uint32_t buffer) { bring(kp, p, own + buffer * F::kBufferBytes, key_swizzle); };
    const auto bring_values = [&](const Places& p, uint32_t buffer) {
      bring(vp, p, own + buffer * F::kBufferBytes + kKeys * kRowBytes, value_swizzle);
    };
    // Empties rows of values that are in LDS.
    const auto mend = [&](uint32_t t, uint32_t buffer, uint64_t live) {
      if (live == kAll && !some_see(t)) return;
      char* values = own + buffer * F::kBufferBytes + kKeys * kRowBytes;
      for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t row = stage_row + load_row + i * kLoadRows;
        u32x4* at_lds = reinterpret_cast<u32x4*>(values + row * kRowBytes + load_chunk * 16);
        if (!kept(t, row, live, *at_lds)) *at_lds = zero;
      }
    };
    const auto ready = [&] {  // what is put is there for all that read it
      if constexpr (kRowWaves > 1)
        __syncthreads();
      else {  // the wave itself, whose LDS accesses are carried out in order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    };

    // queries: dims 16 s + 8 g .. + 7 (bf16), 8 s + 4 g .. + 3 (fp32) of the lane's row, negated for a negative scale
    u32x4 q[kSteps];
    {
      const char* qp = a.q + (static_cast<int64_t>(s.token + node) * a.q_token + static_cast<int64_t>(q_head) * a.q_head) * sizeof(T);
#pragma unroll
      for (uint32_t c = 0; c < kSteps; ++c) {
        q[c] = u32x4{0, 0, 0, 0};
        if (mine) q[c] = kAny ? load_chunk_of<T>(qp, (2 * c + g) * (16 / sizeof(T)), a.dim) : *reinterpret_cast<const u32x4_any*>(qp + (2 * c + g) * 16);
        if (a.scale < 0.0f) q[c] ^= kWide ? 0x80000000u : 0x80008000u;
      }
    }
    // a scale of 0 would make a NaN of a masked score: all weights are 1 with the smallest one as well
    const float scale = fmaxf(fabsf(a.scale), 1.17549435e-38f);

    float m = -INFINITY, l = 0.0f;
    f32x16 o[kOuts];
#pragma unroll
    for (uint32_t e = 0; e < kOuts; ++e) o[e] = f32x16{};

    int64_t place = -1;
    int32_t id = -1;
    uint64_t live, live_next = 0;
    Places next;
    if constexpr (kAny) {
      place = row_of(t_begin, id_of(t_begin));
      live = __ballot(place >= 0) & kAll;
      fetch(place);
      id = id_of(t_begin + 1);
    } else {
      live = live_of(t_begin);
    }
    __syncthreads();  // the item before is done with the LDS
    if (threadIdx.x == 0) odd_there[turn ^ 1] = 0;
    if constexpr (kAny) {
      put(t_begin, 0, live);
      place = row_of(t_begin + 1, id);
      live_next = __ballot(place >= 0) & kAll;
    } else {
      next = places_of(t_begin);
      bring_keys(next, 0);
      bring_values(next, 0);
      if constexpr (kRowWaves > 1) {
        loads_left<0>();
        mend(t_begin, 0, live);
      }
    }
    ready();

    uint32_t buffer = 0;
    for (uint32_t t = t_begin; t < t_end; ++t) {
      const bool more = t + 1 < t_end;
      const uint32_t other = (buffer + 1) % F::kBuffers;
      if constexpr (kAny) {
        if (more) fetch(place);
        id = id_of(t + 2);
      } else {
        if constexpr (kRowWaves > 1) {
          if (more) {
            live_next = live_of(t + 1);
            next = places_of(t + 1);
            bring_keys(next, other);
            bring_values(next, other);
          }
        } else {
          loads_left<kLoads>();  // the keys are there
          ready();
        }
      }
      const uint32_t key0 = t * kTile + kw * kKeys;
      const bool use = key0 < wave_end;
      const char* keys = own + buffer * F::kBufferBytes;
      const char* values = keys + kKeys * kRowBytes;
      f32x16 x[kBlocks];
      if (use) {
        u32x4 kf[kBlocks][kSteps];
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b)
#pragma unroll
          for (uint32_t c = 0; c < kSteps; ++c) kf[b][c] = *reinterpret_cast<const u32x4*>(keys + b * 32 * kRowBytes + (key_at ^ (c * 32)));
        __builtin_amdgcn_sched_barrier(0);  // all reads on their way before the first product waits for one
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b) {
          x[b] = f32x16{};
#pragma unroll
          for (uint32_t c = 0; c < kSteps; ++c) {
            if constexpr (kWide) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[b][c][e]), __uint_as_float(q[c][e]), x[b], 0, 0, 0);
            } else {
              x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[b][c]), __builtin_bit_cast(bf16x8, q[c]), x[b], 0, 0, 0);
            }
          }
        }
      }
      if constexpr (!kAny && kRowWaves == 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the keys are read
        ready();
        if (more) {
          live_next = live_of(t + 1);
          next = places_of(t + 1);
          bring_keys(next, 0);
          loads_left<kLoads>();  // the values are there
        } else {
          loads_left<0>();
        }
        mend(t, 0, live);
        ready();
      }
      if (use) {
        const bool some = key0 + kKeys > wave_sees || live != kAll;
        uint32_t see[kBlocks];
        if (some) {
#pragma unroll
          for (uint32_t b = 0; b < kBlocks; ++b) {
            const int32_t e0 = static_cast<int32_t>(key0 + 32 * b) - static_cast<int32_t>(s.cached);  // of the new tokens
            if (e0 <= -32) {
              see[b] = ~0u;
            } else if (a.seen == nullptr) {
              const int32_t n = static_cast<int32_t>(node) + 1 - e0;
              see[b] = n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1;
            } else {
              const uint64_t* words = a.seen + static_cast<int64_t>(s.token + node) * a.seen_stride;
              const auto word = [&](uint32_t w) { return mine && w < a.words ? words[w] : 0ull; };
              if (e0 < 0) {
                see[b] = ((1u << -e0) - 1) | static_cast<uint32_t>(word(0) << -e0);
              } else {
                const uint32_t w = static_cast<uint32_t>(e0) / 64, by = static_cast<uint32_t>(e0) % 64;
                uint64_t bits = word(w) >> by;
                if (by > 32) bits |= word(w + 1) << (64 - by);
                see[b] = static_cast<uint32_t>(bits);
              }
            }
            see[b] &= static_cast<uint32_t>(live >> (32 * b));
            const uint32_t shown = see[b] >> (4 * g);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[b][i] = shown >> (8 * (i / 4) + i % 4) & 1 ? x[b][i] : -INFINITY;
          }
        }
        // the values' operands, on their way while the weights are computed
        u32x4 vf[kWide ? 1 : kOuts][2];
        const auto read_values = [&](uint32_t b) {
          if constexpr (!kWide) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
            for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
              for (uint32_t c = 0; c < 2; ++c) {
                const char* from = values + (32 * b + 16 * c) * kRowBytes + (value_at ^ (e * 64));
                const u32x2 v0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from));
                const u32x2 v1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 8 * kRowBytes)));
                vf[e][c] = u32x4{v0.x, v0.y, v1.x, v1.y};
              }
          }
        };
        read_values(0);
        __builtin_amdgcn_sched_barrier(0);
        float top = x[0][0];
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
        top *= scale;
        if (__any(top > m)) {
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          top = fmaxf(top + kLazy, m);
          const float by = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);  // m = -inf: 0
          l *= by;
#pragma unroll
          for (uint32_t e = 0; e < kOuts; ++e) o[e] *= by;
          m = top;
        }
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b) {
          float p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][i], scale, -ref));
          l += ((p[0] + p[1]) + (p[2] + p[3]) + ((p[4] + p[5]) + (p[6] + p[7]))) + ((p[8] + p[9]) + (p[10] + p[11]) + ((p[12] + p[13]) + (p[14] + p[15])));
          const char* vb = values + b * 32 * kRowBytes;
          if constexpr (kWide) {
#pragma unroll
            for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float vf = *reinterpret_cast<const float*>(vb + value_at + (8 * (i / 4) + i % 4) * kRowBytes + e * 128);
                o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, p[i], o[e], 0, 0, 0);
              }
          } else {
            // weights as a sum of two bf16, 16 bits of each, so that only the output is rounded to 8. Both are positive: the largest
            // bf16 below the weight and what is left of it. A signed or empty rest would make a NaN of an infinite value.
            u32x4 hi[2], lo[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float p0 = p[2 * i], p1 = p[2 * i + 1];
              const uint32_t b0 = __builtin_elementwise_sub_sat(__float_as_uint(p0), 1u), b1 = __builtin_elementwise_sub_sat(__float_as_uint(p1), 1u);
              hi[i / 4][i % 4] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
              lo[i / 4][i % 4] = pack_bf16x2(p0 - __uint_as_float(b0 & 0xFFFF0000u), p1 - __uint_as_float(b1 & 0xFFFF0000u));
            }
            if (b == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
              for (uint32_t c = 0; c < 2; ++c) {
                const bf16x8 v = __builtin_bit_cast(bf16x8, vf[e][c]);
                o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, hi[c]), o[e], 0, 0, 0);
                o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, lo[c]), o[e], 0, 0, 0);
              }
            if (b + 1 < kBlocks) read_values(b + 1);
          }
        }
      }
      if constexpr (kAny) {
        if constexpr (F::kBuffers == 1) ready();  // with the tile
        if (more) put(t + 1, other, live_next);
        place = row_of(t + 2, id);
        live = live_next;
        live_next = __ballot(place >= 0) & kAll;
      } else {
        if constexpr (kRowWaves > 1) {
          loads_left<0>();
          if (more) mend(t + 1, other, live_next);
        } else {
          asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the values are read
          ready();
          if (more) bring_values(next, 0);
        }
        live = live_next;
      }
      buffer = other;
      ready();
    }
    if constexpr (kRowWaves == 1) __syncthreads();
    // Values with an infinity or a NaN in tiles that only some rows see: one key at a time, for the rows that see it. Its score is
    // in m and l already.
    if (odd_there[turn] != 0) {
      for (uint32_t t = t_begin; t < t_end; ++t) {
        if (!some_see(t)) continue;
        for (uint32_t j = t * kTile + kw * kKeys; j < min(t * kTile + (kw + 1) * kKeys, wave_end); ++j) {
          const int32_t page = ids[page_of(j)];
          if (static_cast<uint32_t>(page) >= a.pages) continue;
          const int64_t at_row = page * a.page_bytes + static_cast<int64_t>(j - page_of(j) * a.page_tokens) * a.token_bytes;
          const T* key = reinterpret_cast<const T*>(kp + at_row);
          const T* value = reinterpret_cast<const T*>(vp + at_row);
          bool odd = false;
          for (uint32_t dim = lane; dim < a.dim; dim += kWave) {
            const float v = S::load1(value + dim);
            odd = odd || !(fabsf(v) <= 3.402823466e38f);
          }
          if (__ballot(odd) == 0) continue;
          const int32_t e = static_cast<int32_t>(j) - static_cast<int32_t>(s.cached);
          bool sees_it = mine && e < 0;
          if (mine && e >= 0)
            sees_it = a.seen == nullptr ? static_cast<uint32_t>(e) <= node
                                        : static_cast<uint32_t>(e) / 64 < a.words &&
                                              (a.seen[static_cast<int64_t>(s.token + node) * a.seen_stride + e / 64] >> (e % 64) & 1);
          if (!sees_it) continue;
          const T* query = reinterpret_cast<const T*>(a.q) + static_cast<int64_t>(s.token + node) * a.q_token + static_cast<int64_t>(q_head) * a.q_head;
          float score = 0.0f;
          for (uint32_t dim = 0; dim < a.dim; ++dim) score = __builtin_fmaf(S::load1(query + dim), S::load1(key + dim), score);
          const float weight = __builtin_amdgcn_exp2f(__builtin_fmaf(a.scale < 0.0f ? -score : score, scale, -m));
#pragma unroll
          for (uint32_t c = 0; c < kOuts; ++c)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
              const uint32_t dim = 32 * c + 8 * (i / 4) + 4 * g + i % 4;
              if (!kAny || dim < a.dim) o[c][i] += weight * S::load1(value + dim);
            }
        }
      }
    }
    l += __shfl_xor(l, 32, 64);

    // Waves with the same rows join theirs in LDS: two and two, then the two.
    if constexpr (F::kKeyWaves > 1) {
      constexpr uint32_t kRow = kDim + 4;
      float* rest = reinterpret_cast<float*>(lds);
#pragma unroll
      for (uint32_t n = F::kKeyWaves / 2; n > 0; n /= 2) {
        __syncthreads();
        if (kw >= n && kw < 2 * n) {
          if (g == 0) merge_sums[kw - n][r] = make_float2(m, l);
#pragma unroll
          for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
            for (uint32_t i = 0; i < 16; i += 4)
              *reinterpret_cast<f32x4*>(rest + ((kw - n) * 32 + r) * kRow + 32 * e + 2 * i + 4 * g) = f32x4{o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]};
        }
        __syncthreads();
        if (kw < n) {
          const float2 ml = merge_sums[kw][r];
          const float all = fmaxf(m, ml.x), ref = all == -INFINITY ? 0.0f : all;
          const float s0 = __builtin_amdgcn_exp2f(m - ref), s1 = __builtin_amdgcn_exp2f(ml.x - ref);
          l = l * s0 + ml.y * s1;
          m = all;
#pragma unroll
          for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
            for (uint32_t i = 0; i < 16; i += 4) {
              const f32x4 theirs = *reinterpret_cast<const f32x4*>(rest + (kw * 32 + r) * kRow + 32 * e + 2 * i + 4 * g);
#pragma unroll
              for (uint32_t n4 = 0; n4 < 4; ++n4) o[e][i + n4] = o[e][i + n4] * s0 + theirs[n4] * s1;
            }
        }
      }
    }

    const bool whole = t_begin == 0 && t_end == tiles;
    if (t_end == tiles && threadIdx.x == 0 && item < a.most_items) {
      const uint32_t first = t_begin == 0 ? worker : runs.worker_of(item_first);
      const uint32_t slot = runs.first(first) == item_first ? 0 : 1;
      a.items[item] = Item{2 * first + slot, worker, s.token, row0, in_block, head, {0, 0}};
    }
    if (kw == 0 && mine) {
      float* part = part_at<kRows>(a, worker, at == begin ? 0 : 1) + static_cast<size_t>(rw * 32 + r) * a.part_row;
      if (!whole && g == 0) *reinterpret_cast<float2*>(part) = make_float2(m, l);
#pragma unroll
      for (uint32_t e = 0; e < kOuts; ++e)
#pragma unroll
        for (uint32_t i = 0; i < 16; i += 4) {
          const uint32_t dim = 32 * e + 2 * i + 4 * g;
          const f32x4 four = {o[e][i], o[e][i + 1], o[e][i + 2], o[e][i + 3]};
          if (whole)
            write_row<S>(a, s.token + node, q_head, dim, m, l, four);
          else if (!kAny || dim < a.dim)
            *reinterpret_cast<f32x4*>(part + 4 + dim) = four;
        }
    }
    // the next item
    at = item_first + t_end;
    if (t_end == tiles) {
      item_first += tiles;
      if (item < a.most_items) ++item;
      if (++block == s.blocks) {
        block = 0;
        if (++head == a.heads) {
          head = 0;
          if (at < end)
            do s = seq_of<kRows>(a, ++seq);
            while (s.blocks == 0);  // `at` < the total: one with tiles follows
        }
      }
    }
  }
}

// Joins the parts of items that were split. A workgroup takes every gridDim.x-th item; a thread has four dims of a row.
template <class S, uint32_t kRows>
__global__ void __launch_bounds__(kThreads) join_kernel(const Attend a) {
  const uint32_t items = *a.item_count, quads = (a.dim + 3) / 4;
  for (uint32_t i = blockIdx.x; i < items; i += gridDim.x) {
    const Item it = a.items[i];
    const uint32_t first = it.first_slot / 2, slot = it.first_slot & 1;
    if (it.last == first) continue;
    for (uint32_t e = blockIdx.y * kThreads + threadIdx.x; e < it.rows * quads; e += gridDim.y * kThreads) {
      const uint32_t row = e / quads, dim = (e - row * quads) * 4;
      float m = -INFINITY, l = 0.0f;
      f32x4 o = {0, 0, 0, 0};
#pragma unroll 4
      for (uint32_t w = first; w <= it.last; ++w) {
        const float* part = part_at<kRows>(a, w, w == first ? slot : 0) + static_cast<size_t>(row) * a.part_row;
        const float2 ml = *reinterpret_cast<const float2*>(part);
        const f32x4 po = *reinterpret_cast<const f32x4*>(part + 4 + dim);
        const float top = fmaxf(m, ml.x), ref = top == -INFINITY ? 0.0f : top;
        const float s0 = __builtin_amdgcn_exp2f(m - ref), s1 = __builtin_amdgcn_exp2f(ml.x - ref);
        l = l * s0 + ml.y * s1;
        o = o * s0 + po * s1;
        m = top;
      }
      const uint32_t node = node_of(a, it.row + row);
      write_row<S>(a, it.token + node, it.head * a.group + it.row + row - node * a.group, dim, m, l, o);
    }
  }
}

template <class S, uint32_t kDim, uint32_t kRowWaves, bool kAny>
int launch(Attend& a, hipStream_t st) {
  typedef Form<S, kDim, kRowWaves, kAny> F;
  if (F::kLds > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(&attend_kernel<S, kDim, kRowWaves, kAny>), hipFuncAttributeMaxDynamicSharedMemorySize,
                          F::kLds) != hipSuccess)
    return ZO_ERR_HIP;
  attend_kernel<S, kDim, kRowWaves, kAny><<<dim3(a.workers), dim3(kThreads), F::kLds, st>>>(a);
  const int rc = launched();
  if (rc != ZO_OK) return rc;
  const uint32_t parts = std::max(1u, std::min(16u, F::kRows * ((a.dim + 3) / 4) / kThreads));
  join_kernel<S, F::kRows><<<dim3(std::min(a.most_items, 1024u), parts), dim3(kThreads), 0, st>>>(a);
  return launched();
}

template <class S, uint32_t kDim, bool kAny>
int rows(Attend& a, uint32_t row_waves, hipStream_t st) {
  if constexpr (kDim * sizeof(typename S::storage) <= 512) {
    if (row_waves == 1) return launch<S, kDim, 1, kAny>(a, st);
  }
  return launch<S, kDim, 4, kAny>(a, st);
}

template <class S>
int attend(Attend& a, uint32_t row_waves, hipStream_t st) {
  // pages of whole sixteens, in which 32-bit offsets reach every row, at vectors' addresses
  const uint64_t places = reinterpret_cast<uint64_t>(a.k) | reinterpret_cast<uint64_t>(a.v) | a.page_bytes | a.head_bytes | a.token_bytes;
  const bool fast = a.page_tokens % 16 == 0 && places % 16 == 0 && a.token_bytes < (int64_t{1} << 28);
  if (fast && a.dim == 64) return rows<S, 64, false>(a, row_waves, st);
  if (fast && a.dim == 128) return rows<S, 128, false>(a, row_waves, st);
  if (fast && a.dim == 256) return rows<S, 256, false>(a, row_waves, st);
  if (a.dim <= 64) return rows<S, 64, true>(a, row_waves, st);
  if (a.dim <= 128) return rows<S, 128, true>(a, row_waves, st);
  return rows<S, 256, true>(a, row_waves, st);
}

}  // namespace
}  // namespace zo

extern "C" int zo_tree_attend(const zo_tree_attention* p, void* stream) {
  using namespace zo;
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = check_tree_attend(*p);
  if (rc != ZO_OK) return rc;
  if (p->table.seqs == 0 || p->tokens == 0 || p->q_heads == 0) return ZO_OK;
  const TreeShape shape = tree_shape(p->tokens, p->table.seqs, p->q_heads, p->cache.heads, p->cache.dim, p->dtype);
  const int64_t elem = static_cast<int64_t>(elem_bytes(p->dtype));
  Attend a;
  a.q = static_cast<const char*>(p->q.data);
  a.k = static_cast<const char*>(p->cache.k);
  a.v = static_cast<const char*>(p->cache.v);
  a.out = static_cast<char*>(p->out.data);
  a.lse = p->lse;
  char* work = static_cast<char*>(p->work);
  a.item_count = reinterpret_cast<uint32_t*>(work);
  a.items = reinterpret_cast<Item*>(work + 16);
  a.parts = reinterpret_cast<float*>(work + 16 + shape.items * sizeof(Item));
  a.ids = p->table.ids;
  a.lengths = p->lengths;
  a.starts = p->starts;
  a.seen = p->seen;
  a.seen_stride = p->seen_stride;
  a.q_token = p->q.token_stride;
  a.q_head = p->q.head_stride;
  a.out_token = p->out.token_stride;
  a.out_head = p->out.head_stride;
  a.page_bytes = p->cache.page_stride * elem;
  a.head_bytes = p->cache.head_stride * elem;
  a.token_bytes = p->cache.token_stride * elem;
  a.table_stride = p->table.stride;
  a.group = p->q_heads / p->cache.heads;
  a.inv_group = 1.0 / a.group;
  a.most_items = static_cast<uint32_t>(shape.items);
  a.tokens = p->tokens;
  a.words = p->words;
  a.seqs = p->table.seqs;
  a.width = p->table.width;
  a.pages = p->cache.pages;
  a.page_tokens = p->cache.page_tokens;
  a.page_shift = (a.page_tokens & (a.page_tokens - 1)) == 0 ? __builtin_ctz(a.page_tokens) : -1;
  a.heads = p->cache.heads;
  a.dim = p->cache.dim;
  a.workers = shape.workers;
  a.part_row = (a.dim + 3) / 4 * 4 + 4;
  a.scale = p->scale * 1.4426950408889634f;
  (void)hipGetLastError();
  hipStream_t st = static_cast<hipStream_t>(stream);
  return p->dtype == ZO_F32 ? attend<F32>(a, shape.row_waves, st) : attend<BF16>(a, shape.row_waves, st);
}
