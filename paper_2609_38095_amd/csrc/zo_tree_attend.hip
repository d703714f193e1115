// Attention of several new tokens of each sequence over the paged cache, for gfx950: drafted trees and prompts.
//
// Mathematics. As for one token (zo_attend.hip): one pass over the keys with a running bound m of the scores and a sum l, p_j =
// 2^(x_j - m), o = sum p_j v_j; only a score above the bound raises it, to 8 above the largest. What is new are the rows: a row
// is a new token and a query head of one key head's group, so rows share keys, and each sees its own of the sequence's new tokens.
//
// Split. An item is a sequence, a key head and kRows rows; it is cut into tiles of kTile tokens up to the last one that a row of
// it can see. The tiles of all items, in order, are dealt out in equal runs to the workgroups, which find theirs from
// lengths and starts by themselves; an item's own time (first loads, results) counts as a few tiles more. A run that covers an item writes
// its output, others leave (m, l, o) in the workspace, at most two parts for each workgroup, and join_kernel joins them. Runs
// that follow each other, which read the same keys, lie on one XCD.
//
// Tile. S^T = K Q^T and O^T = V^T P^T in 32 x 32 products, a row in each lane (r = lane % 32), so a row's bound and sum stay in
// its two lanes (g = lane / 32). A wave has 32 rows. kRowWaves = 8 or 4: the waves have different rows and share a tile's keys and
// values, two buffers of them in LDS; kRowWaves = 1 (sequences of few rows): four waves have the same rows and a quarter of the
// tile's keys each, in LDS of their own, without a barrier; they join at an item's end. Which form is taken is measured in tree_shape().
//   - Keys and values go straight into LDS, 16 bytes a lane, a tile ahead of their use (through registers: prompts 2,198 us, this way
//     1,847 at that step). LDS rows are swizzled by 16-byte chunks, so that few reads meet in a bank;
//   - S^T leaves in lane (r, g) the keys 8 i + 4 g .. + 3: the second product's operand as it is, if the contraction's index
//     is permuted alike; the values' operand is read by the transposing LDS read (bf16), four keys of 16 dims at a time.
//   - bf16 heads of 64 and 128 in more than one row wave run as a pipeline of 32 keys (step()): the products of one block's scores and of
//     another's weights with the values lie under the exponentials of the one between, one barrier a tile (prompts 1,847 -> 1,342 us).
//
// What a row does not see. Scores are masked, and values that no row of the call may use are zeros in LDS. A value that is infinite or
// NaN in a tile that only some of the rows see would reach the others as 0 times itself: it is a zero in LDS too, and is
// added to the results of the rows that see it after these are written.
//
// Rounding. fp32 sums and bounds. bf16 weights are a sum of two bf16 (2^-16 of a weight is lost), two products with the values each: weights
// rounded once would be 2^-8 of the weighted magnitudes, as much as the output's own rounding, for 1,060 instead of 1,342 us (prompts).
//
// Measured, heads of 128: four prompts of up to 6,001 tokens of 32 heads on 8 behind up to 2,048, 1,342 to 1,392 us (1.12 to 1.16 PFLOP/s
// with the second parts' products; a large matrix product reaches 1.20); 48 trees of up to 64 behind up to 4,096, 204 to 207 us (2.9 TB/s:
// 1.5 to 2.5 us a tile, 14 an item, 15 the join); one tree of 12 behind 1,037, 15.8 to 16.5 us (latencies: the deal 2.6 us, first loads 4,
// results 5, the join 4). fp32 trees, 16 of up to 23, 32 heads of 64 behind up to 2,050: 85 to 86 us (4.4 TB/s).

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "zo_checks.h"
#include "zo_lanes.h"
#include "zo_tree_deal.h"

namespace zo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kThreads = 256, kWave = 64, kWaves = kThreads / kWave, kXcds = 8;
constexpr float kLazy = 8.0f;  // how far (in powers of two) the bound of the scores is set above their maximum
// Scores from here on are rounded before the bound is taken from them. Below, an unrounded product differs from its rounding, which the bound is
// made of, by half at most; at 2^125 all weights of a row would be 0 or infinite for that.
constexpr float kLarge = 16777216.0f;

// An item that was split: its parts are those of the workgroup that this is the entry of, in slot 1, and of the ones up to `last`, in
// slot 0. At most one item that is split begins in a workgroup's run. last = 0: none does. Written by the workgroup of the item's last
// tile, or by the entry's own workgroup where none is split.
struct Split {
  uint32_t last;
  uint32_t token, row, rows, head;  // the sequence's first new token; the item's first row and their number; key head
  uint32_t unused[3];
};
static_assert(sizeof(Split) == kTreeSplitWords * 4, "the workspace holds entries of this size");

struct Attend : Batch {
  const char *q, *k, *v;
  char* out;
  float* lse;
  uint32_t* active;  // workgroups that have tiles
  Split* splits;
  float* parts;
  const int32_t* ids;
  int64_t seen_stride, q_token, q_head, out_token, out_head, page_bytes, head_bytes, token_bytes, table_stride;
  double inv_page;  // of a page's sixteens
  uint32_t words, pages, dim, workers, part_row;
  float scale;         // times log2(e)
};

// A value that all lanes of a wave hold, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return static_cast<uint64_t>(uniform(static_cast<uint32_t>(v >> 32))) << 32 | uniform(static_cast<uint32_t>(v));
}

// A sequence in scalar registers.
__device__ __forceinline__ Seq uniform(const Seq& s) {
  return {uniform(s.token), uniform(s.count), uniform(s.cached), uniform(s.len), uniform(s.blocks)};
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

// The deal's sums by all lanes of a wave together.
template <uint32_t kRows>
struct Lanes {
  const Batch& batch;
  const Seq* seqs;  // in LDS, where each thread has one; else NULL
  uint32_t lane;
  __device__ __forceinline__ Seq seq(uint32_t n) const { return uniform(seqs ? seqs[n] : seq_of<kRows>(batch, n)); }
  template <class F>
  __device__ __forceinline__ uint64_t sum(uint32_t n, const F& f) const {
    uint64_t mine = 0;
    for (uint32_t i = lane; i < n; i += kWave) mine += f(i);
    return uniform(__shfl(sums_upto(mine, lane), 63, 64));
  }
  template <class F>
  __device__ __forceinline__ bool first_over(uint32_t n, uint64_t rest, const F& f, uint32_t& at, uint64_t& before) const {
    before = 0;
    for (uint32_t i = 0; i < n; i += kWave) {
      const uint32_t mine = i + lane < n ? f(i + lane) : 0;
      const uint64_t upto = sums_upto(mine, lane), over = __ballot(before + upto > rest);
      if (over != 0) {
        const uint32_t l = static_cast<uint32_t>(__builtin_ctzll(over));
        at = i + l;
        before += uniform(__shfl(upto - mine, l, 64));
        return true;
      }
      before += uniform(__shfl(upto, 63, 64));
    }
    return false;
  }
};

// The cost before each thread's sequences, and the sequences where each thread has one. Thread t counts sequences [t each, (t + 1) each).
struct Deal {
  uint64_t total;
  uint32_t each;
};

template <uint32_t kRows, uint32_t kTile, uint32_t kThreads>
__device__ Deal deal(const Attend& a, uint64_t* before, Seq* seqs) {
  constexpr uint32_t kWaves = kThreads / kWave;
  __shared__ uint64_t wave_cost[kWaves];
  const uint32_t lane = threadIdx.x % kWave;
  Deal d;
  d.each = (a.seqs + kThreads - 1) / kThreads;
  uint64_t cost = 0;
  for (uint32_t i = 0; i < d.each; ++i) {
    const uint32_t seq = threadIdx.x * d.each + i;
    Seq s = {};
    if (seq < a.seqs) s = seq_of<kRows>(a, seq);
    if (d.each == 1) seqs[threadIdx.x] = s;
    // Blocks that a thread counts by itself; a longer sequence's by the whole wave. 300 chains of 100, 32 heads on 8 of 64: 223 us, with
    // all by the wave 281, with up to 64 by a thread 224.
    constexpr uint32_t kFew = 8;
    if (a.seen) {
      if (s.blocks) cost += static_cast<uint64_t>(s.blocks) * cost_of<kRows, kTile>(a, s, 0);
    } else {
      if (s.blocks <= kFew)
        for (uint32_t b = 0; b < s.blocks; ++b) cost += cost_of<kRows, kTile>(a, s, b);
      for (uint64_t left = __ballot(s.blocks > kFew); left != 0; left &= left - 1) {
        const uint32_t from = static_cast<uint32_t>(__builtin_ctzll(left));
        Seq one;
        one.token = 0;
        one.count = __builtin_amdgcn_readlane(s.count, from);
        one.cached = __builtin_amdgcn_readlane(s.cached, from);
        one.len = __builtin_amdgcn_readlane(s.len, from);
        one.blocks = __builtin_amdgcn_readlane(s.blocks, from);
        const uint64_t all = head_cost<kRows, kTile>(a, one, Lanes<kRows>{a, nullptr, lane});
        if (lane == from) cost += all;
      }
    }
  }
  const uint64_t upto = sums_upto(cost, lane);
  if (lane == 63) wave_cost[threadIdx.x / kWave] = upto;
  __syncthreads();
  uint64_t at = 0, all = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < threadIdx.x / kWave) at += wave_cost[w];
    all += wave_cost[w];
  }
  before[threadIdx.x] = (at + upto - cost) * a.heads;
  d.total = uniform(all * a.heads);
  __syncthreads();
  return d;
}

// A part in the workspace: for each row [m, l, -, -, o[dim]].
template <uint32_t kRows>
__device__ __forceinline__ float* part_at(const Attend& a, uint32_t worker, uint32_t slot) {
  return a.parts + (static_cast<size_t>(worker) * 2 + slot) * kRows * a.part_row;
}

// Whether a row with the sum l of weights saw anything (a NaN among its scores counts).
__device__ __forceinline__ bool any_seen(float l) { return l > 0.0f || l != l; }

// Four dims of a row's output. Where weights were rounded a mean of the largest bf16 values can come out above them: it is the largest one.
template <class T>
__device__ __forceinline__ void store_four(T* to, f32x4 four) {
  if constexpr (sizeof(T) == 2) {
    constexpr float kMost = 3.3895313892515355e38f;
#pragma unroll
    for (int i = 0; i < 4; ++i) four[i] = fabsf(four[i]) <= 3.402823466e38f ? __builtin_amdgcn_fmed3f(four[i], -kMost, kMost) : four[i];
  }
  if constexpr (sizeof(T) == 4) {
    typedef f32x4 __attribute__((aligned(4))) f32x4_any;
    *reinterpret_cast<f32x4_any*>(to) = four;
  } else {
    typedef u32x2 __attribute__((aligned(2))) u32x2_any;
    *reinterpret_cast<u32x2_any*>(to) = u32x2{pack_bf16x2(four[0], four[1]), pack_bf16x2(four[2], four[3])};
  }
}

// The log-sum of a row's scores.
__device__ __forceinline__ float log_sum(float m, float l) { return any_seen(l) ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY; }

// Sixteen bytes of values with zeros for those that are infinite or NaN.
template <class T>
__device__ __forceinline__ u32x4 without_odd(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] &= 0xFFFFu;
      if ((v[i] & 0x7F80u) == 0x7F80u) v[i] &= 0xFFFF0000u;
    } else {
      if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] = 0;
    }
  }
  return v;
}

// A weight as a sum of two bf16, 16 bits of it, so that only the output is rounded to 8. Both parts are positive: the largest bf16 below
// the weight and what is left of it. A signed or empty rest would make a NaN of an infinite value. below(p) holds the first part's bits.
__device__ __forceinline__ uint32_t below(float p) { return __builtin_elementwise_sub_sat(__float_as_uint(p), 1u); }
__device__ __forceinline__ uint32_t first_parts(uint32_t b0, uint32_t b1) { return __builtin_amdgcn_perm(b1, b0, 0x07060302u); }
__device__ __forceinline__ uint32_t rests_of(float p0, float p1, uint32_t b0, uint32_t b1) {
  return pack_bf16x2(p0 - __uint_as_float(b0 & 0xFFFF0000u), p1 - __uint_as_float(b1 & 0xFFFF0000u));
}

// The kernel's arguments read anew: a copy of its own for each part of the kernel, so that those of one part do not hold (and spill) the
// scalar registers of another.
__device__ __forceinline__ Attend arguments() {
  typedef const __attribute__((address_space(4))) Attend* Arguments;
  Arguments from = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(from));
  return *(const Attend*)from;
}

template <class S, uint32_t kDim, uint32_t kRowWaves>
struct Form {
  typedef typename S::storage T;
  static constexpr uint32_t kRowBytes = kDim * sizeof(T), kChunks = kRowBytes / 16;
  static constexpr uint32_t kWaves = kRowWaves > 4 ? kRowWaves : 4, kThreads = kWaves * kWave;
  static constexpr uint32_t kRows = 32 * kRowWaves, kKeyWaves = kWaves / kRowWaves;
  static constexpr uint32_t kBlocks = kRowWaves > 1 && kRowBytes <= 256 ? 2 : 1;  // of 32 keys, of a wave in a tile
  static constexpr uint32_t kKeys = 32 * kBlocks, kTile = kKeys * kKeyWaves;
  static constexpr uint32_t kStageRows = kKeys / kRowWaves;          // rows that a wave brings
  static constexpr uint32_t kLoadRows = kWave / kChunks;             // rows of a load of all lanes
  static constexpr uint32_t kLoads = kStageRows / kLoadRows;         // of the keys, and as many of the values
  static constexpr uint32_t kBuffers = kRowWaves > 1 ? 2 : 1;
  static constexpr uint32_t kBufferBytes = 2 * kTile * kRowBytes;
  static constexpr uint32_t kLds = kBuffers * kBufferBytes;
  static constexpr bool kPiped = kRowWaves > 1 && sizeof(T) == 2 && kBlocks == 2;
  // An item's own time in tiles. 0: prompts 1,415 us, 48 trees 229, fp32 trees (one row wave) 93; 1: 1,399, 217, 86; 2: 1,381, 221, 87;
  // 4: 1,359, 204, 90; 6: 1,351, 205, 91.
  static constexpr uint32_t kVisit = kRowWaves > 1 ? 4 : 1;
  static constexpr uint32_t kSimdWaves = kRowBytes <= 256 ? 2 : 1;
  static_assert(kLoadRows <= 8 && kStageRows % kLoadRows == 0, "a load's rows lie in one sixteen");
};

typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ uint32_t lds_address(const char* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char*)p)); }

// Sixteen bytes of each lane from base + offset straight into LDS, one lane behind another from `to` on. The compiler does not
// count these loads: loads_left() waits for them.
__device__ __forceinline__ void load_to_lds(uint32_t to, uint64_t base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(uniform(to)), "v"(offset), "s"(uniform(base)) : "memory", "m0");
}
template <int kLeft>
__device__ __forceinline__ void loads_left() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLeft) : "memory");
  // The same, for the compiler: what it brought back from scratch memory before a loop is there as well, and it adds no waits inside the
  // loop, which would be for all of the wave's loads (48 trees, weights of one part: 199 -> 173 us).
  __builtin_amdgcn_s_waitcnt(kLeft % 16 | 7 << 4 | 15 << 8 | kLeft / 16 << 14);
}

// Heads of kDim, pages of whole sixteens of tokens, rows at 16-byte aligned places.
template <class S, uint32_t kDim, uint32_t kRowWaves>
__global__ void __launch_bounds__((Form<S, kDim, kRowWaves>::kThreads), (Form<S, kDim, kRowWaves>::kSimdWaves)) attend_kernel(const Attend) {
  typedef Form<S, kDim, kRowWaves> F;
  typedef typename S::storage T;
  constexpr bool kWide = sizeof(T) == 4;
  constexpr uint32_t kRowBytes = F::kRowBytes, kChunks = F::kChunks, kRows = F::kRows, kBlocks = F::kBlocks, kKeys = F::kKeys;
  constexpr uint32_t kTile = F::kTile, kLoads = F::kLoads, kLoadRows = F::kLoadRows, kOuts = kDim / 32, kSteps = kChunks / 2;
  extern __shared__ __align__(16) char lds[];
  __shared__ uint64_t before[F::kThreads];
  __shared__ Seq seqs[F::kThreads];
  __shared__ uint32_t odd_there[2];  // odd values in this item's tiles, and emptied for the next item's
  __shared__ float2 sums[F::kWaves][32];

  const uint32_t wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 32, g = lane / 32;
  const uint32_t rw = wave % kRowWaves, kw = wave / kRowWaves;  // which rows, which keys
  Deal d;
  uint32_t workers;
  {
    const Attend a = arguments();
    d = deal<kRows, kTile, F::kThreads>(a, before, seqs);
    workers = a.workers;
  }
  Runs runs(d.total, workers);
  runs.each = uniform(runs.each);
  if (blockIdx.x == 0 && threadIdx.x == 0) *arguments().active = d.total > 0 ? runs.workers : 0;
  // neighbouring runs on one XCD: workgroup b runs on XCD b % 8
  const uint32_t per_xcd = (runs.workers + kXcds - 1) / kXcds;
  const uint32_t slot_of = blockIdx.x / kXcds, worker = blockIdx.x % kXcds * per_xcd + slot_of;
  if (slot_of >= per_xcd || worker >= runs.workers) return;
  const uint64_t begin = uniform(runs.first(worker)), end = uniform(runs.first(worker + 1));
  uint64_t at = begin;
  if (at >= end) return;

  // the sequence, key head and block that `at` lies in
  const Seq* lds_seqs = d.each == 1 ? seqs : nullptr;
  Item item;
  {
    const Attend a = arguments();
    uint32_t chunk = 0;  // the last thread's sequences that begin at or before it
#pragma unroll
    for (uint32_t step = F::kThreads / 2; step > 0; step /= 2)
      if (before[chunk + step] <= at) chunk += step;
    chunk = uniform(chunk);
    if (!seek<kRows, kTile>(a, chunk * d.each, uniform(before[chunk]), at, Lanes<kRows>{a, lds_seqs, lane}, item)) return;
    item.head = uniform(item.head);
    item.block = uniform(item.block);
    item.first = uniform(item.first);
  }

  // LDS places of the lane's shares: of the rows that it brings, of the key and of the values that it uses
  const uint32_t stage_row = rw * F::kStageRows, load_row = lane / kChunks, load_chunk = lane % kChunks;
  char* own = lds + kw * 2 * kKeys * kRowBytes;  // the keys of the waves that share them, and their values behind these
  // Rows are swizzled by 16-byte chunks: eight neighbouring rows' same chunks (the keys' reads), and four rows' four chunks (the values')
  // lie in different banks. The keys' still meet a third of the time: lanes are served in groups of rows 0-3, 12-15, 20-23 and 24-27. A swizzle of
  // theirs over sixteen rows ends that, and the offsets of two swizzles cost registers (weights of one part: prompts 1,074 -> 1,069 us, 48
  // trees 175 -> 178).
  const auto swizzle = [](uint32_t row) {
    return kChunks >= 16 ? row % 4 * 4 + row / 4 % 2 : row / 2 % 2 * 4 + row / 4 % 2;
  };
  const auto value_swizzle = [&](uint32_t row) { return kWide ? 0u : swizzle(row); };
  const uint32_t key_at = r * kRowBytes + ((g ^ swizzle(r)) * 16);
  uint32_t value_at;
  if constexpr (kWide) {
    value_at = 4 * g * kRowBytes + r * 4;
  } else {
    const uint32_t row = 4 * g + lane % 16 / 4;
    value_at = row * kRowBytes + ((lane / 16 % 2 * 2 + lane % 4 / 2) ^ swizzle(row)) * 16 + lane % 2 * 8;
  }

  if (threadIdx.x == 0) odd_there[0] = 0;
  for (uint32_t turn = 0; at < end && item.first < end; turn ^= 1) {
    const Attend a = arguments();
    const Seq& s = item.s;
    const uint32_t seq = item.seq, head = item.head, block = item.block;
    const uint64_t item_first = item.first;
    const uint32_t rows = s.count * a.group, row0 = block * kRows, in_block = min(kRows, rows - row0);
    const uint32_t sees = uniform(visible(a, s, row0 + kRows));
    const uint32_t tiles = max(1u, (sees + kTile - 1) / kTile);
    const Share share(at, end, item_first, tiles);
    const uint32_t t_begin = uniform(share.begin), t_end = uniform(share.end);
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

    // The page of a token (tokens below 2^31, in sixteens: the product's error stays below the half's share).
    const auto page_of = [&](uint32_t j) { return static_cast<uint32_t>((static_cast<double>(j / 16) + 0.5) * a.inv_page); };
    constexpr uint64_t kAll = kKeys == 64 ? ~0ull : (1ull << (kKeys % 64)) - 1;
    // Whether values of the tile may have to be emptied: not all rows see all of its keys.
    const auto some_see = [&](uint32_t t) { return t * kTile + kTile > all_see; };
    // Where 64 sixteens of tokens lie, one in each lane, found at once; the next 64's page ids are on their way. Rows of an absent
    // page are read from page 0, those behind the last token are inside their page.
    uint64_t lane_place = 0;                  // bytes from a tensor's first row
    uint32_t lane_count = 0, lane_ids = ~0u;  // live tokens; which 64 these are
    uint64_t whole_sixteens = 0;              // whose tokens are all live
    int32_t coming_id = -1;                   // of the next 64
    const auto sixteen_of = [&](uint32_t t) { return t * (kTile / 16) + kw * (kKeys / 16); };
    const auto sixteens_id = [&](uint32_t which) {
      const uint32_t j = (which * 64 + lane) * 16;
      return j < sees ? ids[page_of(j)] : -1;
    };
    const auto find_sixteens = [&](uint32_t which, int32_t id) {
      const uint32_t j = (which * 64 + lane) * 16;
      const bool there = static_cast<uint32_t>(id) < a.pages;  // so j < sees
      lane_place = there ? id * a.page_bytes + static_cast<int64_t>(j - page_of(j) * a.page_tokens) * a.token_bytes : 0;
      lane_count = there ? min(16u, sees - j) : 0u;
      whole_sixteens = __ballot(lane_count == 16);
      lane_ids = which;
      coming_id = sixteens_id(which + 1);
    };
    constexpr uint32_t kSixteens = (F::kStageRows + 15) / 16;  // that the rows that a wave brings lie in
    struct Places {
      uint64_t at[kSixteens];
      uint64_t live;  // the wave's keys of the tile
    };
    const auto places_of = [&](uint32_t t) {
      const uint32_t first = sixteen_of(t), at = first % 64;
      if (first / 64 != lane_ids) find_sixteens(first / 64, coming_id);
      Places p;
#pragma unroll
      for (uint32_t k = 0; k < kSixteens; ++k) {
        const uint32_t from = at + stage_row / 16 + k;
        p.at[k] = static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(lane_place >> 32), from)) << 32 |
                  static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(lane_place), from));
      }
      p.live = kAll;
      if ((~(whole_sixteens >> at) & ((1u << (kKeys / 16)) - 1)) != 0) {
        p.live = 0;
        for (uint32_t k = 0; k < kKeys / 16; ++k)
          p.live |= static_cast<uint64_t>((1u << __builtin_amdgcn_readlane(lane_count, at + k)) - 1) << (16 * k);
      }
      return p;
    };
    const auto offset_of = [&](uint32_t i, auto swizzle) {  // of the lane's share of load i, from its sixteen's first row
      const uint32_t row = stage_row + i * kLoadRows + load_row;
      return row % 16 * static_cast<uint32_t>(a.token_bytes) + ((load_chunk ^ swizzle(row)) * 16);
    };
    const auto bring = [&](const char* from, const Places& p, char* to, auto swizzle) {
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i)
        load_to_lds(lds_address(to) + (stage_row + i * kLoadRows) * kRowBytes, reinterpret_cast<uint64_t>(from) + p.at[i * kLoadRows / 16],
                    offset_of(i, swizzle));
    };
    const auto bring_keys = [&](const Places& p, uint32_t buffer) { bring(kp, p, own + buffer * F::kBufferBytes, swizzle); };
    const auto bring_values = [&](const Places& p, uint32_t buffer) {
      bring(vp, p, own + buffer * F::kBufferBytes + kKeys * kRowBytes, value_swizzle);
    };
    // Values of the lane's that are in LDS, as the products may meet them: zeros where the row is dead, and for infinities and NaN in a
    // tile that only some rows see.
    const auto mend = [&](uint32_t t, uint32_t buffer, uint64_t live) {
      if (live == kAll && !some_see(t)) return;
      char* values = own + buffer * F::kBufferBytes + kKeys * kRowBytes;
#pragma unroll 1
      for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t row = stage_row + load_row + i * kLoadRows;
        u32x4* at_lds = reinterpret_cast<u32x4*>(values + row * kRowBytes + load_chunk * 16);
        const u32x4 v = *at_lds;
        u32x4 kept = live >> row & 1 ? v : u32x4{0, 0, 0, 0};
        if (some_see(t)) {
          const u32x4 even = without_odd<T>(kept);
          if (__any(even.x != kept.x || even.y != kept.y || even.z != kept.z || even.w != kept.w)) {
            if (lane == 0) odd_there[turn] = 1;
            kept = even;
          }
        }
        *at_lds = kept;
      }
    };
    const auto ready_wave = [&] {  // what the wave put is there for its lanes: its LDS accesses are carried out in order
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const auto ready = [&] {  // what is put is there for all that read it
      if constexpr (kRowWaves > 1)
        __syncthreads();
      else
        ready_wave();
    };

    // queries: dims 16 s + 8 g .. + 7 (bf16), 8 s + 4 g .. + 3 (fp32) of the lane's row, negated for a negative scale
    u32x4 q[kSteps];
    {
      const char* qp = a.q + (static_cast<int64_t>(s.token + node) * a.q_token + static_cast<int64_t>(q_head) * a.q_head) * sizeof(T);
#pragma unroll
      for (uint32_t c = 0; c < kSteps; ++c) {
        q[c] = u32x4{0, 0, 0, 0};
        if (mine && a.scale != 0.0f) q[c] = *reinterpret_cast<const u32x4_any*>(qp + (2 * c + g) * 16);
        if (a.scale < 0.0f) q[c] ^= kWide ? 0x80000000u : 0x80008000u;
      }
    }
    // Scores of 32 keys from `key` on (of which `live` are) that the lane's row does not see.
    const auto hide = [&](f32x16& x, uint32_t key, uint32_t live) {
      const int32_t e0 = static_cast<int32_t>(key) - static_cast<int32_t>(s.cached);  // of the new tokens
      uint32_t see;
      if (e0 <= -32) {
        see = ~0u;
      } else if (a.seen == nullptr) {
        const int32_t n = static_cast<int32_t>(node) + 1 - e0;
        see = n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1;
      } else {
        const uint64_t* words = a.seen + static_cast<int64_t>(s.token + node) * a.seen_stride;
        const auto word = [&](uint32_t w) { return mine && w < a.words ? words[w] : 0ull; };
        if (e0 < 0) {
          see = ((1u << -e0) - 1) | static_cast<uint32_t>(word(0) << -e0);
        } else {
          const uint32_t w = static_cast<uint32_t>(e0) / 64, by = static_cast<uint32_t>(e0) % 64;
          uint64_t bits = word(w) >> by;
          if (by > 32) bits |= word(w + 1) << (64 - by);
          see = static_cast<uint32_t>(bits);
        }
      }
      const uint32_t shown = (see & live) >> (4 * g);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = shown >> (8 * (i / 4) + i % 4) & 1 ? x[i] : -INFINITY;
    };
    // a scale of 0 would make a NaN of a masked score: the queries are 0 instead
    const float scale = a.scale == 0.0f ? 1.0f : fabsf(a.scale);
    // What the lane's scores of this block are still multiplied by, and whether some are large or may meet a large bound. Looked at where the
    // bound rises, and in each block from then on that some are: for every block it costs prompts 6 %.
    float times = scale;
    bool some_large = false;
    const auto is_large = [](float v) { return fabsf(v) >= kLarge && fabsf(v) < INFINITY; };

    float m = -INFINITY, l = 0.0f;
    f32x16 o[kOuts];
#pragma unroll
    for (uint32_t e = 0; e < kOuts; ++e) o[e] = f32x16{};

    if constexpr (F::kPiped) {
      // Blocks of 32 keys in a pipeline: while the products of the next block's scores and of the block before with the values run on
      // the matrix cores, the vector units turn this block's scores into weights. Keys run a tile ahead of the values
      // in their two buffers each, so that one barrier a tile does.
      find_sixteens(sixteen_of(t_begin) / 64, sixteens_id(sixteen_of(t_begin) / 64));
      Places now_at = places_of(t_begin), next_at = now_at, after_at;  // of the values' tile, the keys' tile, and the one behind it
      __syncthreads();  // the item before is done with the LDS
      if (threadIdx.x == 0) odd_there[turn ^ 1] = 0;
      bring_keys(now_at, 0);
      bring_values(now_at, 0);
      if (t_begin + 1 < t_end) {
        next_at = places_of(t_begin + 1);
        bring_keys(next_at, 1);
        loads_left<2 * kLoads>();
      } else {
        loads_left<kLoads>();
      }
      __syncthreads();

      f32x16 x;                  // this block's scores
      uint32_t weights[8] = {}, rests[8] = {};  // the block before's in two parts, bf16 in pairs
      // Operands are read ahead of their products, into the registers that a product has left: keys two products ahead (four spill 22
      // more registers: 48 trees 215 us instead of 205, prompts 1,380 instead of 1,342, one answer's tree 19 instead of 16.5).
      constexpr uint32_t kAhead = 2;
      u32x4 kf[kAhead], vf[kOuts];
      // Where the lane's operands are, in the buffer in turn; blocks and sixteens are constant offsets behind it.
      uint32_t key_from[kSteps], value_from[kOuts];
#pragma unroll
      for (uint32_t c = 0; c < kSteps; ++c) key_from[c] = lds_address(own) + (key_at ^ (c * 32));
#pragma unroll
      for (uint32_t e = 0; e < kOuts; ++e) value_from[e] = lds_address(own) + kKeys * kRowBytes + (value_at ^ (e * 64));
      const auto turn_to = [&](auto& from, uint32_t buffer) {  // from the other one
        const uint32_t by = buffer ? F::kBufferBytes : 0u - F::kBufferBytes;
#pragma unroll
        for (uint32_t& at : from) {
          at += by;
          asm volatile("" : "+v"(at));  // kept as it is, instead of both buffers' addresses
        }
      };
      const auto read_key = [&](uint32_t b, uint32_t c) {
        typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;
        return *(lds_u32x4*)(key_from[c] + b * 32 * kRowBytes);
      };
      const auto read_value = [&](uint32_t b, uint32_t n) {  // n = 0 .. 2 kOuts - 1: dims n % kOuts, sixteen n / kOuts
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const uint32_t from = value_from[n % kOuts] + (32 * b + 16 * (n / kOuts)) * kRowBytes;
        const u32x2 v0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from));
        const u32x2 v1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 8 * kRowBytes)));
        return u32x4{v0.x, v0.y, v1.x, v1.y};
      };
      const auto score = [&](f32x16& y, uint32_t n) {
        y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[n % kAhead]), __builtin_bit_cast(bf16x8, q[n]), y, 0, 0, 0);
      };
      const auto weigh = [&](uint32_t n, const uint32_t (&part)[8]) {
        const uint32_t e = n % kOuts, c = n / kOuts;
        const u32x4 w = {part[4 * c], part[4 * c + 1], part[4 * c + 2], part[4 * c + 3]};
        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[e]), __builtin_bit_cast(bf16x8, w), o[e], 0, 0, 0);
      };
      // The bound of the scores: above them by 8, a whole number, so that rescaling is exact also for the weights that wait.
      const auto bounded = [&](uint32_t key, uint32_t live) {
        if (key + 32 > wave_sees || live != ~0u) hide(x, key, live);
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
        top *= scale;
        if (__any(top > m) || some_large) {
          const bool large = is_large(top);
          x *= large ? scale : 1.0f;
          times = large ? 1.0f : scale;
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          top = fmaxf(__builtin_ceilf(top) + kLazy, m);
          const float by = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);  // m = -inf: 0
          l *= by;
#pragma unroll
          for (uint32_t e = 0; e < kOuts; ++e) o[e] *= by;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            weights[i] = pack_bf16x2(__uint_as_float(weights[i] << 16) * by, __uint_as_float(weights[i] & 0xFFFF0000u) * by);
            rests[i] = pack_bf16x2(__uint_as_float(rests[i] << 16) * by, __uint_as_float(rests[i] & 0xFFFF0000u) * by);
          }
          m = top;
          some_large = __any(large || is_large(m));
        }
      };
      // One step: the scores of block kb of a tile, the products of the waiting weights with the values of block vb of a tile (kValues),
      // this block's weights. A third of two weights' arithmetic lies behind each product (in the compiler's own order 3 % more). The first
      // operands are there; the next step's first ones (of blocks kb + 1 and vb + 1) are read at its end (kNext).
      const auto step = [&](auto scores, auto values, auto next, uint32_t kb, uint32_t vb) {
        constexpr bool kScores = scores.value, kValues = values.value, kNext = next.value;
        f32x16 y = {};
        uint32_t now[8], rest[8];
        const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (uint32_t n = 0; n < 8; ++n) {
          if (kScores && n < kSteps) {
            score(y, n);
            if (n + kAhead < kSteps)
              kf[n % kAhead] = read_key(kb, n + kAhead);
            else if (kNext)
              kf[n % kAhead] = read_key(kb + 1, n + kAhead - kSteps);
          }
          const bool weighs = kValues && n < 2 * kOuts;
          float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * n], times, -ref));
          float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * n + 1], times, -ref));
          asm volatile("" : "+v"(p0), "+v"(p1));  // here, under the products, and not where they are used
          __builtin_amdgcn_sched_barrier(0);
          if (weighs) weigh(n, weights);
          l += p0 + p1;
          uint32_t b0 = below(p0), b1 = below(p1);
          now[n] = first_parts(b0, b1);
          asm volatile("" : "+v"(b0), "+v"(b1), "+v"(l), "+v"(now[n]));
          __builtin_amdgcn_sched_barrier(0);
          if (weighs) {
            weigh(n, rests);
            if (n < kOuts)
              vf[n] = read_value(vb, n + kOuts);
            else if (kNext)
              vf[n - kOuts] = read_value(vb + 1, n - kOuts);
          }
          rest[n] = rests_of(p0, p1, b0, b1);
          asm volatile("" : "+v"(rest[n]));
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < 8; ++n) weights[n] = now[n], rests[n] = rest[n];
        if constexpr (kScores) x = y;
      };
      const std::true_type yes{};
      const std::false_type no{};
      if (wave_rows) {
        x = f32x16{};
#pragma unroll
        for (uint32_t n = 0; n < kAhead; ++n) kf[n] = read_key(0, n);
#pragma unroll
        for (uint32_t n = 0; n < kSteps; ++n) {
          score(x, n);
          kf[n % kAhead] = n + kAhead < kSteps ? read_key(0, n + kAhead) : read_key(1, n + kAhead - kSteps);
        }
        bounded(t_begin * kTile, static_cast<uint32_t>(now_at.live));
        step(yes, no, no, 1, 0);
        bounded(t_begin * kTile + 32, static_cast<uint32_t>(now_at.live >> 32));
      }
      uint32_t buffer = 0;
      for (uint32_t t = t_begin; t + 1 < t_end; ++t) {
        const uint32_t other = buffer ^ 1;
        loads_left<0>();
        asm volatile("" : "+v"(coming_id));  // used here, where no wait is added for it
        mend(t, buffer, now_at.live);
        __syncthreads();
        turn_to(key_from, other);
        if (t > t_begin) turn_to(value_from, buffer);
        if (wave_rows) {  // on their way before the tiles' own loads are
#pragma unroll
          for (uint32_t n = 0; n < kAhead; ++n) kf[n] = read_key(0, n);
#pragma unroll
          for (uint32_t n = 0; n < kOuts; ++n) vf[n] = read_value(0, n);
        }
        bring_values(next_at, other);
        if (t + 2 < t_end) {
          after_at = places_of(t + 2);
          bring_keys(after_at, buffer);
        }
        if (wave_rows) {
          step(yes, yes, yes, 0, 0);
          bounded((t + 1) * kTile, static_cast<uint32_t>(next_at.live));
          step(yes, yes, no, 1, 1);
          bounded((t + 1) * kTile + 32, static_cast<uint32_t>(next_at.live >> 32));
        }
        now_at = next_at;
        next_at = after_at;
        buffer = other;
      }
      loads_left<0>();
      mend(t_end - 1, buffer, now_at.live);
      __syncthreads();
      if (t_end - 1 > t_begin) turn_to(value_from, buffer);
      if (wave_rows) {
#pragma unroll
        for (uint32_t n = 0; n < kOuts; ++n) vf[n] = read_value(0, n);
        step(no, yes, yes, 0, 0);
#pragma unroll
        for (uint32_t n = 0; n < 2 * kOuts; ++n) {
          weigh(n, weights);
          weigh(n, rests);
          if (n < kOuts) vf[n] = read_value(1, n + kOuts);
        }
      }
    } else {
      // a wave that has keys of its own leaves out a last tile that ends before them
      const uint32_t t_last = kRowWaves > 1 ? t_end : uniform(min(t_end, sees > kw * kKeys ? (sees - kw * kKeys + kTile - 1) / kTile : 0u));
      find_sixteens(sixteen_of(t_begin) / 64, sixteens_id(sixteen_of(t_begin) / 64));
      Places now_at = places_of(t_begin), next_at = now_at;
      __syncthreads();  // the item before is done with the LDS
      if (threadIdx.x == 0) odd_there[turn ^ 1] = 0;
      if (t_begin < t_last) {
        bring_keys(now_at, 0);
        bring_values(now_at, 0);
      }
      if constexpr (kRowWaves > 1) {
        loads_left<0>();
        mend(t_begin, 0, now_at.live);
      }
      ready();

      uint32_t buffer = 0;
      for (uint32_t t = t_begin; t < t_last; ++t) {
        const bool more = t + 1 < t_last;
        const uint32_t other = (buffer + 1) % F::kBuffers;
        if constexpr (kRowWaves > 1) {
          if (more) {
            next_at = places_of(t + 1);
            bring_keys(next_at, other);
            bring_values(next_at, other);
          }
        } else {
          loads_left<kLoads>();  // the keys are there
          ready();
        }
        const uint64_t live = now_at.live;
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
        if constexpr (kRowWaves == 1) {
          asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the keys are read
          ready();
          if (more) {
            next_at = places_of(t + 1);
            bring_keys(next_at, 0);
            loads_left<kLoads>();  // the values are there
          } else {
            loads_left<0>();
          }
          mend(t, 0, live);
          ready();
        }
        if (use) {
          const bool some = key0 + kKeys > wave_sees || live != kAll;
          if (some) {
#pragma unroll
            for (uint32_t b = 0; b < kBlocks; ++b) hide(x[b], key0 + 32 * b, static_cast<uint32_t>(live >> (32 * b)));
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
          if (__any(top > m) || some_large) {
            const bool large = is_large(top);
#pragma unroll
            for (uint32_t b = 0; b < kBlocks; ++b) x[b] *= large ? scale : 1.0f;
            times = large ? 1.0f : scale;
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            top = fmaxf(top + kLazy, m);
            const float by = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);  // m = -inf: 0
            l *= by;
#pragma unroll
            for (uint32_t e = 0; e < kOuts; ++e) o[e] *= by;
            m = top;
            some_large = __any(large || is_large(m));
          }
          const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
          for (uint32_t b = 0; b < kBlocks; ++b) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][i], times, -ref));
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
              u32x4 hi[2], lo[2];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint32_t b0 = below(p[2 * i]), b1 = below(p[2 * i + 1]);
                hi[i / 4][i % 4] = first_parts(b0, b1);
                lo[i / 4][i % 4] = rests_of(p[2 * i], p[2 * i + 1], b0, b1);
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
        if constexpr (kRowWaves > 1) {
          loads_left<0>();
          if (more) mend(t + 1, other, next_at.live);
        } else {
          asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the values are read
          ready();
          if (more) bring_values(next_at, 0);
        }
        now_at = next_at;
        buffer = other;
        ready();
      }
    }
    l += __shfl_xor(l, 32, 64);

    const bool whole = t_begin == 0 && t_end == tiles;
    if (threadIdx.x == 0 && t_end == tiles && !whole)  // so it began in another run
      a.splits[runs.worker_of(item_first)] = Split{worker, s.token, row0, in_block, head, {0, 0, 0}};
    // Results through LDS, for whole lines: rows swizzled by 16 bytes, then four dims of a row for each lane.
    float* parts = part_at<kRows>(a, worker, t_begin == 0 ? 1 : 0);
    const auto write_four = [&](uint32_t i, uint32_t dim, f32x4 four) {  // of row i of the item
      if (whole) {
        const uint32_t out_row = row0 + i, out_node = node_of(a, out_row);
        T* to = reinterpret_cast<T*>(a.out) + static_cast<int64_t>(s.token + out_node) * a.out_token +
                static_cast<int64_t>(head * a.group + out_row - out_node * a.group) * a.out_head + dim;
        store_four(to, four);
      } else {
        *reinterpret_cast<f32x4*>(parts + static_cast<size_t>(i) * a.part_row + 4 + dim) = four;
      }
    };
    const auto write_sums = [&](uint32_t i, uint32_t out_token, uint32_t out_head, float row_m, float row_l) {
      if (!whole)
        *reinterpret_cast<float2*>(parts + static_cast<size_t>(i) * a.part_row) = make_float2(row_m, row_l);
      else if (a.lse)
        a.lse[static_cast<size_t>(out_token) * a.heads * a.group + out_head] = log_sum(row_m, row_l);
    };
    // What a whole row's sum is multiplied by; a row that saw nothing holds zeros.
    const auto over = [&](float row_l) { return whole && any_seen(row_l) ? 1.0f / row_l : 1.0f; };
    __syncthreads();  // the last tile is read
    constexpr uint32_t kRoom = F::kLds / (F::kWaves * 32 * 4), kPass = kDim < kRoom ? kDim : kRoom;  // dims of a row at a time
    constexpr uint32_t kQuads = kPass / 4, kEach = kWave / kQuads;                                  // rows of a wave at a time
    float* rest = reinterpret_cast<float*>(lds) + wave * 32 * kPass;
    float scaled = 1.0f;
    if constexpr (F::kKeyWaves > 1) {
      if (g == 0) sums[wave][r] = make_float2(m, l);
    } else {
      scaled = over(l);
      if (mine && g == 0) write_sums(rw * 32 + r, s.token + node, q_head, m, l);
    }
#pragma unroll
    for (uint32_t pass = 0; pass < kDim / kPass; ++pass) {
      if (wave_rows) {
#pragma unroll
        for (uint32_t e = 0; e < kPass / 32; ++e)
#pragma unroll
          for (uint32_t i = 0; i < 16; i += 4) {
            const f32x16& from = o[pass * (kPass / 32) + e];
            *reinterpret_cast<f32x4*>(rest + r * kPass + ((8 * e + i / 2 + g) ^ r % kQuads) * 4) =
                f32x4{from[i], from[i + 1], from[i + 2], from[i + 3]} * scaled;
          }
      }
      const uint32_t quad = lane % kQuads;
      if constexpr (F::kKeyWaves > 1) {  // the waves have the same rows: each joins a share of them
        static_assert(kPass == kDim, "all rows of all waves have room");
        __syncthreads();
        constexpr uint32_t kShare = 32 / F::kWaves;
        for (uint32_t i = wave * kShare + lane / kQuads; i < min((wave + 1) * kShare, in_block); i += kEach) {
          float row_m = -INFINITY, row_l = 0.0f;
#pragma unroll
          for (uint32_t w = 0; w < F::kWaves; ++w) row_m = fmaxf(row_m, sums[w][i].x);
          const float ref = row_m == -INFINITY ? 0.0f : row_m;
          f32x4 four = {0, 0, 0, 0};
#pragma unroll
          for (uint32_t w = 0; w < F::kWaves; ++w) {
            const float by = __builtin_amdgcn_exp2f(sums[w][i].x - ref);
            row_l += sums[w][i].y * by;
            four += *reinterpret_cast<const f32x4*>(reinterpret_cast<float*>(lds) + (w * 32 + i) * kPass + (quad ^ i % kQuads) * 4) * by;
          }
          write_four(i, quad * 4, four * over(row_l));
          if (quad == 0) {
            const uint32_t out_row = row0 + i, out_node = node_of(a, out_row);
            write_sums(i, s.token + out_node, head * a.group + out_row - out_node * a.group, row_m, row_l);
          }
        }
      } else {
        ready_wave();
        const uint32_t count = wave_rows ? min(32u, in_block - rw * 32) : 0u;
#pragma unroll 2
        for (uint32_t i = lane / kQuads; i < count; i += kEach) {
          write_four(rw * 32 + i, pass * kPass + quad * 4, *reinterpret_cast<const f32x4*>(rest + i * kPass + (quad ^ i % kQuads) * 4));
        }
        ready_wave();
      }
    }
    // Infinities and NaN in tiles that only some rows see, to the results of the rows that see them. (The waves have passed a barrier
    // since the last one was found.)
    if (odd_there[turn] != 0) {
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");  // the results are written
      if constexpr (F::kKeyWaves > 1) __syncthreads();      // by all waves
    }
    if (kw == 0 && wave_rows && odd_there[turn] != 0) {
      float* part = parts + static_cast<size_t>(rw * 32 + r) * a.part_row + 4;
      T* result = reinterpret_cast<T*>(a.out) + static_cast<int64_t>(s.token + node) * a.out_token + static_cast<int64_t>(q_head) * a.out_head;
      const auto odd = [](float v) { return !(fabsf(v) <= 3.402823466e38f); };
      for (uint32_t j = t_begin * kTile; j < min(t_end * kTile, wave_end); ++j) {
        if (!some_see(j / kTile)) continue;
        const int32_t page = ids[page_of(j)];
        if (static_cast<uint32_t>(page) >= a.pages) continue;
        const T* value = reinterpret_cast<const T*>(vp + page * a.page_bytes + static_cast<int64_t>(j - page_of(j) * a.page_tokens) * a.token_bytes);
        bool any = false;
        for (uint32_t dim = lane; dim < kDim; dim += kWave) any = any || odd(S::load1(value + dim));
        if (__ballot(any) == 0) continue;
        const int32_t e = static_cast<int32_t>(j) - static_cast<int32_t>(s.cached);
        bool sees_it = mine && e < 0;
        if (mine && e >= 0)
          sees_it = a.seen == nullptr ? static_cast<uint32_t>(e) <= node
                                      : static_cast<uint32_t>(e) / 64 < a.words &&
                                            (a.seen[static_cast<int64_t>(s.token + node) * a.seen_stride + e / 64] >> (e % 64) & 1);
        if (!sees_it) continue;
        for (uint32_t dim = g * (kDim / 2); dim < (g + 1) * (kDim / 2); ++dim) {
          const float v = S::load1(value + dim);
          if (!odd(v)) continue;
          if (whole)
            S::store1(result + dim, S::load1(result + dim) + v);
          else
            part[dim] += v;
        }
      }
    }
    // the next item
    at = item_first + t_end;
    if (t_end == tiles && !next_item(a, at, end, Lanes<kRows>{a, lds_seqs, lane}, item)) break;
  }
  // unless the last item goes on that began in this run
  if (threadIdx.x == 0 && !leaves_open(begin, at, item.first)) arguments().splits[worker].last = 0;
}

// Joins the parts of the items that were split. A workgroup takes a run of entries (few items lie evenly among these, so that
// every n-th entry would be all items to one), and of its items' rows, four dims a thread, every gridDim.y-th share; kSlices groups of its threads take every kSlices-th part each and join theirs through LDS, so that an item of
// many parts is not read one after another.
template <class S, uint32_t kDim, uint32_t kRows, uint32_t kSlices>
__global__ void __launch_bounds__(kThreads) join_kernel(const Attend a) {
  typedef typename S::storage T;
  constexpr uint32_t kShare = kThreads / kSlices, kQuads = kDim / 4;
  __shared__ float2 sums[kSlices > 1 ? kThreads : 1];
  __shared__ f32x4 rows[kSlices > 1 ? kThreads : 1];
  const uint32_t lane = threadIdx.x % kWave, slice = threadIdx.x / kShare;
  uint32_t active = a.workers;
  for (uint32_t i0 = 0; i0 < (active + gridDim.x - 1) / gridDim.x; i0 += kWave) {
    const Split guess = a.splits[min(blockIdx.x, a.workers - 1)];  // where each workgroup has one entry, with the count at once
    active = *a.active;
    const uint32_t each = (active + gridDim.x - 1) / gridDim.x, mine = blockIdx.x * each + i0 + lane;
    const bool have = i0 + lane < each && mine < active;
    const Split own = each == 1 ? guess : a.splits[have ? mine : 0];
    // what no run has written, because lengths or starts changed under the call, is not taken for an entry outside the rows
    const uint32_t room = own.token < a.tokens ? (a.tokens - own.token) * a.group : 0u;
    const bool inside = own.last < active && own.head < a.heads && own.rows <= kRows && own.row < room && own.rows <= room - own.row;
    for (uint64_t left = __ballot(have && own.last != 0 && inside); left != 0; left &= left - 1) {
      const uint32_t from = static_cast<uint32_t>(__builtin_ctzll(left)), first = blockIdx.x * each + i0 + from;
      const auto there = [&](uint32_t v) -> uint32_t { return __builtin_amdgcn_readlane(v, from); };
      const uint32_t last = there(own.last), token = there(own.token), row0 = there(own.row);
      const uint32_t item_rows = there(own.rows), head = there(own.head);
      for (uint32_t share = blockIdx.y; share * kShare < item_rows * kQuads; share += gridDim.y) {
        const uint32_t e = share * kShare + threadIdx.x % kShare, row = e / kQuads, dim = e % kQuads * 4;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0, 0, 0, 0};
        const auto add = [&](float2 ml, f32x4 po) {
          const float top = fmaxf(m, ml.x), ref = top == -INFINITY ? 0.0f : top;
          const float s0 = __builtin_amdgcn_exp2f(m - ref), s1 = __builtin_amdgcn_exp2f(ml.x - ref);
          l = l * s0 + ml.y * s1;
          o = o * s0 + po * s1;
          m = top;
        };
        if (row < item_rows) {
#pragma unroll 4
          for (uint32_t w = first + slice; w <= last; w += kSlices) {
            const float* part = part_at<kRows>(a, w, w == first ? 1 : 0) + static_cast<size_t>(row) * a.part_row;
            add(*reinterpret_cast<const float2*>(part), *reinterpret_cast<const f32x4*>(part + 4 + dim));
          }
        }
        if constexpr (kSlices > 1) {
          __syncthreads();  // the share before is joined
          sums[threadIdx.x] = make_float2(m, l);
          rows[threadIdx.x] = o;
          __syncthreads();
          if (slice == 0)
#pragma unroll
            for (uint32_t n = 1; n < kSlices; ++n) add(sums[threadIdx.x + n * kShare], rows[threadIdx.x + n * kShare]);
        }
        if (slice == 0 && row < item_rows) {
          const uint32_t node = node_of(a, row0 + row), q_head = head * a.group + row0 + row - node * a.group;
          store_four(reinterpret_cast<T*>(a.out) + static_cast<int64_t>(token + node) * a.out_token + static_cast<int64_t>(q_head) * a.out_head + dim,
                     o * (any_seen(l) ? 1.0f / l : 0.0f));
          if (a.lse && dim == 0) a.lse[static_cast<size_t>(token + node) * a.heads * a.group + q_head] = log_sum(m, l);
        }
      }
    }
  }
}

// Any head size, page size and alignment: a workgroup has a row at a time, its waves every fourth 64 keys. 64 keys' scores at once, one
// in each lane, then their values, a dim in each lane (and the dims 64, 128 and 192 behind it); each 64's sum is added to what was
// there, and the waves join at the end. A token that the row does not see is not read. Every row reads its keys anew. 40 new tokens of
// 4 heads of 96 behind 1,000: 72 us in bf16, 48 in fp32 (heads of 128 by the other kernel: 17 and 23).
template <class S>
__global__ void __launch_bounds__(kThreads) plain_kernel(const Attend a) {
  typedef typename S::storage T;
  constexpr uint32_t kVec = 16 / sizeof(T), kDims = ZO_DIM_MAX / kWave, kTogether = 16;
  __shared__ float queries[ZO_DIM_MAX], outs[kWaves][ZO_DIM_MAX], weights[kWaves][kWave];
  __shared__ float2 sums[kWaves];
  __shared__ int64_t places[kWaves][kWave];
  const uint32_t wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, q_heads = a.heads * a.group, rows = a.tokens * q_heads;
  const auto ready_wave = [] {  // what the wave put is there for its lanes
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const uint32_t token = row / q_heads, q_head = row - token * q_heads, head = q_head / a.group;
    // the last sequence that begins at or before the token; with `starts` as they should be it is the token's, if any is
    uint32_t low = 0, high = a.seqs;
    while (low + 1 < high) {
      const uint32_t middle = (low + high) / 2;
      if (a.starts[middle] <= static_cast<int64_t>(token))
        low = middle;
      else
        high = middle;
    }
    const Seq s = seq_of<32>(a, low);
    if (token < s.token || token - s.token >= s.count) continue;
    const uint32_t node = token - s.token, sees = a.seen ? s.len : min(s.len, s.cached + node + 1);
    const T* qp = reinterpret_cast<const T*>(a.q) + static_cast<int64_t>(token) * a.q_token + static_cast<int64_t>(q_head) * a.q_head;
    __syncthreads();  // the row before is done with the LDS
    for (uint32_t d = threadIdx.x; d < a.dim; d += kThreads) queries[d] = S::load1(qp + d);
    __syncthreads();
    const int32_t* ids = a.ids + static_cast<int64_t>(low) * a.table_stride;
    const char* kp = a.k + head * a.head_bytes;
    const char* vp = a.v + head * a.head_bytes;
    float m = -INFINITY, l = 0.0f, o[kDims] = {};
    for (uint32_t base = wave * kWave; base < sees; base += kThreads) {
      const uint32_t j = base + lane;
      bool live = j < sees;
      if (live && a.seen && j >= s.cached) {
        const uint32_t e = j - s.cached;
        live = e / 64 < a.words && (a.seen[static_cast<int64_t>(token) * a.seen_stride + e / 64] >> (e % 64) & 1);
      }
      int64_t place = -1;
      if (live) {
        const uint32_t page = j / a.page_tokens;
        const int32_t id = ids[page];
        if (static_cast<uint32_t>(id) < a.pages) place = id * a.page_bytes + static_cast<int64_t>(j - page * a.page_tokens) * a.token_bytes;
      }
      float score = -INFINITY;
      if (place >= 0) {
        const T* key = reinterpret_cast<const T*>(kp + place);
        float sum = 0.0f;
        uint32_t d = 0;
#pragma unroll 4
        for (; d + kVec <= a.dim; d += kVec) {
          const u32x4 four = *reinterpret_cast<const u32x4_any*>(key + d);
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) {
            if constexpr (kVec == 8) {
              sum = __builtin_fmaf(queries[d + 2 * i], __uint_as_float(four[i] << 16), sum);
              sum = __builtin_fmaf(queries[d + 2 * i + 1], __uint_as_float(four[i] & 0xFFFF0000u), sum);
            } else {
              sum = __builtin_fmaf(queries[d + i], __uint_as_float(four[i]), sum);
            }
          }
        }
        for (; d < a.dim; ++d) sum = __builtin_fmaf(queries[d], S::load1(key + d), sum);
        score = sum * a.scale;
      }
      float top = score;
#pragma unroll
      for (uint32_t n = 1; n < kWave; n *= 2) top = fmaxf(top, __shfl_xor(top, n, 64));
      top = top > m ? top + kLazy : m;
      const float ref = top == -INFINITY ? 0.0f : top, by = __builtin_amdgcn_exp2f(m - ref);
      const float weight = place >= 0 ? __builtin_amdgcn_exp2f(score - ref) : 0.0f;
      float all = weight;
#pragma unroll
      for (uint32_t n = 1; n < kWave; n *= 2) all += __shfl_xor(all, n, 64);
      l = l * by + all;
      m = top;
      weights[wave][lane] = weight;
      places[wave][lane] = place;
      const uint64_t there = __ballot(place >= 0);
      ready_wave();
      float part[kDims] = {};
      for (uint32_t i0 = 0; i0 < kWave; i0 += kTogether) {
        if ((there >> i0 & ((1ull << kTogether) - 1)) == 0) continue;
#pragma unroll
        for (uint32_t c = 0; c < kDims; ++c) {
          if (c * kWave >= a.dim) break;
          const bool in = c * kWave + lane < a.dim;
          float v[kTogether];
#pragma unroll
          for (uint32_t i = 0; i < kTogether; ++i) {
            const int64_t from = places[wave][i0 + i];
            v[i] = in && from >= 0 ? S::load1(reinterpret_cast<const T*>(vp + from) + c * kWave + lane) : 0.0f;
          }
#pragma unroll
          for (uint32_t i = 0; i < kTogether; ++i) part[c] = __builtin_fmaf(weights[wave][i0 + i], v[i], part[c]);
        }
      }
#pragma unroll
      for (uint32_t c = 0; c < kDims; ++c) o[c] = o[c] * by + part[c];
      ready_wave();
    }
    if (lane == 0) sums[wave] = make_float2(m, l);
#pragma unroll
    for (uint32_t c = 0; c < kDims; ++c) outs[wave][c * kWave + lane] = o[c];
    __syncthreads();
    float top = -INFINITY, total = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) top = fmaxf(top, sums[w].x);
    const float ref = top == -INFINITY ? 0.0f : top;
    float by[kWaves];
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
      by[w] = __builtin_amdgcn_exp2f(sums[w].x - ref);
      total += sums[w].y * by[w];
    }
    T* op = reinterpret_cast<T*>(a.out) + static_cast<int64_t>(token) * a.out_token + static_cast<int64_t>(q_head) * a.out_head;
    if (threadIdx.x < a.dim) {
      float out = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) out += outs[w][threadIdx.x] * by[w];
      S::store1(op + threadIdx.x, any_seen(total) ? out / total : 0.0f);
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = log_sum(top, total);
  }
}
static_assert(ZO_DIM_MAX == kThreads, "a thread writes a dim");

template <class S, uint32_t kDim, uint32_t kRowWaves>
int launch(Attend& a, hipStream_t st) {
  typedef Form<S, kDim, kRowWaves> F;
  if (F::kLds > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(&attend_kernel<S, kDim, kRowWaves>), hipFuncAttributeMaxDynamicSharedMemorySize,
                          F::kLds) != hipSuccess)
    return ZO_ERR_HIP;
  const uint64_t items = (static_cast<uint64_t>(a.tokens) * a.group / F::kRows + a.seqs) * a.heads;  // there are no more
  // with few items all workgroups have one or two, and what an item costs would only leave some without a tile: trees of 12 behind 1,500, 32 heads
  // on 8 of 128, 4 of them 20.3 us without and 22.4 with, 8: 24.3 and 25.2 (12: 34.8 and 31.5, 16: 31.7 and 33.8, 24: 44.6 and 43.8)
  a.visit = items * 2 >= a.workers ? F::kVisit : 0;
  attend_kernel<S, kDim, kRowWaves><<<dim3(a.workers), dim3(F::kThreads), F::kLds, st>>>(a);
  const int rc = launched();
  if (rc != ZO_OK) return rc;
  // slices where an item has several parts: of the same trees, one 16.7 us with and 17.4 without, 4 20.1 both, 8 25.3 and 24.0, 16 36.7 and 33.9
  const uint32_t most = static_cast<uint32_t>(std::min<uint64_t>(a.workers, items));
  if (items * 6 <= a.workers)
    join_kernel<S, kDim, F::kRows, 4><<<dim3(most, std::min(32u, F::kRows * kDim / 256)), dim3(kThreads), 0, st>>>(a);
  else
    join_kernel<S, kDim, F::kRows, 1><<<dim3(most, std::min(16u, F::kRows * kDim / 1024)), dim3(kThreads), 0, st>>>(a);
  return launched();
}

template <class S, uint32_t kDim>
int rows(Attend& a, uint32_t row_waves, hipStream_t st) {
  if constexpr (kDim * sizeof(typename S::storage) <= 512) {
    if (row_waves == 1) return launch<S, kDim, 1>(a, st);
  }
  if constexpr (Form<S, kDim, 8>::kPiped && kDim > 64) {
    return launch<S, kDim, 8>(a, st);
  } else {
    if constexpr (Form<S, kDim, 8>::kPiped) {
      if (row_waves == 8) return launch<S, kDim, 8>(a, st);
    }
    return launch<S, kDim, 4>(a, st);
  }
}

template <class S>
int attend(Attend& a, uint32_t row_waves, hipStream_t st) {
  // pages of whole sixteens, in which 32-bit offsets reach every row, at vectors' addresses
  const uint64_t places = reinterpret_cast<uint64_t>(a.k) | reinterpret_cast<uint64_t>(a.v) | a.page_bytes | a.head_bytes | a.token_bytes;
  if (a.page_tokens % 16 == 0 && places % 16 == 0 && a.token_bytes < (int64_t{1} << 28)) {
    if (a.dim == 64) return rows<S, 64>(a, row_waves, st);
    if (a.dim == 128) return rows<S, 128>(a, row_waves, st);
    if (a.dim == 256) return rows<S, 256>(a, row_waves, st);
  }
  plain_kernel<S><<<dim3(std::min(a.tokens * a.heads * a.group, 65536u)), dim3(kThreads), 0, st>>>(a);
  return launched();
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
  a.active = reinterpret_cast<uint32_t*>(work);
  a.splits = reinterpret_cast<Split*>(work + 16);
  a.parts = reinterpret_cast<float*>(work + 16 + shape.workers * sizeof(Split));
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
  a.tokens = p->tokens;
  a.words = p->words;
  a.seqs = p->table.seqs;
  a.width = p->table.width;
  a.pages = p->cache.pages;
  a.page_tokens = p->cache.page_tokens;
  a.inv_page = 16.0 / a.page_tokens;
  a.heads = p->cache.heads;
  a.dim = p->cache.dim;
  a.workers = shape.workers;
  a.part_row = a.dim + 4;
  a.scale = p->scale * 1.4426950408889634f;
  (void)hipGetLastError();
  hipStream_t st = static_cast<hipStream_t>(stream);
  return p->dtype == ZO_F32 ? attend<F32>(a, shape.row_waves, st) : attend<BF16>(a, shape.row_waves, st);
}
