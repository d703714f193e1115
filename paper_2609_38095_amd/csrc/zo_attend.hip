// Attention of one new token of each sequence over the paged cache, for gfx950.
//
// Mathematics. One pass over the cached tokens with a running bound m of the scores and a sum l:
// x_j = scale log2(e) q . k_j, p_j = 2^(x_j - m), l = sum p_j, o = sum p_j v_j; a larger bound scales l
// and o by 2^(m - m'). Only a score above the bound raises it, to 8 above the largest score, so that the usual
// tile neither exchanges maxima between lanes nor rescales o; weights are at most 1 all the same, as in a
// softmax by the maximum itself, and values up to the type's largest do not overflow by them.
// Parts of a sequence join by the same rule.
//
// Split. An item is one sequence, one key head and up to 16 of its query heads: they read the same
// keys, so they are the columns of one matrix product, and the cache is read once. Every item is cut
// into tiles of 32 (bf16) or 16 (fp32) tokens; all tiles of the call, in order, are dealt out in
// equal runs to the workers, each of them a wave on its own (no barrier, no LDS in the loop). Lengths are
// known on the device alone, so each worker adds them up itself. A run that covers a whole item writes
// its output; other runs leave (m, l, o) in the workspace, at most two parts for each worker and one for a
// workgroup whose four runs lie in one item,
// and join_kernel joins them.
//
// Tile. S^T = K Q^T and O^T = V^T P^T on the matrix cores. The contraction's index may be permuted if both
// operands are, which lets every operand stay where its loads or the product before put it:
//   - lane (r = lane % 16, g = lane / 16) loads key row r, 16 bytes at 16 g + 64 c: an operand as it is;
//   - S^T leaves head r, keys 4 g .. 4 g + 3 of each 16 in lane (r, g): the second product's operand;
//   - the values of those keys are loaded with lane r holding dims r D/16 .. (r + 1) D/16 - 1, whole
//     rows by 16 lanes; for bf16 pairs of keys are put together by byte permutes (both members are in
//     the lane); output row r of product e is then dim r D/16 + e.
// Nothing passes through LDS. fp32 takes the fp32 matrix instructions: its products are exact to fp32.
//
// Bound by HBM: the keys and values of the live tokens, once. Measured by the device's clock: 1.89 GB of 4 long
// sequences in 286 us and 5 for the join (6.5 TB/s; a plain read of 4 GiB reaches 7.0), 0.53 GB of 48 ragged ones in
// 96 us and 5. One short sequence: 11 us a call.

#include <algorithm>
#include <cmath>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kThreads = 256;
constexpr uint32_t kWave = 64, kWaves = kThreads / kWave;
constexpr float kLazy = 8.0f;  // how far (in powers of two) the bound of the scores is set above their maximum

// Where an item's parts are: those of workers first .. last, the first one's in `slot`, the others' in slot 0;
// the waves of workgroups group0 .. group1 - 1 have theirs together, with the workgroup's first wave.
// first = last: that worker wrote the output. Written by the worker of the item's last tile.
struct Parts {
  uint32_t first_slot;  // 2 first + slot
  uint32_t last, group0, group1;
};

struct Attend {
  const char *q, *k, *v;
  char* out;
  float* lse;
  Parts* items;
  float* parts;
  const int32_t* ids;
  const int32_t* lengths;
  int64_t q_seq, q_head, out_seq, out_head, page_stride, head_stride, token_stride, table_stride;
  uint32_t seqs, width, pages, page_tokens, heads, group, group_blocks, dim, workers, part_row;
  float scale;  // times log2(e)
};

// A value that all lanes of a wave hold, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return static_cast<uint64_t>(uniform(static_cast<uint32_t>(v >> 32))) << 32 | uniform(static_cast<uint32_t>(v));
}

// The tokens of a sequence that the table can hold.
__device__ __forceinline__ uint32_t live_tokens(const Attend& a, uint32_t seq) {
  const int64_t room = static_cast<int64_t>(a.width) * a.page_tokens;
  const int64_t n = a.lengths[seq];
  return static_cast<uint32_t>(n < 0 ? 0 : n > room ? room : n);
}

// Tiles before each thread's sequences. Thread t counts sequences [t each, (t + 1) each).
struct Deal {
  uint64_t total;  // tiles of all items
  uint32_t each;
};

template <uint32_t kTile>
__device__ Deal deal(const Attend& a, uint64_t* before) {
  __shared__ uint64_t wave_sum[kWaves];
  Deal d;
  d.each = (a.seqs + kThreads - 1) / kThreads;
  uint64_t mine = 0;
  for (uint32_t i = 0; i < d.each; ++i) {
    const uint32_t s = threadIdx.x * d.each + i;
    if (s < a.seqs) mine += (live_tokens(a, s) + kTile - 1) / kTile;
  }
  uint64_t upto = mine;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t lower = __shfl_up(upto, m, 64);
    if (threadIdx.x % 64 >= static_cast<uint32_t>(m)) upto += lower;
  }
  if (threadIdx.x % 64 == 63) wave_sum[threadIdx.x / 64] = upto;
  __syncthreads();
  uint64_t offset = 0, all = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < threadIdx.x / 64) offset += wave_sum[w];
    all += wave_sum[w];
  }
  const uint64_t items = static_cast<uint64_t>(a.heads) * a.group_blocks;
  before[threadIdx.x] = (offset + upto - mine) * items;
  d.total = uniform(all * items);
  __syncthreads();
  return d;
}

// Floor of n / d for n below 2^52: exact, since quotients of neighbours are further apart than an fp64 rounding.
__device__ __forceinline__ uint64_t quotient(uint64_t n, uint64_t d) {
  return static_cast<uint64_t>(static_cast<double>(n) / static_cast<double>(d));
}

// The first tile of worker w: total tiles in equal runs, the first ones a tile longer.
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

// A part in the workspace: for each of the item's query heads a row [m, l, -, -, o[dim rounded up to 4]].
__device__ __forceinline__ float* part_at(const Attend& a, uint32_t worker, uint32_t slot, uint32_t group) {
  return a.parts + (static_cast<size_t>(worker) * 2 + slot) * group * a.part_row;
}

// Waves for each SIMD: as many as the tile's keys and values (64 registers of a lane in the larger forms), the
// sums and the queries leave room for without spilling into the loop. Loads in flight come from the waves:
// asking for the next tile's before this one's use, at fewer waves, measured the same (bf16, 128 dims, 0.56 GB:
// 98 us either way) or slower, and a spilled form 133.
template <class S>
constexpr uint32_t waves_for(uint32_t dim) {
  return sizeof(typename S::storage) == 2 ? (dim > 128 ? 2 : dim > 64 ? 3 : 4) : (dim > 128 ? 1 : dim > 64 ? 2 : 4);
}

// Four dims of a head's output from its sums, and its log-sum once.
template <class S>
__device__ __forceinline__ void write_head(const Attend& a, uint32_t seq, uint32_t q_head, uint32_t dim, float m, float l, f32x4 o) {
  typedef typename S::storage T;
  const bool any = l > 0.0f || l != l;
  T* op = reinterpret_cast<T*>(a.out) + static_cast<int64_t>(seq) * a.out_seq + static_cast<int64_t>(q_head) * a.out_head;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    if (dim + i < a.dim) S::store1(op + dim + i, any ? o[i] / l : 0.0f);
  if (a.lse && dim == 0)
    a.lse[static_cast<size_t>(seq) * a.heads * a.group + q_head] = any ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

template <class S>
struct Mfma;

// bf16: tiles of 32 keys, 16 x 16 x 32 products.
template <>
struct Mfma<BF16> {
  static constexpr uint32_t kTile = 32, kSubs = 2, kLoadDims = 8;
};
// fp32: tiles of 16 keys, 16 x 16 x 4 products.
template <>
struct Mfma<F32> {
  static constexpr uint32_t kTile = 16, kSubs = 1, kLoadDims = 4;
};

__device__ __forceinline__ f32x4 mul_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// kDim: the head size, or (kAny) the size that it is padded to with zeros; kAny also takes any
// page size and any strides, with one lookup and one bounds check for each element's row.
template <class S, uint32_t kDim, bool kAny>
__global__ void __launch_bounds__(kThreads, kAny ? (kDim > 128 ? 1 : 2) : waves_for<S>(kDim)) attend_kernel(const Attend a) {
  typedef typename S::storage T;
  constexpr uint32_t kTile = Mfma<S>::kTile, kSubs = Mfma<S>::kSubs, kLoad = Mfma<S>::kLoadDims;
  constexpr uint32_t kKeyLoads = kDim / (4 * kLoad);      // 16-byte loads of a key row for each lane
  constexpr uint32_t kLaneDims = kDim / 16;               // dims of a value row for each lane
  constexpr uint32_t kValWords = kLaneDims * sizeof(T) / 4;
  constexpr uint32_t kKeys = 4 * kSubs;                   // keys of a tile for each lane
  constexpr uint32_t kRow = kDim + 4;                     // of a head's sums in LDS, shifted by 4 banks
  __shared__ uint64_t before[kThreads];
  __shared__ float2 wave_sums[kWaves][16];
  __shared__ __align__(16) float wave_rows[kWaves][16][kRow];
  const Deal d = deal<kTile>(a, before);
  const Runs runs(d.total, a.workers);
  const uint32_t wave = uniform(threadIdx.x / kWave), worker = blockIdx.x * kWaves + wave;
  const uint32_t lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  if (worker >= runs.workers) return;
  const uint64_t begin = runs.first(worker), end = runs.first(worker + 1);
  uint64_t at = begin;
  if (at >= end) return;

  // the sequence that tile `at` lies in: the last thread's block that begins at or before it
  uint32_t block = 0;
#pragma unroll
  for (uint32_t step = kThreads / 2; step > 0; step /= 2)
    if (before[block + step] <= at) block += step;
  block = uniform(block);
  uint32_t seq = block * d.each;
  const uint32_t items = a.heads * a.group_blocks, part_heads = min(16u, a.group);
  uint64_t seq_first = uniform(before[block]);  // its first tile

  // byte offsets of the lane's share of a key row, and of value rows 4 g .. 4 g + 3, from a sixteen's first row
  // (the fast form: 32 bits behind a scalar address)
  const uint32_t step = static_cast<uint32_t>(a.token_stride);
  const uint32_t key_at = (r * step + g * kLoad) * sizeof(T);
  uint32_t value_at[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) value_at[i] = ((g * 4 + i) * step + r * kLaneDims) * sizeof(T);

  while (at < end) {
    uint32_t len, tiles;
    for (;;) {  // `at` < the total: a sequence holds it
      len = uniform(live_tokens(a, seq));
      tiles = (len + kTile - 1) / kTile;
      if (at < seq_first + static_cast<uint64_t>(tiles) * items) break;
      seq_first += static_cast<uint64_t>(tiles) * items;
      ++seq;
    }
    const uint32_t item = uniform(static_cast<uint32_t>(quotient(at - seq_first, tiles)));
    const uint64_t item_first = seq_first + static_cast<uint64_t>(item) * tiles;
    const uint32_t t_begin = static_cast<uint32_t>(at - item_first);
    const uint32_t t_end = end - item_first < tiles ? static_cast<uint32_t>(end - item_first) : tiles;
    const uint32_t head = uniform(item / a.group_blocks), gb = item - head * a.group_blocks;
    const uint32_t in_group = min(16u, a.group - gb * 16);  // query heads of this item
    const uint32_t q_head0 = head * a.group + gb * 16;
    const int32_t* ids = a.ids + static_cast<int64_t>(seq) * a.table_stride;
    const T* kp = reinterpret_cast<const T*>(a.k) + static_cast<int64_t>(head) * a.head_stride;
    const T* vp = reinterpret_cast<const T*>(a.v) + static_cast<int64_t>(head) * a.head_stride;

    // The fast form has the page ids of 64 sixteens of tokens at a time, one in each lane: a lookup of its
    // own for each would wait for the loads before it.
    int32_t lane_id = -1;
    uint32_t lane_ids = ~0u;  // which 64 these are
    u32x4 kr[kSubs][kKeyLoads];
    uint32_t vr[kKeys][kValWords];

    // Issues the loads of a tile's keys. Fast: pages hold whole sixteens of tokens, so each 16 keys lie in
    // one page and its address is scalar; rows behind the length are inside the page (and masked), an
    // absent page's are read from page 0 (and masked). row: of the tile's first token in its page.
    const auto sub_base = [&](uint32_t t, uint32_t s, uint32_t row, uint32_t& count) {
      const uint32_t sub = t * kSubs + s, j = sub * 16;
      const int32_t id = __builtin_amdgcn_readlane(lane_id, sub % 64);
      const bool there = static_cast<uint32_t>(id) < a.pages;
      count = there ? min(16u, len - j) : 0u;
      const uint32_t page_row = row + s * 16 < a.page_tokens ? row + s * 16 : 0;
      return (there ? id : 0) * a.page_stride + static_cast<int64_t>(page_row) * a.token_stride;
    };
    const auto load_keys = [&](uint32_t t, uint32_t row) {
      if constexpr (kAny) {
#pragma unroll
        for (uint32_t s = 0; s < kSubs; ++s) {
          const uint32_t j = t * kTile + s * 16 + r;
          const uint32_t p = j / a.page_tokens;
          const int32_t id = j < len ? ids[p] : -1;
          const bool there = static_cast<uint32_t>(id) < a.pages;
          const T* src = kp + (there ? id * a.page_stride + static_cast<int64_t>(j - p * a.page_tokens) * a.token_stride : 0);
#pragma unroll
          for (uint32_t c = 0; c < kKeyLoads; ++c) {
            T tmp[kLoad] = {};
#pragma unroll
            for (uint32_t e = 0; e < kLoad; ++e) {
              const uint32_t i = c * 4 * kLoad + g * kLoad + e;
              if (there && i < a.dim) tmp[e] = src[i];
            }
            __builtin_memcpy(&kr[s][c], tmp, 16);
          }
        }
      } else {
        if (t * kSubs / 64 != lane_ids) {
          lane_ids = t * kSubs / 64;
          const uint32_t j = (lane_ids * 64 + lane) * 16;
          lane_id = j < len ? ids[j / a.page_tokens] : -1;
          // waited for here, once in 64, and not at every use: such a wait would take in the loads of the tile
          asm volatile("s_waitcnt vmcnt(0)" : "+v"(lane_id));
        }
        uint32_t at = key_at;
        asm volatile("" : "+v"(at));  // a 32-bit offset behind the scalar address: widened outside the loop it costs two registers
#pragma unroll
        for (uint32_t s = 0; s < kSubs; ++s) {
          uint32_t count;
          const char* ks = reinterpret_cast<const char*>(kp + sub_base(t, s, row, count));
#pragma unroll
          for (uint32_t c = 0; c < kKeyLoads; ++c) kr[s][c] = ld_stream(ks + at + c * 64);
        }
      }
    };
    // Issues the loads of a tile's values, and says which of the lane's keys (4 g + i of each 16) are live; all
    // ones: every key of the tile is.
    const auto load_values = [&](uint32_t t, uint32_t row) {
      uint32_t live = 0;
      if constexpr (kAny) {
#pragma unroll
        for (uint32_t i = 0; i < kKeys; ++i) {
          const uint32_t j = t * kTile + i / 4 * 16 + g * 4 + i % 4;
          const uint32_t p = j / a.page_tokens;
          const int32_t id = j < len ? ids[p] : -1;
          const bool there = static_cast<uint32_t>(id) < a.pages;
          live |= there ? 1u << i : 0u;
          const T* src = vp + (there ? id * a.page_stride + static_cast<int64_t>(j - p * a.page_tokens) * a.token_stride : 0);
          T tmp[kLaneDims] = {};
#pragma unroll
          for (uint32_t e = 0; e < kLaneDims; ++e)
            if (there && r * kLaneDims + e < a.dim) tmp[e] = src[r * kLaneDims + e];
          __builtin_memcpy(vr[i], tmp, sizeof tmp);
        }
      } else {
        bool whole = true;
        uint32_t count[kSubs];
#pragma unroll
        for (uint32_t s = 0; s < kSubs; ++s) {
          const char* vs = reinterpret_cast<const char*>(vp + sub_base(t, s, row, count[s]));
          whole = whole && count[s] == 16;
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) {
            uint32_t at = value_at[i];
            asm volatile("" : "+v"(at));
            const char* src = vs + at;
            if constexpr (kValWords == 2) {
              typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
              const u32x2_any w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any*>(src));
              vr[s * 4 + i][0] = w.x;
              vr[s * 4 + i][1] = w.y;
            } else {
#pragma unroll
              for (uint32_t w = 0; w < kValWords; w += 4) {
                const u32x4 x = ld_stream(src + w * 4);
                vr[s * 4 + i][w] = x.x;
                vr[s * 4 + i][w + 1] = x.y;
                vr[s * 4 + i][w + 2] = x.z;
                vr[s * 4 + i][w + 3] = x.w;
              }
            }
          }
        }
        live = ~0u;
        if (!whole) {
          live = 0;
#pragma unroll
          for (uint32_t i = 0; i < kKeys; ++i) live |= g * 4 + i % 4 < count[i / 4] ? 1u << i : 0u;
        }
      }
      return live;
    };

    uint32_t row = 0;
    if constexpr (!kAny) row = uniform(t_begin * kTile % a.page_tokens);
    // queries of head r, zeros for columns without one
    u32x4 q[kKeyLoads];
    {
      const T* qp = reinterpret_cast<const T*>(a.q) + static_cast<int64_t>(seq) * a.q_seq +
                    static_cast<int64_t>(q_head0 + (r < in_group ? r : 0)) * a.q_head;
#pragma unroll
      for (uint32_t c = 0; c < kKeyLoads; ++c) {
        q[c] = u32x4{0, 0, 0, 0};
        if constexpr (kAny) {
          T tmp[kLoad] = {};
#pragma unroll
          for (uint32_t e = 0; e < kLoad; ++e) {
            const uint32_t i = c * 4 * kLoad + g * kLoad + e;
            if (r < in_group && i < a.dim) tmp[e] = qp[i];
          }
          __builtin_memcpy(&q[c], tmp, 16);
        } else {
          if (r < in_group) q[c] = *reinterpret_cast<const u32x4_any*>(qp + c * 4 * kLoad + g * kLoad);
        }
      }
    }

    float m = -INFINITY, l = 0.0f;
    f32x4 o[kLaneDims];
#pragma unroll
    for (uint32_t e = 0; e < kLaneDims; ++e) o[e] = f32x4{0, 0, 0, 0};

    for (uint32_t t = t_begin; t < t_end; ++t) {
      load_keys(t, row);
      const uint32_t live = load_values(t, row);
      if constexpr (!kAny) {
        row += kTile;
        if (row >= a.page_tokens) row = a.page_tokens >= kTile ? row - a.page_tokens : 0;
      }
      // scores of head r with keys 4 g .. 4 g + 3 of each 16
      float x[kKeys];
#pragma unroll
      for (uint32_t s = 0; s < kSubs; ++s) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t c = 0; c < kKeyLoads; ++c) {
          if constexpr (sizeof(T) == 2) {
            acc = mul_bf16(kr[s][c], q[c], acc);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[s][c][e]), __uint_as_float(q[c][e]), acc, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[s * 4 + i] = acc[i] * a.scale;
      }
      if (live != ~0u) {
#pragma unroll
        for (uint32_t i = 0; i < kKeys; ++i) {
          x[i] = live >> i & 1 ? x[i] : -INFINITY;
#pragma unroll
          for (uint32_t w = 0; w < kValWords; ++w) vr[i][w] = live >> i & 1 ? vr[i][w] : 0u;  // 0 times whatever lies there
        }
      }
      float top = x[0];
#pragma unroll
      for (uint32_t i = 1; i < kKeys; ++i) top = fmaxf(top, x[i]);
      if (__any(top > m)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        top = fmaxf(top + kLazy, m);
        const float scale = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);  // m = -inf: 0
        l *= scale;
#pragma unroll
        for (uint32_t e = 0; e < kLaneDims; ++e) o[e] *= scale;
        m = top;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      float p[kKeys];
#pragma unroll
      for (uint32_t i = 0; i < kKeys; ++i) {
        p[i] = __builtin_amdgcn_exp2f(x[i] - ref);
        l += p[i];
      }

      if constexpr (sizeof(T) == 2) {
        // weights as a sum of two bf16, 16 bits of each, so that only the output is rounded to 8. Both are positive: the largest
        // bf16 below the weight and what is left of it. A signed or empty rest would make a NaN of an infinite value.
        u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = p[2 * i], p1 = p[2 * i + 1];
          const uint32_t b0 = __builtin_elementwise_sub_sat(__float_as_uint(p0), 1u), b1 = __builtin_elementwise_sub_sat(__float_as_uint(p1), 1u);
          hi[i] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
          lo[i] = pack_bf16x2(p0 - __uint_as_float(b0 & 0xFFFF0000u), p1 - __uint_as_float(b1 & 0xFFFF0000u));
        }
#pragma unroll
        for (uint32_t w = 0; w < kValWords; ++w) {
          u32x4 even, odd;  // dims 2 w and 2 w + 1 of the lane, keys in pairs
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            even[i] = __builtin_amdgcn_perm(vr[2 * i + 1][w], vr[2 * i][w], 0x05040100u);
            odd[i] = __builtin_amdgcn_perm(vr[2 * i + 1][w], vr[2 * i][w], 0x07060302u);
          }
          o[2 * w] = mul_bf16(even, lo, mul_bf16(even, hi, o[2 * w]));
          o[2 * w + 1] = mul_bf16(odd, lo, mul_bf16(odd, hi, o[2 * w + 1]));
        }
      } else {
#pragma unroll
        for (uint32_t e = 0; e < kLaneDims; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[i][e]), p[i], o[e], 0, 0, 0);
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // Lane (r, g) holds head r, dims (4 g + i) kLaneDims + e. A worker with the whole item writes its output.
    // A workgroup whose runs all lie inside one item joins them here, so that they leave one part.
    const uint64_t item_end = item_first + tiles;
    if (t_end == tiles && lane == 0) {
      const uint32_t first = t_begin == 0 ? worker : runs.worker_of(item_first);
      const uint32_t slot = runs.first(first) == item_first ? 0 : 1;
      a.items[static_cast<size_t>(seq) * items + item] =
          Parts{2 * first + slot, worker, (first + slot + kWaves - 1) / kWaves, (worker + (end == item_end ? 1 : 0)) / kWaves};
    }
    const uint32_t block0 = blockIdx.x * kWaves;
    const bool together = !(t_begin == 0 && t_end == tiles) && block0 + kWaves <= runs.workers && runs.first(block0) >= item_first &&
                          runs.first(block0 + kWaves) <= item_end;
    if (together) {
      if (g == 0) wave_sums[wave][r] = make_float2(m, l);
      if (r < in_group) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
          for (uint32_t e = 0; e < kLaneDims; e += 4)
            *reinterpret_cast<f32x4*>(&wave_rows[wave][r][(4 * g + i) * kLaneDims + e]) = f32x4{o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]};
      }
      __syncthreads();
      float* part = part_at(a, block0, 0, part_heads);
      for (uint32_t i = threadIdx.x; i < in_group * (kDim / 4); i += kThreads) {
        const uint32_t h = i / (kDim / 4), dim = i % (kDim / 4) * 4;
        float2 sum[kWaves];
        float top = -INFINITY, total = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
          sum[w] = wave_sums[w][h];
          top = fmaxf(top, sum[w].x);
        }
        const float ref = top == -INFINITY ? 0.0f : top;
        f32x4 all = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
          const float scale = __builtin_amdgcn_exp2f(sum[w].x - ref);
          total += sum[w].y * scale;
          all += *reinterpret_cast<const f32x4*>(&wave_rows[w][h][dim]) * scale;
        }
        float* row_at = part + static_cast<size_t>(h) * a.part_row;
        if (dim == 0) *reinterpret_cast<float2*>(row_at) = make_float2(top, total);
        if (!kAny || dim < a.dim) *reinterpret_cast<f32x4*>(row_at + 4 + dim) = all;
      }
      return;  // the runs end with it
    }
    if (r < in_group) {
      if (t_begin == 0 && t_end == tiles) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
          for (uint32_t e = 0; e < kLaneDims; e += 4)
            write_head<S>(a, seq, q_head0 + r, (4 * g + i) * kLaneDims + e, m, l, f32x4{o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]});
      } else {
        float* part = part_at(a, worker, at == begin ? 0 : 1, part_heads) + static_cast<size_t>(r) * a.part_row;
        if (g == 0) *reinterpret_cast<float2*>(part) = make_float2(m, l);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
          for (uint32_t e = 0; e < kLaneDims; e += 4) {
            const uint32_t dim = (4 * g + i) * kLaneDims + e;
            if (!kAny || dim < a.dim) *reinterpret_cast<f32x4*>(part + 4 + dim) = f32x4{o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]};
          }
      }
    }
    at = item_first + t_end;
  }
}

// Joins the parts of an item, or writes zeros for an empty sequence. A workgroup has a run of kThreads /
// kSlices float4 of the item's rows of all its heads; kSlices groups of its threads take every kSlices-th
// part each and join theirs through LDS, so that an item of many parts is not read one after another.
template <class S, uint32_t kSlices>
__global__ void __launch_bounds__(kThreads) join_kernel(const Attend a) {
  constexpr uint32_t kQuads = kThreads / kSlices;
  __shared__ float2 sums[kSlices > 1 ? kThreads : 1];
  __shared__ f32x4 rows[kSlices > 1 ? kThreads : 1];
  const uint32_t items = a.heads * a.group_blocks;
  const uint32_t seq = blockIdx.x / items, item = blockIdx.x - seq * items;
  const uint32_t head = item / a.group_blocks, gb = item - head * a.group_blocks;
  const uint32_t in_group = min(16u, a.group - gb * 16), q_head0 = head * a.group + gb * 16;
  const uint32_t part_heads = min(16u, a.group), quads = (a.dim + 3) / 4;
  const uint32_t slice = threadIdx.x / kQuads, e = blockIdx.y * kQuads + threadIdx.x % kQuads;
  const uint32_t h = e / quads, dim = (e - h * quads) * 4;
  const bool mine = h < in_group;
  const Parts at = a.items[blockIdx.x];
  const uint32_t first = at.first_slot / 2, slot = at.first_slot & 1;
  // parts: single waves up to the workgroups that lie in the item, these, single waves behind them
  const uint32_t groups = at.group1 > at.group0 ? at.group1 - at.group0 : 0;
  const uint32_t head_parts = groups ? at.group0 * kWaves - first : at.last - first + 1;
  uint32_t count = groups ? head_parts + groups + (at.last + 1 - at.group1 * kWaves) : head_parts;
  if (live_tokens(a, seq) == 0)
    count = 0;  // no worker came here, and `at` holds anything
  else if (at.last == first)
    return;

  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  const auto add = [&](float pm, float pl, f32x4 po) {
    const float top = fmaxf(m, pm), ref = top == -INFINITY ? 0.0f : top;
    const float s = __builtin_amdgcn_exp2f(m - ref), ps = __builtin_amdgcn_exp2f(pm - ref);
    l = l * s + pl * ps;
    o = o * s + po * ps;
    m = top;
  };
  if (mine) {
#pragma unroll 4
    for (uint32_t w = slice; w < count; w += kSlices) {
      const uint32_t behind = w - head_parts;
      const uint32_t worker = w < head_parts ? first + w : behind < groups ? (at.group0 + behind) * kWaves : at.group1 * kWaves + behind - groups;
      const float* part = part_at(a, worker, w == 0 ? slot : 0, part_heads) + static_cast<size_t>(h) * a.part_row;
      const float2 ml = *reinterpret_cast<const float2*>(part);
      add(ml.x, ml.y, *reinterpret_cast<const f32x4*>(part + 4 + dim));
    }
  }
  if constexpr (kSlices > 1) {
    sums[threadIdx.x] = make_float2(m, l);
    rows[threadIdx.x] = o;
#pragma unroll
    for (uint32_t n = kSlices / 2; n > 0; n /= 2) {
      __syncthreads();
      if (slice < n) {
        const float2 ml = sums[threadIdx.x + n * kQuads];
        add(ml.x, ml.y, rows[threadIdx.x + n * kQuads]);
        sums[threadIdx.x] = make_float2(m, l);
        rows[threadIdx.x] = o;
      }
    }
  }
  if (mine && slice == 0) write_head<S>(a, seq, q_head0 + h, dim, m, l, o);
}

template <class S, uint32_t kSlices>
void join(const Attend& a, hipStream_t st) {
  const uint32_t rows = std::min(16u, a.group) * ((a.dim + 3) / 4);
  const dim3 grid(a.seqs * a.heads * a.group_blocks, (rows - 1) / (kThreads / kSlices) + 1);
  join_kernel<S, kSlices><<<grid, dim3(kThreads), 0, st>>>(a);
}

template <class S>
int attend(Attend& a, hipStream_t st) {
  a.workers = std::min(attend_workers(a.dim), 1024 * waves_for<S>(a.dim));
  const dim3 grid(a.workers / kWaves), block(kThreads);
  // a page of whole sixteens, in which 32-bit offsets reach every row, and a head size with a kernel
  const int64_t reach = 16 * a.token_stride + a.dim;
  const bool fast = a.page_tokens % 16 == 0 && reach < (int64_t{1} << 28);
  if (fast && a.dim == 64)
    attend_kernel<S, 64, false><<<grid, block, 0, st>>>(a);
  else if (fast && a.dim == 128)
    attend_kernel<S, 128, false><<<grid, block, 0, st>>>(a);
  else if (fast && a.dim == 256)
    attend_kernel<S, 256, false><<<grid, block, 0, st>>>(a);
  else if (a.dim <= 64)
    attend_kernel<S, 64, true><<<grid, block, 0, st>>>(a);
  else if (a.dim <= 128)
    attend_kernel<S, 128, true><<<grid, block, 0, st>>>(a);
  else
    attend_kernel<S, 256, true><<<grid, block, 0, st>>>(a);
  int rc = launched();
  if (rc != ZO_OK) return rc;
  // as many slices as an item has parts when all sequences are as long as the table
  const uint64_t items = static_cast<uint64_t>(a.seqs) * a.heads * a.group_blocks;
  const uint64_t room = static_cast<uint64_t>(a.width) * a.page_tokens;
  const uint64_t parts = std::min(a.workers / items, room / Mfma<S>::kTile) / kWaves;
  if (parts >= 24)
    join<S, 32>(a, st);
  else if (parts >= 6)
    join<S, 8>(a, st);
  else
    join<S, 2>(a, st);
  return launched();
}

}  // namespace
}  // namespace zo

extern "C" int zo_cache_attend(const zo_attend* p, void* stream) {
  using namespace zo;
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = check_attend(*p);
  if (rc != ZO_OK) return rc;
  if (p->table.seqs == 0 || p->q_heads == 0) return ZO_OK;
  Attend a;
  a.q = static_cast<const char*>(p->q.data);
  a.k = static_cast<const char*>(p->cache.k);
  a.v = static_cast<const char*>(p->cache.v);
  a.out = static_cast<char*>(p->out.data);
  a.lse = p->lse;
  a.items = static_cast<Parts*>(p->work);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(p->work) + attend_items_bytes(p->table.seqs, p->q_heads, p->cache.heads));
  a.ids = p->table.ids;
  a.lengths = p->lengths;
  a.q_seq = p->q.token_stride;
  a.q_head = p->q.head_stride;
  a.out_seq = p->out.token_stride;
  a.out_head = p->out.head_stride;
  a.page_stride = p->cache.page_stride;
  a.head_stride = p->cache.head_stride;
  a.token_stride = p->cache.token_stride;
  a.table_stride = p->table.stride;
  a.seqs = p->table.seqs;
  a.width = p->table.width;
  a.pages = p->cache.pages;
  a.page_tokens = p->cache.page_tokens;
  a.heads = p->cache.heads;
  a.group = p->q_heads / p->cache.heads;
  a.group_blocks = (a.group + 15) / 16;
  a.dim = p->cache.dim;
  a.part_row = (a.dim + 3) / 4 * 4 + 4;
  a.scale = p->scale * 1.4426950408889634f;
  (void)hipGetLastError();
  hipStream_t st = static_cast<hipStream_t>(stream);
  return p->dtype == ZO_F32 ? attend<F32>(a, st) : attend<BF16>(a, st);
}
