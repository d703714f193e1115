// The draw of a token from each row of logits, for gfx950: one workgroup for a row, more for few long rows.
//
// Mathematics. Weights are whole numbers, w_i = round(2^44 exp((l_i - max) / T)), from fp64 exponentials;
// their sums (below 2^62 for 2^18 tokens) are exact in any order, so the token is the same whatever the
// order of the additions, and atomics may be used. Top-k, top-p and min-p each keep a prefix of the
// falling order (logit, then index), so what is kept is all tokens down to a last one. That one is found
// without sorting the row:
//   top-k up to 512  The k-th largest of the threads' own maxima is below no more than k - 1 tokens. What
//                    reaches it (few more than k) goes into a list in LDS, the only part that is sorted
//                    and weighed.
//   top-p alone      (fp32) Weights are added up in 2,888 equal ranges of (l - max) / T; the range in which
//                    top_p's share is reached goes into the list, and tokens above it are kept anyway.
//   bf16             has few values: 8 bits of each power of two between the largest logit and e^-31 of
//                    its weight. Their tokens are counted, and each value is weighed once.
//   otherwise        (more ties than the list holds, a larger k, or a temperature that spreads bf16 over
//                    too many values) Ranges of 32-bit keys of the logits' order are divided until one
//                    key is left, by 2,048 counts and weights at a time.
// The drawn token is then found in index order: weights of runs of 512 tokens, their running sums, and
// the tokens of the run that holds the drawn share.
//
// The row is read from HBM once; later passes read it from the Infinity Cache (of 256 bf16 rows of 304 KB a die has
// 32 at once, and 4 MB of L2: 3.7 times the rows' bytes behind the L2s). A row is one workgroup's chain of passes with
// barriers between; at 256 rows no unit is full (VALU 0.45 busy, LDS 0.17, CUs 0.72: the slowest row ends last).
// Measured, of 151,936 logits: 256 bf16 rows with top-p 0.95 and min-p in 95 to 107 us by the rows, one fp32
// row in 25 us with top-k 50 and in 108 with top-p 0.95 alone. Few long rows are therefore split over workgroups
// where the caller gives a workspace: 33 us.

#include <cmath>
#include <type_traits>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
constexpr uint32_t kBuckets = 2048;
constexpr uint32_t kRun = 512;                  // tokens of a run: 8 for each lane of a wave
constexpr uint32_t kRuns = (1u << 18) / kRun;   // at most
constexpr double kOne = 17592186044416.0;       // 2^44
constexpr uint32_t kList = 4096;                // tokens that are sorted, at most
constexpr int32_t kMostK = 512;                 // top-k by the threads' maxima
constexpr uint32_t kSteps = 1024;               // of the exponential's table, for a factor of 2
constexpr uint32_t kBins = 8192;                // values of a bf16 row that are weighed once each, at most
constexpr uint32_t kSmall = 0x3A7F;             // bf16 below 2^-10 (of which there are very many values) share a bin
constexpr uint32_t kRanges = 2888;              // of 16 steps, down to the smallest weight (45 halvings)

// A logit as it counts: NaN as -inf, +inf as the largest finite number of its type. The median of three of which one is a NaN is
// the smallest; the instruction itself, since the compiler takes the median with -inf for a minimum, NaN or not.
template <class S>
__device__ __forceinline__ float sound(float l) {
  const float most = __uint_as_float(sizeof(typename S::storage) == 2 ? 0x7F7F0000u : 0x7F7FFFFFu);
  float r;
  asm("v_med3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(l), "v"(-INFINITY), "v"(most));
  return r;
}

// Order of logits as unsigned numbers; both zeros are one.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// exp by table and polynomial (P. Tang, 1989): x = (1024 q + j + f) ln 2 / 1024, |f| <= 1/2, exp x = 2^q 2^(j/1024) e^r
// with r = f ln 2 / 1024 below 3.4e-4, where the third-degree Taylor polynomial is off by 6e-16; with the rounding of
// x - r times its weight, the weight is off by less than 2^-49 where its last place is 2^-44. The whole number
// n = 1024 q + j also gives the token's range, counted down from the largest logit.
typedef const __attribute__((address_space(3))) double* LdsTable;  // said, not left to be found out: it is read for each token
struct Weigh {
  double max, inv;  // 1 / temperature
  LdsTable table;   // 2^(44 + j / 1024)
  // n: 0 .. -16 kRanges (of a weight that is not 0). Straight-line code, so that several tokens' chains of
  // operations overlap. Rounding to whole numbers is the addition of a power of two whose last place is 1,
  // and scaling by 2^q an addition to the exponent: fp64 operations take twice as long as others, its
  // conversions longer.
  __device__ __forceinline__ uint64_t operator()(float l, int& n) const {
    const double x = fmax((static_cast<double>(l) - max) * inv, -32.0);  // a weight of 0 from -31.2 on (and of 0 times inf)
    constexpr double kRound = 6755399441055744.0;  // 1.5 2^52
    const double shifted = fma(x, kSteps * 1.4426950408889634074, kRound), k = shifted - kRound;
    n = static_cast<int>(__builtin_bit_cast(uint64_t, shifted));
    const double r = fma(k, -0.69314718055994530942 / kSteps, x);
    const double e = fma(r * r, fma(r, 1.0 / 6, 0.5), r);
    const double t = table[n & (kSteps - 1)];
    const uint64_t y = __builtin_bit_cast(uint64_t, fma(t, e, t));
    const uint32_t scaled = static_cast<uint32_t>(y >> 32) + (static_cast<uint32_t>(n & ~static_cast<int>(kSteps - 1)) << 10);
    const double w = __builtin_bit_cast(double, static_cast<uint64_t>(scaled) << 32 | static_cast<uint32_t>(y));
    return __builtin_bit_cast(uint64_t, w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ uint64_t operator()(float l) const {
    int n;
    return (*this)(l, n);
  }
};

// floor(weight parts / 2^24), weight below 2^62, parts up to 2^24
__device__ __forceinline__ uint64_t share(uint64_t weight, uint32_t parts) {
  return (weight >> 24) * parts + (((weight & 0xFFFFFF) * parts) >> 24);
}

template <class S>
struct Eight {  // 8 logits as they are stored
  u32x4 v[sizeof(typename S::storage) / 2];
};

template <class S>
__device__ __forceinline__ Eight<S> load_eight(const typename S::storage* at) {
  constexpr uint32_t kParts = sizeof(typename S::storage) / 2;
  Eight<S> x;
#pragma unroll
  for (uint32_t c = 0; c < kParts; ++c) x.v[c] = *reinterpret_cast<const u32x4_any*>(at + c * (8 / kParts));
  return x;
}

template <class S>
__device__ __forceinline__ void unpack_eight(const Eight<S>& x, float (&l)[8]) {
  if constexpr (sizeof(typename S::storage) == 2) {
    S::unpack(x.v[0], l);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) l[e] = __uint_as_float(x.v[e / 4][e % 4]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) l[e] = sound<S>(l[e]);
}

// The eight of a row from index i on, -inf behind the end.
template <class S>
__device__ __forceinline__ Eight<S> some_eight(const typename S::storage* row, uint32_t i, uint32_t vocab) {
  if (i + 8 <= vocab) return load_eight<S>(row + i);
  typename S::storage tmp[8];
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    S::store1(&tmp[e], -INFINITY);
    if (i + e < vocab) tmp[e] = row[i + e];
  }
  Eight<S> x;
  __builtin_memcpy(&x, tmp, sizeof x);
  return x;
}

template <class S>
__device__ __forceinline__ void load8(const typename S::storage* row, uint32_t i, uint32_t vocab, float (&l)[8]) {
  unpack_eight<S>(some_eight<S>(row, i, vocab), l);
}

// What a walk hands on of an eight: its logits, or (f takes an Eight) the eight as it is stored.
template <class S, class F>
__device__ __forceinline__ void hand(F& f, uint32_t i, const Eight<S>& x) {
  if constexpr (std::is_invocable<F&, uint32_t, const Eight<S>&>::value) {
    f(i, x);
  } else {
    float l[8];
    unpack_eight<S>(x, l);
    f(i, l);
  }
}

template <class S, uint32_t kBatch, class F>
__device__ __forceinline__ uint32_t walk_batches(const typename S::storage* row, uint32_t vocab, uint32_t run0, F& f) {
  constexpr uint32_t kStep = kWaves * kRun;
  const uint32_t lane0 = threadIdx.x % 64 * 8;
#pragma unroll 1
  for (; run0 + (kBatch - 1) * kStep + kRun <= vocab; run0 += kBatch * kStep) {
    Eight<S> x[kBatch];
#pragma unroll
    for (uint32_t u = 0; u < kBatch; ++u) x[u] = load_eight<S>(row + run0 + u * kStep + lane0);
#pragma unroll
    for (uint32_t u = 0; u < kBatch; ++u) hand<S>(f, run0 + u * kStep + lane0, x[u]);
  }
  return run0;
}

// Calls f(index of the first, logits) for the eights of a row that this lane has: wave w takes runs w, w + kWaves,
// .. (a lane 8 tokens of each), kBatch of them loaded before the first is used, as long as there are so many. All
// lanes of a wave make the same calls; tokens behind the end are -inf.
template <class S, uint32_t kBatch, class F>
__device__ __forceinline__ void walk(const typename S::storage* row, uint32_t vocab, F f) {
  uint32_t run0 = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * kRun;
  run0 = walk_batches<S, kBatch>(row, vocab, run0, f);
  if constexpr (kBatch > 2) run0 = walk_batches<S, 2>(row, vocab, run0, f);
#pragma unroll 1
  for (; run0 < vocab; run0 += kWaves * kRun) {
    const uint32_t i = run0 + threadIdx.x % 64 * 8;
    hand<S>(f, i, some_eight<S>(row, i, vocab));
  }
}

// The sum over a wave, the same in all lanes: rows of 16 by data-parallel moves, the four rows in scalars.
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
  const auto add = [&](auto ctrl) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(v), ctrl.value, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(v >> 32), ctrl.value, 0xF, 0xF, true);
    v += static_cast<uint64_t>(hi) << 32 | lo;
  };
  add(std::integral_constant<int, 0xB1>{});   // neighbours
  add(std::integral_constant<int, 0x4E>{});   // pairs of a quad
  add(std::integral_constant<int, 0x141>{});  // quads of a half row
  add(std::integral_constant<int, 0x140>{});  // halves of a row
  uint64_t sum = 0;
#pragma unroll
  for (int row = 0; row < 64; row += 16) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), row);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), row);
    sum += static_cast<uint64_t>(hi) << 32 | lo;
  }
  return sum;
}

__device__ __forceinline__ uint64_t wave_upto(uint64_t v) {  // sum over this and the lanes before
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t lower = __shfl_up(v, m, 64);
    if (threadIdx.x % 64 >= static_cast<uint32_t>(m)) v += lower;
  }
  return v;
}

struct Lds {
  union {
    struct {  // find_cut
      uint64_t weight[kBuckets];
      uint32_t count[kBuckets];
    };
    uint64_t range[kRanges];
    float kept[4 * kThreads];  // a few logits for each thread
    struct {                   // bf16 by value
      uint64_t bin_weight[kBins];
      uint32_t bin_count[kBins + 1];
    };
    struct {
      uint64_t list[kList];         // ~key << 32 | index: in rising order, tokens in falling order
      uint64_t list_weight[kList];
    };
  };
  double table[kSteps];
  uint64_t part_weight[kWaves];
  uint64_t part_count[kWaves];
  uint64_t run_weight[kRuns];
  uint32_t run_ties[kRuns];
  uint32_t thread_max[kThreads];
  uint64_t before_weight, found_weight, small_weight;
  uint32_t before_count, found, found_count, listed, bound[2];
};

// Sums of (weight, count) over the threads before this one, and over all.
__device__ __forceinline__ void block_before(Lds& s, uint64_t w, uint64_t c, uint64_t& w_before, uint64_t& c_before, uint64_t& w_all,
                                             uint64_t& c_all) {
  const uint64_t wu = wave_upto(w), cu = wave_upto(c);
  __syncthreads();
  if (threadIdx.x % 64 == 63) {
    s.part_weight[threadIdx.x / 64] = wu;
    s.part_count[threadIdx.x / 64] = cu;
  }
  __syncthreads();
  w_before = wu - w;
  c_before = cu - c;
  w_all = c_all = 0;
  for (uint32_t i = 0; i < kWaves; ++i) {
    if (i < threadIdx.x / 64) {
      w_before += s.part_weight[i];
      c_before += s.part_count[i];
    }
    w_all += s.part_weight[i];
    c_all += s.part_count[i];
  }
}

// The last token that is kept: those of a larger key are, and of the same key those up to `last`.
struct Cut {
  uint32_t key, last;
  uint64_t weight;  // of all that is kept (find_cut)
  __device__ __forceinline__ bool keeps(uint32_t k, uint32_t index) const { return k > key || (k == key && index <= last); }
};

// The index of the n-th token (from 1) of a key.
template <class S>
__device__ __forceinline__ uint32_t index_of_tie(Lds& s, const typename S::storage* row, uint32_t vocab, uint32_t key, uint32_t n) {
  const uint32_t runs = (vocab + kRun - 1) / kRun;
  for (uint32_t run = threadIdx.x / 64; run < runs; run += kWaves) {
    float l[8];
    load8<S>(row, run * kRun + threadIdx.x % 64 * 8, vocab, l);
    uint32_t ties = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) ties += key_of(l[e]) == key ? 1 : 0;
    ties = static_cast<uint32_t>(wave_sum(ties));
    if (threadIdx.x % 64 == 0) s.run_ties[run] = ties;
  }
  __syncthreads();
  const uint64_t mine = threadIdx.x < runs ? s.run_ties[threadIdx.x] : 0;
  uint64_t before, all, x, y;
  block_before(s, 0, mine, x, before, y, all);
  if (before < n && n <= before + mine) {  // one run of all
    s.found = threadIdx.x;
    s.before_count = static_cast<uint32_t>(before);
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const uint32_t i0 = s.found * kRun + threadIdx.x * 8;
    float l[8];
    load8<S>(row, i0, vocab, l);
    uint32_t ties = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) ties += key_of(l[e]) == key ? 1 : 0;
    uint32_t at = s.before_count + static_cast<uint32_t>(wave_upto(ties)) - ties;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (key_of(l[e]) == key && ++at == n) s.found_count = i0 + e;
  }
  __syncthreads();
  return s.found_count;
}

// Sorts the first n entries of the list (n <= kList, all different), smallest first. Up to 512 by counting for each
// how many are smaller, an entry's count shared by as many waves as there are; longer ones by a bitonic network.
__device__ __forceinline__ void sort_list(Lds& s, uint32_t n) {
  if (n <= 512) {
    const uint32_t size = n <= 64 ? 64 : (n + 63) / 64 * 64, copies = kThreads / size, copy = threadIdx.x / size;
    const uint32_t i = threadIdx.x - copy * size;
    if (threadIdx.x < n) s.thread_max[threadIdx.x] = 0;  // ranks
    __syncthreads();
    const uint64_t mine = i < n ? s.list[i] : 0;
    if (i < n && copy < copies) {
      uint32_t rank = 0;
      const uint32_t end = (copy + 1) * n / copies;
#pragma unroll 8
      for (uint32_t j = copy * n / copies; j < end; ++j) rank += s.list[j] < mine ? 1 : 0;
      atomicAdd(&s.thread_max[i], rank);
    }
    __syncthreads();
    if (threadIdx.x < n) s.list[s.thread_max[threadIdx.x]] = mine;
    __syncthreads();
    return;
  }
  uint32_t size = 1024;
  while (size < n) size *= 2;
  for (uint32_t i = n + threadIdx.x; i < size; i += kThreads) s.list[i] = ~0ull;
  for (uint32_t run = 2; run <= size; run *= 2)
    for (uint32_t gap = run / 2; gap > 0; gap /= 2) {
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < size / 2; i += kThreads) {
        const uint32_t a = 2 * i - (i & (gap - 1)), b = a + gap;
        const uint64_t x = s.list[a], y = s.list[b];
        if ((x > y) == ((a & run) == 0)) {
          s.list[a] = y;
          s.list[b] = x;
        }
      }
    }
  __syncthreads();
}

// Adds the tokens of a row from logit `low` to `high` to the list; false: there are more than it holds.
template <class S>
__device__ __forceinline__ bool fill_list(Lds& s, const typename S::storage* row, uint32_t vocab, float low, float high) {
  if (threadIdx.x == 0) s.listed = 0;
  __syncthreads();
  walk<S, 8>(row, vocab, [&](uint32_t i, const float(&l)[8]) {
    float best = l[0];
#pragma unroll
    for (uint32_t e = 1; e < 8; ++e) best = fmaxf(best, l[e]);
    if (!(best >= low)) return;  // most lanes of most waves
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      if (!(l[e] >= low && l[e] <= high) || i + e >= vocab) continue;
      const uint32_t at = atomicAdd(&s.listed, 1u);
      if (at < kList) s.list[at] = static_cast<uint64_t>(~key_of(l[e])) << 32 | (i + e);
    }
  });
  __syncthreads();
  return s.listed <= kList;
}

// Weighs the sorted list and finds what top-k, top-p and min-p keep of it, given the weight above it. all: weight
// of everything that top-p shares out; 0: of the list's first k. Returns the number kept; their weights
// are in list_weight.
__device__ __forceinline__ uint32_t cut_list(Lds& s, uint32_t n, const Weigh& weigh, uint32_t k, uint64_t above, uint64_t all, bool by_weight, uint32_t parts,
                             uint64_t least) {
  constexpr uint32_t kEach = kList / kThreads;
  uint64_t w[kEach], sum = 0;
#pragma unroll
  for (uint32_t j = 0; j < kEach; ++j) {
    const uint32_t i = threadIdx.x * kEach + j;
    w[j] = i < n && i < k ? (weigh(logit_of(~static_cast<uint32_t>(s.list[i] >> 32)))) : 0;
    s.list_weight[i] = w[j];
    sum += w[j];
  }
  uint64_t before, total, x, y;
  block_before(s, sum, 0, before, x, total, y);
  uint64_t need = ~0ull;
  if (by_weight) {
    need = share(all ? all : total, parts);
    if (need == 0) need = 1;
  }
  uint32_t kept = 0;
  before += above;
#pragma unroll
  for (uint32_t j = 0; j < kEach; ++j) {  // each keeps a prefix
    if (w[j] > 0 && before < need && w[j] >= least) ++kept;
    before += w[j];
  }
  block_before(s, 0, kept, x, before, y, total);
  return static_cast<uint32_t>(total);
}

// The cut at which the count reaches `most`, or (by_weight) the weight reaches `need`, whichever is
// asked for; false: the row's weights end before. Tokens of no weight do not count.
// kSplit: the kernel that calls it. A function of its own for each lets the compiler see where its arguments come
// from; shared by two kernels, `weigh` and `cut` are kept in memory and read from there for each token, and passes over
// all tokens took almost twice as long.
template <class S, bool kSplit>
__device__ __attribute__((noinline)) bool find_cut(Lds& s, const typename S::storage* row, uint32_t vocab, const Weigh& weigh, uint32_t top,
                                                   bool by_weight, uint64_t need, Cut& cut) {
  uint32_t hi = top, lo = 0;
  uint64_t above_weight = 0, above_count = 0;
  for (;;) {
    const uint32_t span = hi - lo;
    const int shift = span < kBuckets ? 0 : 32 - __clz(span) - 11;
    for (uint32_t b = threadIdx.x; b < kBuckets; b += kThreads) {
      s.weight[b] = 0;
      s.count[b] = 0;
    }
    __syncthreads();
    walk<S, 2>(row, vocab, [&](uint32_t, const float(&l)[8]) {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t key = key_of(l[e]);
        if (key < lo || key > hi) continue;
        const uint64_t w = weigh(l[e]);
        if (w == 0) continue;
        const uint32_t b = (hi - key) >> shift;
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.weight[b]), static_cast<unsigned long long>(w));
        atomicAdd(&s.count[b], 1u);
      }
    });
    __syncthreads();
    constexpr uint32_t kEach = kBuckets / kThreads;
    uint64_t w[kEach], c[kEach], w_sum = 0, c_sum = 0, w_before, c_before, w_all, c_all;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
      w[j] = s.weight[kEach * threadIdx.x + j];
      c[j] = s.count[kEach * threadIdx.x + j];
      w_sum += w[j];
      c_sum += c[j];
    }
    block_before(s, w_sum, c_sum, w_before, c_before, w_all, c_all);
    if ((by_weight ? above_weight + w_all : above_count + c_all) < need) return false;
    uint64_t wb = above_weight + w_before, cb = above_count + c_before;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
      const uint64_t was = by_weight ? wb : cb, now = was + (by_weight ? w[j] : c[j]);
      if (was < need && now >= need) {  // one bucket of all
        s.found = kEach * threadIdx.x + j;
        s.before_weight = wb;
        s.before_count = static_cast<uint32_t>(cb);
        s.found_weight = w[j];
        s.found_count = static_cast<uint32_t>(c[j]);
      }
      wb += w[j];
      cb += c[j];
    }
    __syncthreads();
    const uint32_t found = s.found, count = s.found_count;
    above_weight = s.before_weight;
    above_count = s.before_count;
    const uint64_t found_weight = s.found_weight;
    __syncthreads();
    hi -= found << shift;
    const uint32_t range = shift == 0 ? 0 : (1u << shift) - 1;
    lo = hi - lo > range ? hi - range : lo;
    if (lo == hi || shift == 0) {
      const uint64_t each = found_weight / count;
      cut.key = hi;
      uint64_t ties = by_weight ? (need - above_weight + each - 1) / each : need - above_count;
      if (ties > count) ties = count;
      cut.weight = above_weight + ties * each;
      cut.last = vocab;
      if (ties < count) cut.last = index_of_tie<S>(s, row, vocab, hi, static_cast<uint32_t>(ties));
      return true;
    }
  }
}

struct Draw {
  const char* logits;
  int64_t row_stride;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* logprobs;
  uint32_t vocab;
};

// bf16 values in their order, neighbouring values neighbouring numbers; all below 2^-10 are 0.
__device__ __forceinline__ int code_of(float l) {
  const uint32_t bits = __float_as_uint(l), a = (bits & 0x7FFFFFFFu) >> 16;
  const int up = static_cast<int>(max(a, kSmall) - kSmall);
  return bits & 0x80000000u ? -up : up;
}
__device__ __forceinline__ float value_of(int code) {  // not 0
  const uint32_t a = static_cast<uint32_t>(code < 0 ? -code : code) + kSmall;
  return __uint_as_float((code < 0 ? 0x8000u | a : a) << 16);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// code_top - code of two stored bf16, modulo 2^16, at most `bins`: what is larger than the largest (a NaN) or weighs
// nothing gets `bins` too, since codes span less than 2^16.
__device__ __forceinline__ u16x2 bins_of(uint32_t pair, int code_top, uint32_t bins) {
  const u16x2 a = __builtin_bit_cast(u16x2, pair & 0x7FFF7FFFu);
  const u16x2 up = __builtin_elementwise_max(a, u16x2(static_cast<unsigned short>(kSmall))) - u16x2(static_cast<unsigned short>(kSmall));
  const i16x2 sign = __builtin_bit_cast(i16x2, pair) >> 15;
  const i16x2 code = (__builtin_bit_cast(i16x2, up) ^ sign) - sign;
  const u16x2 bin = __builtin_bit_cast(u16x2, i16x2(static_cast<short>(code_top)) - code);
  return __builtin_elementwise_min(bin, u16x2(static_cast<unsigned short>(bins)));
}

// Adds the weights of the tokens in `small` (few of a row).
__device__ __forceinline__ void add_small(Lds& s, const float (&l)[8], uint32_t small, const Weigh& weigh) {
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e)
    if (small >> e & 1) atomicAdd(reinterpret_cast<unsigned long long*>(&s.small_weight), static_cast<unsigned long long>(weigh(l[e])));
}

// A bf16 row by value: its weights come from one exponential for each value instead of each token, and top-k and
// top-p from a count of each value's tokens. false: the values that weigh anything are more than the bins, or a cut falls
// among those below 2^-10; nothing is done then.
template <bool kSplit>
__device__ bool cut_by_value(Lds& s, const uint16_t* row, uint32_t vocab, const Weigh& weigh, int code_top, uint32_t bins,
                             uint32_t k, bool by_weight, uint32_t parts, Cut& cut) {
  const bool cuts = k > 0 || by_weight;
  for (uint32_t i = threadIdx.x; i <= bins; i += kThreads) s.bin_count[i] = 0;
  if (threadIdx.x == 0) s.small_weight = 0;
  __syncthreads();
  if (cuts) {
    // the bin of small values; where it would be `bins`, they weigh nothing, and `bins` is that of all that does not count
    const uint32_t small_bin = static_cast<uint32_t>(code_top) < bins ? static_cast<uint32_t>(code_top) : ~0u;
    walk<BF16, 4>(row, vocab, [&](uint32_t, const Eight<BF16>& x) {
      uint32_t small = 0;
#pragma unroll
      for (uint32_t c = 0; c < 4; ++c) {
        const u16x2 bin = bins_of(x.v[0][c], code_top, bins);
        atomicAdd(&s.bin_count[bin.x], 1u);  // (`bins` is a bin of what does not count)
        atomicAdd(&s.bin_count[bin.y], 1u);
        small |= (bin.x == small_bin ? 1u << 2 * c : 0u) | (bin.y == small_bin ? 2u << 2 * c : 0u);
      }
      if (small) {
        float l[8];
        unpack_eight<BF16>(x, l);
        add_small(s, l, small, weigh);
      }
    });
  }
  __syncthreads();
  constexpr uint32_t kEach = kBins / kThreads;
  uint64_t each[kEach], w_sum = 0, c_sum = 0, w_before, c_before, w_all, c_all;
  uint32_t count[kEach];
  const uint32_t i0 = threadIdx.x * kEach;
#pragma unroll
  for (uint32_t j = 0; j < kEach; ++j) {
    const int code = code_top - static_cast<int>(i0 + j);
    const bool in = i0 + j < bins;
    each[j] = in && code != 0 ? weigh(value_of(code)) : 0;
    count[j] = in && (code == 0 || each[j] > 0) ? s.bin_count[i0 + j] : 0;
    s.bin_weight[i0 + j] = each[j];
    w_sum += in && code == 0 ? s.small_weight : count[j] * each[j];
    c_sum += count[j];
  }
  if (!cuts) {
    __syncthreads();
    return true;
  }
  block_before(s, w_sum, c_sum, w_before, c_before, w_all, c_all);
  // first the count's bin, then, with the weight down to there, the weight's
  uint64_t all = w_all;
  bool found = false;
  for (int round = 0; round < 2; ++round) {
    const bool weight = round == 1;
    if (weight ? !by_weight : k == 0 || c_all < k) continue;
    uint64_t need = weight ? share(all, parts) : k;
    if (need == 0) need = 1;
    uint64_t wb = w_before, cb = c_before;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
      const bool small = code_top == static_cast<int>(i0 + j);
      const uint64_t w = small ? s.small_weight : count[j] * each[j];
      const uint64_t was = weight ? wb : cb, now = was + (weight ? w : count[j]);
      if (was < need && now >= need) {  // one bin of all
        const uint64_t ties = weight ? (small ? 0 : (need - wb + each[j] - 1) / each[j]) : need - cb;
        s.found = i0 + j;
        s.found_count = small || ties < count[j] ? static_cast<uint32_t>(ties) : 0;  // 0: all of its tokens
        s.before_weight = wb + ties * each[j];
      }
      wb += w;
      cb += count[j];
    }
    __syncthreads();
    found = true;
    all = s.before_weight;
    const int code = code_top - static_cast<int>(s.found);
    const uint32_t ties = s.found_count;
    __syncthreads();
    if (code == 0) return false;
    cut.key = key_of(value_of(code));
    cut.last = ties;  // for now
  }
  if (found && cut.last > 0)
    cut.last = index_of_tie<BF16>(s, row, vocab, cut.key, cut.last);
  else
    cut.last = vocab;
  return true;
}

// The largest key that `takes` does not take, for a `takes` that takes all keys from one on, and not 0. A wave tries
// 64 keys at a time.
template <class F>
__device__ __forceinline__ uint32_t last_untaken(F takes) {
  uint32_t key = 0;
#pragma unroll 1
  for (int shift = 26; shift > -6; shift -= 6) {
    const int at = shift < 0 ? 0 : shift;
    const uint32_t trial = key + ((threadIdx.x % 64) << at);
    const bool mine = shift >= 0 || threadIdx.x % 64 < 4;  // the last round has two bits
    key += (__popcll(__ballot(mine && !takes(trial))) - 1) << at;
  }
  return key;
}

// The largest key whose weight does not reach range `edge`.
__device__ __forceinline__ uint32_t range_edge(const Weigh& weigh, uint32_t top, int32_t edge) {
  return last_untaken([&](uint32_t key) {
    if (key <= key_of(-INFINITY)) return false;
    if (key >= top) return edge >= 0 || key > top;
    int n;
    return weigh(logit_of(key), n) > 0 && -n / 16 <= edge;
  });
}

// What a row is drawn with.
__device__ __forceinline__ float temperature_of(const Draw& a, uint32_t b) { return a.temperature ? a.temperature[b] : 1.0f; }
struct Asked {
  int32_t k;
  bool by_count, by_weight;
  uint32_t parts, draw;  // of 2^24
  uint64_t least;        // weight
  __device__ __forceinline__ Asked(const Draw& a, uint32_t b) {
    const float p = a.top_p ? a.top_p[b] : 1.0f, mp = a.min_p ? a.min_p[b] : 0.0f, u = a.u[b];
    k = a.top_k ? a.top_k[b] : 0;
    by_count = k > 0 && static_cast<uint32_t>(k) < a.vocab;
    by_weight = p < 1.0f;
    parts = p > 0.0f ? static_cast<uint32_t>(rint(static_cast<double>(fminf(p, 1.0f)) * 16777216.0)) : 0u;
    least = mp > 0.0f ? static_cast<uint64_t>(rint(static_cast<double>(mp < 1.0f ? mp : 1.0f) * kOne)) : 1ull;
    draw = !(u > 0.0f) ? 0u : u >= 1.0f ? 0xFFFFFFu : static_cast<uint32_t>(u * 16777216.0f);
  }
};

// The draw of a row that has no weight, or takes its largest logit.
__device__ __forceinline__ void draw_largest(const Draw& a, uint32_t b, float max, uint32_t first) {
  if (threadIdx.x != 0) return;
  a.tokens[b] = max == -INFINITY ? -1 : static_cast<int32_t>(first);
  if (a.logprobs) a.logprobs[b] = max == -INFINITY ? -INFINITY : 0.0f;
}

// The draw of a row with top-k from the list of n tokens that hold its first k.
__device__ __forceinline__ void draw_listed(Lds& s, const Draw& a, uint32_t b, uint32_t n, const Weigh& weigh, const Asked& asked) {
  sort_list(s, n);
  const uint32_t kept = cut_list(s, n, weigh, static_cast<uint32_t>(asked.k), 0, 0, asked.by_weight, asked.parts, asked.least);
  // what is kept in the order of indices, each with its place in the list
  uint64_t entry = 0;
  const uint32_t i = threadIdx.x;
  if (i < kept) entry = s.list[i] << 32 | i;
  __syncthreads();
  if (i < kept) s.list[i] = entry;
  sort_list(s, kept);
  const uint64_t w = i < kept ? s.list_weight[s.list[i] & 0xFFFFFFFFu] : 0;
  uint64_t before, all, x, y;
  block_before(s, w, 0, before, x, all, y);
  const uint64_t target = share(all, asked.draw);
  if (before <= target && target < before + w) {
    a.tokens[b] = static_cast<int32_t>(s.list[i] >> 32);
    if (a.logprobs) a.logprobs[b] = static_cast<float>(log(static_cast<double>(w) / static_cast<double>(all)));
  }
}

// The draw of a row from the kept weight of each of its runs.
template <class S>
__device__ __forceinline__ void draw_from_runs(Lds& s, const Draw& a, uint32_t b, const typename S::storage* row, const Weigh& weigh,
                                               const Asked& asked, const Cut& cut) {
  const uint32_t runs = (a.vocab + kRun - 1) / kRun;
  const uint64_t in_run = threadIdx.x < runs ? s.run_weight[threadIdx.x] : 0;
  uint64_t w_before, w_all, x, y;
  block_before(s, in_run, 0, w_before, x, w_all, y);
  const uint64_t target = share(w_all, asked.draw);
  if (w_before <= target && target < w_before + in_run) {  // one run of all
    s.found = threadIdx.x;
    s.before_weight = w_before;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;

  // the token inside the run
  const uint32_t i0 = s.found * kRun + threadIdx.x * 8;
  float l[8];
  load8<S>(row, i0, a.vocab, l);
  uint64_t w[8], sum = 0;
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    w[e] = cut.keeps(key_of(l[e]), i0 + e) ? (weigh(l[e])) : 0;
    if (w[e] < asked.least) w[e] = 0;
    sum += w[e];
  }
  uint64_t upto = s.before_weight + wave_upto(sum) - sum;
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    if (upto <= target && target < upto + w[e]) {
      a.tokens[b] = static_cast<int32_t>(i0 + e);
      if (a.logprobs) a.logprobs[b] = static_cast<float>(log(static_cast<double>(w[e]) / static_cast<double>(w_all)));
    }
    upto += w[e];
  }
}

// Few long rows, each split over workgroups of 8 runs, a run for each wave and 8 tokens for each lane. Sums are exact in
// any order, so this gives the token that one workgroup gives; what it cannot serve (a larger k, lists that do not
// hold a part's or the row's tokens) is left to that code.
//   1. the largest logit of each part, and of each 64 tokens of it
//   2. top-p without top-k: the part's weights by ranges, and these by 64 to the halving
//   3. top-k: the bound from the maxima of 64 tokens, by counting; top-p: the halving and the range in it at which
//      the share is reached, from the parts' sums; then the part's list, and the weights of its runs above it
//   4. one workgroup for a row sorts the joined list, cuts it and draws
// 4 fp32 rows of 151,936 with top-p 0.95: 5, 7, 10 and 19 us (one workgroup for each: 108); with top-k 50 4, 2, 8 and 14 (25).
constexpr uint32_t kPartThreads = 512, kPartWaves = kPartThreads / 64;
constexpr uint32_t kHalvings = (kRanges + 63) / 64, kAllRanges = 64 * kHalvings;
constexpr uint32_t kPartList = 1024;
constexpr uint32_t kPartGroups = kDrawPart / 64;
static_assert(kPartThreads * 8 == kDrawPart && kPartWaves * kRun == kDrawPart, "a run for each wave");
static_assert(kDrawPart * 64ull >= 1u << 18, "a lane for each part");
static_assert(kDrawPartWords == 2 + kPartGroups / 2 + 64 + kAllRanges + kPartList + kPartWaves, "words of a part");

struct Split {
  uint64_t *best, *listed, *halving, *range, *list, *run, *sums;
  uint32_t* group_max;
  uint32_t parts;
  __device__ __forceinline__ Split(uint64_t* work, uint32_t b, uint32_t vocab) {
    parts = (vocab + kDrawPart - 1) / kDrawPart;
    best = work + static_cast<size_t>(b) * (parts * kDrawPartWords + kDrawRowWords);
    listed = best + parts;
    halving = listed + parts;
    range = halving + parts * 64;
    list = range + parts * kAllRanges;
    run = list + parts * kPartList;
    group_max = reinterpret_cast<uint32_t*>(run + parts * kPartWaves);
    sums = run + parts * (kPartWaves + kPartGroups / 2);
  }
  // The row's largest key << 32 | ~its lowest index; every wave for itself.
  __device__ __forceinline__ uint64_t largest() const {
    uint64_t v = threadIdx.x % 64 < parts ? best[threadIdx.x % 64] : 0;
#pragma unroll
    for (int m = 32; m > 0; m /= 2) {
      const uint64_t other = __shfl_xor(v, m, 64);
      v = other > v ? other : v;
    }
    return v;
  }
};

enum class Way { kLargest, kCount, kWeight, kAll, kOther };
__device__ __forceinline__ Way way_of(const Draw& a, uint32_t b, const Asked& asked, float max) {
  if (max == -INFINITY || !(temperature_of(a, b) > 0.0f)) return Way::kLargest;
  if (asked.by_count) return asked.k <= kMostK ? Way::kCount : Way::kOther;
  return asked.by_weight ? Way::kWeight : Way::kAll;
}

template <class S>
__device__ __forceinline__ const typename S::storage* row_of(const Draw& a, uint32_t b) {
  return reinterpret_cast<const typename S::storage*>(a.logits) + static_cast<int64_t>(b) * a.row_stride;
}

template <class S>
__global__ void __launch_bounds__(kPartThreads) split_max_kernel(const Draw a, uint64_t* work) {
  __shared__ uint64_t wave_best[kPartWaves];
  const uint32_t b = blockIdx.y, part = blockIdx.x;
  const Split to(work, b, a.vocab);
  const uint32_t i = part * kDrawPart + threadIdx.x * 8;
  float l[8], mine = -INFINITY;
  load8<S>(row_of<S>(a, b), i, a.vocab, l);
  uint32_t at = 0xFFFFFFFFu;
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    at = l[e] > mine ? i + e : at;
    mine = l[e] > mine ? l[e] : mine;
  }
  uint64_t best = static_cast<uint64_t>(key_of(mine)) << 32 | (0xFFFFFFFFu - at);
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint64_t other = __shfl_xor(best, m, 64);
    best = other > best ? other : best;
    if (m == 4 && threadIdx.x % 8 == 0) to.group_max[part * kPartGroups + threadIdx.x / 8] = static_cast<uint32_t>(best >> 32);
  }
  if (threadIdx.x % 64 == 0) wave_best[threadIdx.x / 64] = best;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (uint32_t w = 1; w < kPartWaves; ++w) best = wave_best[w] > best ? wave_best[w] : best;
  to.best[part] = best;
}

template <class S>
__global__ void __launch_bounds__(kPartThreads) split_ranges_kernel(const Draw a, uint64_t* work) {
  __shared__ double table[kSteps];
  __shared__ uint64_t range[kAllRanges];
  const uint32_t b = blockIdx.y, part = blockIdx.x;
  const Split to(work, b, a.vocab);
  const float max = logit_of(static_cast<uint32_t>(to.largest() >> 32));
  if (way_of(a, b, Asked(a, b), max) != Way::kWeight) return;  // all of the workgroup
  float l[8];
  load8<S>(row_of<S>(a, b), part * kDrawPart + threadIdx.x * 8, a.vocab, l);
  for (uint32_t i = threadIdx.x; i < kSteps; i += kPartThreads) table[i] = exp2(44.0 + static_cast<double>(i) / kSteps);
  for (uint32_t i = threadIdx.x; i < kAllRanges; i += kPartThreads) range[i] = 0;
  __syncthreads();
  const Weigh weigh{static_cast<double>(max), 1.0 / static_cast<double>(temperature_of(a, b)), (LdsTable)table};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    int n;
    const uint64_t w = weigh(l[e], n);
    if (w > 0) atomicAdd(reinterpret_cast<unsigned long long*>(&range[-n / 16]), static_cast<unsigned long long>(w));
  }
  __syncthreads();
  for (uint32_t h = threadIdx.x / 64; h < 64; h += kPartWaves) {
    uint64_t sum = 0;
    if (h < kHalvings) {
      const uint64_t w = range[h * 64 + threadIdx.x % 64];
      to.range[part * kAllRanges + h * 64 + threadIdx.x % 64] = w;
      sum = wave_sum(w);
    }
    if (threadIdx.x % 64 == 0) to.halving[part * 64 + h] = sum;
  }
}

// The sums of 64 numbers over the parts, `stride` apart, and the first of them with which `need` is reached: its index, and the
// sum before it. The same in all waves.
struct Reached {
  uint32_t index;
  uint64_t before, all;
};
template <class F>
__device__ __forceinline__ Reached reach(uint64_t (*sums)[64], const uint64_t* from, uint32_t stride, uint32_t parts, F need_of) {
  const uint32_t lane = threadIdx.x % 64;
  uint64_t sum = 0;
#pragma unroll 4
  for (uint32_t part = threadIdx.x / 64; part < parts; part += kPartWaves) sum += from[static_cast<size_t>(part) * stride + lane];
  __syncthreads();  // earlier sums are read
  sums[threadIdx.x / 64][lane] = sum;
  __syncthreads();
  sum = 0;
  for (uint32_t w = 0; w < kPartWaves; ++w) sum += sums[w][lane];
  const uint64_t upto = wave_upto(sum), all = __shfl(upto, 63, 64), need = need_of(all);
  const uint64_t there = __ballot(upto >= need);
  const uint32_t index = there == 0 ? 0 : static_cast<uint32_t>(__builtin_ctzll(there));  // (need is never above all)
  return Reached{index, __shfl(upto - sum, static_cast<int>(index), 64), all};
}

template <class S>
__global__ void __launch_bounds__(kPartThreads) split_list_kernel(const Draw a, uint64_t* work) {
  __shared__ double table[kSteps];
  __shared__ uint64_t sums[kPartWaves][64];
  __shared__ uint32_t counts[16], bound[2], listed;
  const uint32_t b = blockIdx.y, part = blockIdx.x;
  const Split to(work, b, a.vocab);
  const uint32_t top = static_cast<uint32_t>(to.largest() >> 32);
  const float max = logit_of(top);
  const Asked asked(a, b);
  const Way way = way_of(a, b, asked, max);
  if (way == Way::kLargest || way == Way::kOther) return;  // all of the workgroup
  const uint32_t i0 = part * kDrawPart + threadIdx.x * 8;
  float l[8];
  load8<S>(row_of<S>(a, b), i0, a.vocab, l);
  const Weigh weigh{static_cast<double>(max), 1.0 / static_cast<double>(temperature_of(a, b)), (LdsTable)table};
  if (threadIdx.x == 0) listed = 0;

  float low = INFINITY, high = INFINITY;  // of the list
  uint32_t above = 0;                     // keys above this are kept, whatever the list says
  if (way == Way::kCount) {
    // the upper half of the key of the k-th largest of the maxima of 64 tokens
    const uint32_t groups = to.parts * kPartGroups;
    uint32_t m[64 * kPartGroups / kPartThreads];
#pragma unroll
    for (uint32_t j = 0; j < 64 * kPartGroups / kPartThreads; ++j) {
      const uint32_t g = j * kPartThreads + threadIdx.x;
      m[j] = g < groups ? to.group_max[g] : 0;
    }
    if (threadIdx.x < 16) counts[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key = 0;
    for (uint32_t bit = 0x80000000u, turn = 0; turn < 16; bit /= 2, ++turn) {
      uint32_t count = 0;
#pragma unroll
      for (uint32_t j = 0; j < 64 * kPartGroups / kPartThreads; ++j) count += __popcll(__ballot(m[j] >= (key | bit)));
      if (threadIdx.x % 64 == 0) atomicAdd(&counts[turn], count);
      __syncthreads();
      if (counts[turn] >= static_cast<uint32_t>(asked.k)) key |= bit;
    }
    low = key > key_of(-INFINITY) ? logit_of(key) : -INFINITY;  // (a key below that of -inf takes everything in)
  } else {
    for (uint32_t i = threadIdx.x; i < kSteps; i += kPartThreads) table[i] = exp2(44.0 + static_cast<double>(i) / kSteps);
    __syncthreads();
  }
  if (way == Way::kWeight) {
    uint64_t need = 0;
    const Reached halving = reach(sums, to.halving, 64, to.parts, [&](uint64_t all) {
      need = share(all, asked.parts);
      if (need == 0) need = 1;
      return need;
    });
    const Reached in = reach(sums, to.range + halving.index * 64, kAllRanges, to.parts, [&](uint64_t) { return need - halving.before; });
    const int32_t found = static_cast<int32_t>(halving.index * 64 + in.index);
    if (part == 0 && threadIdx.x == 0) {
      to.sums[0] = halving.before + in.before;
      to.sums[1] = halving.all;
    }
    if (threadIdx.x < 128) {
      const uint32_t key = range_edge(weigh, top, threadIdx.x < 64 ? found : found - 1);
      if (threadIdx.x % 64 == 0) bound[threadIdx.x / 64] = key;
    }
    __syncthreads();
    low = logit_of(bound[0] + 1);
    high = logit_of(bound[1]);
    above = bound[1];
  }
  if (way != Way::kCount) {
    uint64_t sum = 0;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      const uint64_t w = weigh(l[e]);
      sum += key_of(l[e]) > above && w >= asked.least ? w : 0;
    }
    sum = wave_sum(sum);
    if (threadIdx.x % 64 == 0) to.run[part * kPartWaves + threadIdx.x / 64] = sum;
  }
  if (way == Way::kAll) return;
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    if (!(l[e] >= low && l[e] <= high) || i0 + e >= a.vocab) continue;
    const uint32_t at = atomicAdd(&listed, 1u);
    if (at < kPartList) to.list[part * kPartList + at] = static_cast<uint64_t>(~key_of(l[e])) << 32 | (i0 + e);
  }
  __syncthreads();
  if (threadIdx.x == 0) to.listed[part] = listed;
}

// The end of a split row; false: it is left to the code for one workgroup.
template <class S>
__device__ __forceinline__ bool draw_split(Lds& s, const Draw& a, uint32_t b, uint64_t* work) {
  const Split from(work, b, a.vocab);
  const uint64_t best = from.largest();
  const float max = logit_of(static_cast<uint32_t>(best >> 32));
  const Asked asked(a, b);
  const Way way = way_of(a, b, asked, max);
  if (way == Way::kOther) return false;
  if (way == Way::kLargest) {
    draw_largest(a, b, max, 0xFFFFFFFFu - static_cast<uint32_t>(best));
    return true;
  }
  const Weigh weigh{static_cast<double>(max), 1.0 / static_cast<double>(temperature_of(a, b)), (LdsTable)s.table};
  Cut cut{0, a.vocab, 0};
  const uint32_t lane = threadIdx.x % 64;
  uint32_t n = 0;
  if (way != Way::kAll) {
    const uint32_t mine = lane < from.parts ? static_cast<uint32_t>(from.listed[lane]) : 0;
    const uint32_t upto = static_cast<uint32_t>(wave_upto(mine));
    n = __builtin_amdgcn_readlane(upto, 63);
    if (__any(mine > kPartList) || n > kList) return false;
    for (uint32_t part = threadIdx.x / 64; part < from.parts; part += kWaves) {
      const uint32_t count = __shfl(mine, static_cast<int>(part), 64), to = __shfl(upto, static_cast<int>(part), 64) - count;
      for (uint32_t i = lane; i < count; i += 64) s.list[to + i] = from.list[part * kPartList + i];
    }
    __syncthreads();
    if (way == Way::kCount) {
      draw_listed(s, a, b, n, weigh, asked);
      return true;
    }
    sort_list(s, n);
    const uint32_t kept = cut_list(s, n, weigh, n, from.sums[0], from.sums[1], true, asked.parts, 0);
    n = kept;
    const uint64_t last = s.list[kept - 1];
    cut.key = ~static_cast<uint32_t>(last >> 32);
    cut.last = static_cast<uint32_t>(last);
  }
  const uint32_t runs = (a.vocab + kRun - 1) / kRun;
  if (threadIdx.x < runs) s.run_weight[threadIdx.x] = from.run[threadIdx.x];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t w = s.list_weight[i];
    if (w >= asked.least)
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.run_weight[static_cast<uint32_t>(s.list[i]) / kRun]), static_cast<unsigned long long>(w));
  }
  __syncthreads();
  draw_from_runs<S>(s, a, b, row_of<S>(a, b), weigh, asked, cut);
  return true;
}

template <class S, bool kSplit>
__global__ void __launch_bounds__(kThreads) draw_kernel(const Draw a, uint64_t* work) {
  typedef typename S::storage T;
  __shared__ Lds s;
  const uint32_t b = blockIdx.x, vocab = a.vocab;
  const T* row = row_of<S>(a, b);
  for (uint32_t i = threadIdx.x; i < kSteps; i += kThreads) s.table[i] = exp2(44.0 + static_cast<double>(i) / kSteps);
  if constexpr (kSplit) {
    __syncthreads();
    if (draw_split<S>(s, a, b, work)) return;  // all of the workgroup
  }

  // the largest logit and its lowest index
  float mine = -INFINITY;
  uint32_t at = 0xFFFFFFFFu;
  walk<S, 8>(row, vocab, [&](uint32_t i, const float(&l)[8]) {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      at = l[e] > mine ? i + e : at;
      mine = l[e] > mine ? l[e] : mine;
    }
  });
  uint64_t best = static_cast<uint64_t>(key_of(mine)) << 32 | (0xFFFFFFFFu - at);
  s.thread_max[threadIdx.x] = key_of(mine);
#pragma unroll
  for (int m = 32; m > 0; m /= 2) {
    const uint64_t other = __shfl_xor(best, m, 64);
    best = other > best ? other : best;
  }
  if (threadIdx.x % 64 == 0) s.part_weight[threadIdx.x / 64] = best;
  __syncthreads();
  for (uint32_t i = 0; i < kWaves; ++i) best = s.part_weight[i] > best ? s.part_weight[i] : best;
  __syncthreads();
  const uint32_t top = static_cast<uint32_t>(best >> 32), first = 0xFFFFFFFFu - static_cast<uint32_t>(best);
  const float max = logit_of(top), temperature = temperature_of(a, b);
  if (max == -INFINITY || !(temperature > 0.0f)) {
    draw_largest(a, b, max, first);
    return;
  }
  const Weigh weigh{static_cast<double>(max), 1.0 / static_cast<double>(temperature), (LdsTable)s.table};
  const Asked asked(a, b);
  const int32_t k = asked.k;
  const bool by_count = asked.by_count, by_weight = asked.by_weight;
  const uint32_t parts = asked.parts;
  const uint64_t least = asked.least;

  if (by_count && k <= kMostK) {
    // the upper half of the key of the k-th largest of the threads' maxima: one wave counts, 16 in each lane
    if (threadIdx.x < 64) {
      uint32_t m[kThreads / 64], least_max = top;
#pragma unroll
      for (uint32_t i = 0; i < kThreads / 64; ++i) {
        m[i] = s.thread_max[i * 64 + threadIdx.x];
        least_max = min(least_max, m[i]);
      }
#pragma unroll
      for (int i = 32; i > 0; i /= 2) least_max = min(least_max, static_cast<uint32_t>(__shfl_xor(static_cast<int>(least_max), i, 64)));
      const uint32_t differ = top ^ least_max;  // bits above its first are the same in all
      uint32_t bit = differ == 0 ? 0 : 0x80000000u >> __clz(differ), bound = bit == 0 ? top : top & ~(2 * bit - 1);
      for (; bit > 0x8000u; bit /= 2) {
        uint32_t count = 0;
#pragma unroll
        for (uint32_t i = 0; i < kThreads / 64; ++i) count += __popcll(__ballot(m[i] >= (bound | bit)));
        if (count >= static_cast<uint32_t>(k)) bound |= bit;
      }
      if (threadIdx.x == 0) s.bound[0] = bound;
    }
    __syncthreads();
    // (a key below that of -inf takes everything in)
    if (fill_list<S>(s, row, vocab, s.bound[0] > key_of(-INFINITY) ? logit_of(s.bound[0]) : -INFINITY, INFINITY)) {
      draw_listed(s, a, b, s.listed, weigh, asked);
      return;
    }
  }

  Cut cut{0, vocab, 0};  // keeps everything
  bool binned = false;
  int code_top = 0;
  uint32_t bins = 0;
  if constexpr (sizeof(T) == 2) {
    code_top = code_of(max);
    const int code_low = code_of(static_cast<float>(weigh.max - 32.0 * static_cast<double>(temperature)));
    bins = static_cast<uint32_t>(code_top - code_low) + 1;
    __syncthreads();  // the list is read
    if (bins <= kBins && top < 0xFF7F0000u) {  // (the largest bf16 may stand for +inf)
      binned = cut_by_value<kSplit>(s, row, vocab, weigh, code_top, bins, by_count ? static_cast<uint32_t>(k) : 0u, by_weight, parts, cut);
      if (!binned) cut = Cut{0, vocab, 0};
    }
  }
  const bool counted = !binned && by_count && find_cut<S, kSplit>(s, row, vocab, weigh, top, false, static_cast<uint64_t>(k), cut);
  if (by_weight && counted) {
    const uint64_t need = share(cut.weight, parts);
    find_cut<S, kSplit>(s, row, vocab, weigh, top, true, need == 0 ? 1 : need, cut);
  } else if (!binned && by_weight) {  // of all tokens that weigh anything: there are no more than k
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kRanges; i += kThreads) s.range[i] = 0;
    __syncthreads();
    walk<S, 2>(row, vocab, [&](uint32_t, const float(&l)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        int n;
        const uint64_t w = weigh(l[e], n);
        if (w > 0) atomicAdd(reinterpret_cast<unsigned long long*>(&s.range[-n / 16]), static_cast<unsigned long long>(w));
      }
    });
    __syncthreads();
    constexpr uint32_t kEach = (kRanges + kThreads - 1) / kThreads;
    uint64_t w[kEach], sum = 0, before, total, x, y;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
      const uint32_t i = threadIdx.x * kEach + j;
      w[j] = i < kRanges ? s.range[i] : 0;
      sum += w[j];
    }
    block_before(s, sum, 0, before, x, total, y);
    uint64_t need = share(total, parts);
    if (need == 0) need = 1;
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) {
      if (before < need && before + w[j] >= need) {  // one range of all
        s.found = threadIdx.x * kEach + j;
        s.before_weight = before;
      }
      before += w[j];
    }
    __syncthreads();
    const int32_t found = static_cast<int32_t>(s.found);
    const uint64_t above = s.before_weight;
    // the keys of that range lie between the last ones that this range and the one above it do not reach
    if (threadIdx.x < 128) {
      const uint32_t key = range_edge(weigh, top, threadIdx.x < 64 ? found : found - 1);
      if (threadIdx.x % 64 == 0) s.bound[threadIdx.x / 64] = key;
    }
    __syncthreads();
    if (fill_list<S>(s, row, vocab, logit_of(s.bound[0] + 1), logit_of(s.bound[1]))) {
      const uint32_t n = s.listed;
      sort_list(s, n);
      const uint32_t kept = cut_list(s, n, weigh, n, above, total, true, parts, 0);
      const uint64_t last = s.list[kept - 1];
      cut.key = ~static_cast<uint32_t>(last >> 32);
      cut.last = static_cast<uint32_t>(last);
    } else {
      find_cut<S, kSplit>(s, row, vocab, weigh, top, true, need, cut);
    }
  }

  __syncthreads();  // the list is read
  // the kept weight of each run of 512 tokens
  if (binned) {
    // (without a cut all bins are kept, whatever the index)
    const uint32_t cut_bin = cut.key == 0 ? bins - 1 : static_cast<uint32_t>(code_top - code_of(logit_of(cut.key)));
    if constexpr (sizeof(T) == 2) walk<S, 4>(row, vocab, [&](uint32_t i0, const Eight<S>& x) {
      uint64_t sum = 0;
      uint32_t small = 0;
#pragma unroll
      for (uint32_t c = 0; c < 4; ++c) {
        const u16x2 two = bins_of(x.v[0][c], code_top, bins);
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          const uint32_t bin = h ? two.y : two.x;
          if (bin < cut_bin || (bin == cut_bin && i0 + 2 * c + h <= cut.last)) {
            const uint64_t w = s.bin_weight[bin];  // (the bin of small values weighs nothing here)
            sum += w >= least ? w : 0;
            small |= static_cast<int>(bin) == code_top ? 1u << (2 * c + h) : 0u;
          }
        }
      }
      if (small) {
        float l[8];
        unpack_eight<S>(x, l);
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
          const uint64_t w = small >> e & 1 ? weigh(l[e]) : 0;
          sum += w >= least ? w : 0;
        }
      }
      const uint64_t all = wave_sum(sum);
      if (threadIdx.x % 64 == 0) s.run_weight[i0 / kRun] = all;
    });
  } else {
    walk<S, 2>(row, vocab, [&](uint32_t i0, const float(&l)[8]) {
      uint32_t in = 0;
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) in |= cut.keeps(key_of(l[e]), i0 + e) ? 1u << e : 0u;
      uint64_t sum = 0;
      if (__any(__popc(in) > 4)) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
          const uint64_t w = weigh(l[e]);
          sum += (in >> e & 1) && w >= least ? w : 0;
        }
      } else {  // few of the eight in any lane: those in a row of their own first
        uint32_t kept = 0;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
          if (in >> e & 1) s.kept[kept++ * kThreads + threadIdx.x] = l[e];
        for (uint32_t j = 0; __any(j < kept); ++j) {
          const uint64_t w = weigh(j < kept ? s.kept[j * kThreads + threadIdx.x] : -INFINITY);
          sum += w >= least ? w : 0;
        }
      }
      const uint64_t all = wave_sum(sum);
      if (threadIdx.x % 64 == 0) s.run_weight[i0 / kRun] = all;
    });
  }
  __syncthreads();
  draw_from_runs<S>(s, a, b, row, weigh, asked, cut);
}

}  // namespace
}  // namespace zo

namespace {

int draw_rows(const zo_draw_args* p, uint64_t* work, void* stream) {
  using namespace zo;
  const Draw a{static_cast<const char*>(p->logits), p->row_stride, p->u, p->temperature, p->top_k, p->top_p, p->min_p, p->tokens,
               p->logprobs, p->vocab};
  (void)hipGetLastError();
  hipStream_t st = static_cast<hipStream_t>(stream);
  const auto launch = [&](auto type) {
    typedef decltype(type) S;
    if (work == nullptr) {
      draw_kernel<S, false><<<dim3(p->rows), dim3(kThreads), 0, st>>>(a, nullptr);
      return;
    }
    const dim3 grid((p->vocab + kDrawPart - 1) / kDrawPart, p->rows);
    split_max_kernel<S><<<grid, dim3(kPartThreads), 0, st>>>(a, work);
    if (p->top_p != nullptr) split_ranges_kernel<S><<<grid, dim3(kPartThreads), 0, st>>>(a, work);
    split_list_kernel<S><<<grid, dim3(kPartThreads), 0, st>>>(a, work);
    draw_kernel<S, true><<<dim3(p->rows), dim3(kThreads), 0, st>>>(a, work);
  };
  if (p->dtype == ZO_F32)
    launch(F32{});
  else
    launch(BF16{});
  return launched();
}

}  // namespace

extern "C" int zo_draw(const zo_draw_args* p, void* stream) {
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = zo::check_draw(*p);
  return rc != ZO_OK || p->rows == 0 ? rc : draw_rows(p, nullptr, stream);
}

extern "C" int zo_draw_split(const zo_draw_args* p, void* work, uint64_t work_bytes, void* stream) {
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = zo::check_draw_split(*p, work, work_bytes);
  if (rc != ZO_OK || p->rows == 0) return rc;
  return draw_rows(p, zo_draw_work(p->rows, p->vocab, p->top_k != nullptr) != 0 ? static_cast<uint64_t*>(work) : nullptr, stream);
}
