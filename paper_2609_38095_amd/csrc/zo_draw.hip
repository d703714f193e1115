// The draw of a token from each row of logits, for gfx950: one workgroup for a row.
//
// Mathematics. Weights are whole numbers, w_i = round(2^44 exp((l_i - max) / T)), from fp64 exponentials;
// their sums (below 2^62 for 2^18 tokens) are exact in any order, so the token is the same whatever the
// order of the additions, and atomics may be used. Top-k, top-p and min-p each keep a prefix of the
// falling order, so what is kept is all logits above a cut and, of those equal to it, the first `ties`
// by index. The cut is found without sorting: logits map to 32-bit keys of the same order; a
// histogram of counts and weights over 2,048 equal ranges of keys tells in which range the k-th
// token, or the token at which the weight reaches top_p's share, lies; that range is divided again until
// it holds a single key (at most three times).
// The drawn token is then found in index order: weights of runs of 512 tokens, their running sums,
// and the tokens of the run that holds the drawn share.
//
// The row is read from HBM once; later passes find it in the L2 (608 KB at 152 k fp32 logits).

#include <cmath>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
constexpr uint32_t kBuckets = 2048;
constexpr uint32_t kRun = 512;                  // tokens of a run: 8 for each lane of a wave
constexpr uint32_t kRuns = (1u << 18) / kRun;   // at most
constexpr double kOne = 17592186044416.0;       // 2^44

// Order of logits as unsigned numbers; NaN as -inf, both zeros as one.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l == l ? l + 0.0f : -INFINITY);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

struct Weigh {
  double max, inv;  // 1 / temperature
  bool at_inf;      // the largest logit is +inf
  __device__ __forceinline__ uint64_t operator()(float l) const {
    if (at_inf) return l == INFINITY ? 1ull << 44 : 0ull;
    const double x = (static_cast<double>(l) - max) * inv;
    if (!(x > -31.25)) return 0;  // less than half of 2^-44 (and NaN)
    return static_cast<uint64_t>(rint(exp(x) * kOne));
  }
};

// floor(weight parts / 2^24), weight below 2^62, parts up to 2^24
__device__ __forceinline__ uint64_t share(uint64_t weight, uint32_t parts) {
  return (weight >> 24) * parts + (((weight & 0xFFFFFF) * parts) >> 24);
}

// The 8 logits of a row from index i on (-inf behind the end).
template <class S>
__device__ __forceinline__ void load8(const typename S::storage* row, uint32_t i, uint32_t vocab, float (&l)[8]) {
  if (i + 8 <= vocab) {
    if constexpr (sizeof(typename S::storage) == 2) {
      S::unpack(*reinterpret_cast<const u32x4_any*>(row + i), l);
    } else {
      float a[4], b[4];
      S::unpack(*reinterpret_cast<const u32x4_any*>(row + i), a);
      S::unpack(*reinterpret_cast<const u32x4_any*>(row + i + 4), b);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        l[e] = a[e];
        l[4 + e] = b[e];
      }
    }
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) l[e] = i + e < vocab ? S::load1(row + i + e) : -INFINITY;
  }
}

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
  for (int m = 32; m > 0; m /= 2) v += __shfl_xor(v, m, 64);
  return v;
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
  uint64_t weight[kBuckets];
  uint32_t count[kBuckets];
  uint64_t part_weight[kWaves];
  uint64_t part_count[kWaves];
  uint64_t run_weight[kRuns];
  uint32_t run_ties[kRuns];
  uint64_t before_weight, found_weight;
  uint32_t before_count, found, found_count;
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

// A cut: logits with key > key are kept, of those with key == key the first `ties` by index.
struct Cut {
  uint32_t key, ties;
  uint64_t weight;  // of all that is kept
};

// The cut at which the count reaches `most`, or (by_weight) the weight reaches `need`, whichever is
// asked for; false: the row's weights end before. Tokens of no weight do not count.
template <class S>
__device__ bool find_cut(Lds& s, const typename S::storage* row, uint32_t vocab, const Weigh& weigh, uint32_t top, bool by_weight,
                         uint64_t need, Cut& cut) {
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
    for (uint32_t i = threadIdx.x * 8; i < vocab; i += kThreads * 8) {
      float l[8];
      load8<S>(row, i, vocab, l);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = key_of(l[e]);
        if (key < lo || key > hi) continue;
        const uint64_t w = weigh(l[e]);
        if (w == 0) continue;
        const uint32_t b = (hi - key) >> shift;
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.weight[b]), static_cast<unsigned long long>(w));
        atomicAdd(&s.count[b], 1u);
      }
    }
    __syncthreads();
    uint64_t w[2], c[2], w_before, c_before, w_all, c_all;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w[j] = s.weight[2 * threadIdx.x + j];
      c[j] = s.count[2 * threadIdx.x + j];
    }
    block_before(s, w[0] + w[1], c[0] + c[1], w_before, c_before, w_all, c_all);
    if ((by_weight ? above_weight + w_all : above_count + c_all) < need) return false;
    uint64_t wb = above_weight + w_before, cb = above_count + c_before;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint64_t was = by_weight ? wb : cb, now = was + (by_weight ? w[j] : c[j]);
      if (was < need && now >= need) {  // one bucket of all
        s.found = 2 * threadIdx.x + j;
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
      cut.ties = static_cast<uint32_t>(ties);
      cut.weight = above_weight + ties * each;
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

template <class S>
__global__ void __launch_bounds__(kThreads) draw_kernel(const Draw a) {
  typedef typename S::storage T;
  __shared__ Lds s;
  const uint32_t b = blockIdx.x, vocab = a.vocab;
  const T* row = reinterpret_cast<const T*>(a.logits) + static_cast<int64_t>(b) * a.row_stride;

  // the largest logit and its lowest index
  uint64_t best = 0;
  for (uint32_t i = threadIdx.x * 8; i < vocab; i += kThreads * 8) {
    float l[8];
    load8<S>(row, i, vocab, l);
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      const uint64_t k = static_cast<uint64_t>(key_of(l[e])) << 32 | (0xFFFFFFFFu - (i + e));
      best = k > best ? k : best;
    }
  }
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
  const float max = logit_of(top), temperature = a.temperature ? a.temperature[b] : 1.0f;
  if (max == -INFINITY || !(temperature > 0.0f)) {
    if (threadIdx.x == 0) {
      a.tokens[b] = max == -INFINITY ? -1 : static_cast<int32_t>(first);
      if (a.logprobs) a.logprobs[b] = max == -INFINITY ? -INFINITY : 0.0f;
    }
    return;
  }
  const Weigh weigh{static_cast<double>(max), 1.0 / static_cast<double>(temperature), max == INFINITY};

  Cut cut{0, 0, 0};  // everything is above it
  const int32_t k = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.0f;
  bool cut_found = false;
  if (k > 0 && static_cast<uint32_t>(k) < vocab)
    cut_found = find_cut<S>(s, row, vocab, weigh, top, false, static_cast<uint64_t>(k), cut);
  if (p < 1.0f) {
    uint64_t total = cut.weight;
    if (!cut_found) {
      uint64_t sum = 0;
      for (uint32_t i = threadIdx.x * 8; i < vocab; i += kThreads * 8) {
        float l[8];
        load8<S>(row, i, vocab, l);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += weigh(l[e]);
      }
      uint64_t x, y, z;
      block_before(s, sum, 0, x, y, total, z);
    }
    const uint32_t parts = p > 0.0f ? static_cast<uint32_t>(rint(static_cast<double>(p) * 16777216.0)) : 0u;
    uint64_t need = share(total, parts);
    if (need == 0) need = 1;
    Cut by_weight;
    if (find_cut<S>(s, row, vocab, weigh, top, true, need, by_weight)) cut = by_weight;
  }
  const float mp = a.min_p ? a.min_p[b] : 0.0f;
  const uint64_t least = mp > 0.0f ? static_cast<uint64_t>(rint(static_cast<double>(mp < 1.0f ? mp : 1.0f) * kOne)) : 0ull;

  // weights above the cut and ties at it, of each run of 512 tokens
  const uint32_t runs = (vocab + kRun - 1) / kRun;
  for (uint32_t run = threadIdx.x / 64; run < runs; run += kWaves) {
    float l[8];
    load8<S>(row, run * kRun + threadIdx.x % 64 * 8, vocab, l);
    uint64_t sum = 0;
    uint32_t ties = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = key_of(l[e]);
      if (key < cut.key) continue;
      const uint64_t w = weigh(l[e]);
      if (w < least) continue;
      if (key > cut.key)
        sum += w;
      else
        ++ties;
    }
    sum = wave_sum(sum);
    ties = static_cast<uint32_t>(wave_sum(ties));
    if (threadIdx.x % 64 == 0) {
      s.run_weight[run] = sum;
      s.run_ties[run] = ties;
    }
  }
  __syncthreads();
  const uint64_t tie_weight = weigh(logit_of(cut.key));
  const uint64_t my_ties = threadIdx.x < runs ? s.run_ties[threadIdx.x] : 0;
  uint64_t w_before, t_before, w_all, t_all, x;
  block_before(s, 0, my_ties, x, t_before, w_all, t_all);
  const auto kept_ties = [&](uint64_t before, uint64_t n) { return before >= cut.ties ? 0ull : n < cut.ties - before ? n : cut.ties - before; };
  const uint64_t mine = threadIdx.x < runs ? s.run_weight[threadIdx.x] + kept_ties(t_before, my_ties) * tie_weight : 0;
  block_before(s, mine, 0, w_before, x, w_all, t_all);
  const float u = a.u[b];
  const uint32_t draw = !(u > 0.0f) ? 0u : u >= 1.0f ? 0xFFFFFFu : static_cast<uint32_t>(u * 16777216.0f);
  const uint64_t target = share(w_all, draw);
  if (w_before <= target && target < w_before + mine) {  // one run of all
    s.found = threadIdx.x;
    s.before_weight = w_before;
    s.before_count = static_cast<uint32_t>(t_before);
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;

  // the token inside the run
  const uint32_t i0 = s.found * kRun + threadIdx.x * 8;
  float l[8];
  load8<S>(row, i0, vocab, l);
  uint64_t w[8];
  uint32_t tie = 0, ties = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t key = key_of(l[e]);
    w[e] = key < cut.key ? 0 : weigh(l[e]);
    if (w[e] < least) w[e] = 0;
    if (key == cut.key && w[e] > 0) {
      tie |= 1u << e;
      ++ties;
    }
  }
  uint64_t tb = s.before_count + wave_upto(ties) - ties;
  uint64_t sum = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (tie >> e & 1) {
      if (tb >= cut.ties) w[e] = 0;
      ++tb;
    }
    sum += w[e];
  }
  uint64_t upto = s.before_weight + wave_upto(sum) - sum;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (upto <= target && target < upto + w[e]) {
      a.tokens[b] = static_cast<int32_t>(i0 + e);
      if (a.logprobs) a.logprobs[b] = static_cast<float>(log(static_cast<double>(w[e]) / static_cast<double>(w_all)));
    }
    upto += w[e];
  }
}

}  // namespace
}  // namespace zo

extern "C" int zo_draw(const zo_draw_args* p, void* stream) {
  using namespace zo;
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = check_draw(*p);
  if (rc != ZO_OK) return rc;
  if (p->rows == 0) return ZO_OK;
  const Draw a{static_cast<const char*>(p->logits), p->row_stride, p->u, p->temperature, p->top_k, p->top_p, p->min_p, p->tokens,
               p->logprobs, p->vocab};
  (void)hipGetLastError();
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p->dtype == ZO_F32)
    draw_kernel<F32><<<dim3(p->rows), dim3(kThreads), 0, st>>>(a);
  else
    draw_kernel<BF16><<<dim3(p->rows), dim3(kThreads), 0, st>>>(a);
  return launched();
}
