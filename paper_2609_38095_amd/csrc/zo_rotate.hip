// Head norms and position rotation for gfx950: forward (into tensors or into the paged cache) and
// backward.
//
// Mathematics. Row x of one head: n = x r g, r = 1 / sqrt(mean x^2 + eps); pairs of n turn by the
// position's angle. The angle 2 pi pos t is reduced in fp64 (pos t minus its nearest whole number of
// turns), so only the last step, sine and cosine of at most half a turn, is fp32.
//
// Layout. The rows of a side (queries, keys, values to put) are numbered token by token; a
// workgroup takes consecutive rows of one side, so that its gammas stay in registers and its few
// tokens' sines and cosines are computed once into LDS and used by every head. A row is held by L
// neighbouring lanes with two 16-byte vectors each, chosen so that both members of a pair are in one
// lane: at dims v and v + rotary / 2 for half pairs, anywhere for interleaved pairs. The norm
// is then a sum over L lanes by data-parallel moves, and nothing of a row passes through LDS.
// Sizes that vectors do not divide take the same code with one element for a vector.
//
// Bound by HBM: one read and one write of each row. 16,387 fp32 tokens of 64 heads of 64 take 94 us
// (5.7 TB/s), eight tokens 5 us. The gradient of 8,192 bf16 tokens of 32 + 8 heads of 128 takes 52 us (4.8 TB/s)
// and 4.5 for the gammas' sum: both sides have 512 workgroups, so the keys' end after a quarter of the queries' walk.

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "zo_checks.h"
#include "zo_lanes.h"

namespace zo {
namespace {

constexpr uint32_t kThreads = 256;

struct Side {
  const char* x;   // forward: input; backward: forward's input (with a gamma)
  const char* dy;  // backward: incoming gradient
  char* y;         // forward: output; backward: dx
  const char* gamma;
  int64_t x_token, x_head, dy_token, dy_head, y_token, y_head;  // strides in elements
  uint32_t heads;
  float inv_heads;
  uint32_t rows;
  uint32_t first_block;  // of the grid
  uint32_t rotary;
  uint32_t put;  // the output rows' places are in the cache
};

struct Rotation {
  Side side[3];
  const int32_t* positions;
  const int32_t* seqs;
  const int32_t* places;  // of the tokens in their sequences, NULL: the positions
  const int32_t* ids;  // page table
  int64_t table_stride, page_stride, cache_token;
  uint32_t table_seqs, table_width, pages, page_tokens;
  uint32_t dim;
  float eps, magnitude;
  uint32_t slots;    // tokens that a workgroup's rows may touch (the size of its LDS tables)
  float* partial;    // backward: gamma gradients of each workgroup
  double turns[ZO_DIM_MAX / 2];
};

// One lane's share of a row. kVec elements make a vector; the lane holds kPairs times two vectors, at dims a(n) and
// b(n), neighbouring lanes neighbouring vectors, so that each access of a wave covers whole lines (lanes with two
// adjacent vectors each left every access with gaps: 16,387 fp32 tokens of 64 heads of 64, interleaved, took
// 180 us with streaming stores). kInside: pairs lie inside a vector (2 i, 2 i + 1), else across the two.
template <class S, int kVec, int kPairs, bool kInside>
struct Share {
  uint32_t a[kPairs], b[kPairs], pair[kPairs];  // pair: of the angles, for a and b together or (inside) for a
  bool in_a[kPairs], in_b[kPairs], turn_a[kPairs], turn_b[kPairs];

  __device__ void place(uint32_t lane, uint32_t lanes, uint32_t dim, uint32_t rotary, bool interleaved) {
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
      const uint32_t j = lane + n * lanes, turning = rotary / (2 * kVec);
      if (kInside) {
        a[n] = kVec * j;
        b[n] = dim / 2 + a[n];
        pair[n] = a[n] / 2;
        in_a[n] = a[n] < dim / 2;
        turn_a[n] = a[n] < rotary;
        turn_b[n] = b[n] < rotary;
      } else if (kVec == 1 && interleaved) {
        a[n] = 2 * j;
        b[n] = a[n] + 1;
        pair[n] = j;
        in_a[n] = a[n] < dim;
        turn_a[n] = turn_b[n] = j < turning;
      } else if (j < turning) {
        a[n] = pair[n] = kVec * j;
        b[n] = a[n] + rotary / 2;
        in_a[n] = true;
        turn_a[n] = turn_b[n] = true;
      } else {  // the rest of the row, in two halves (the first one longer by an element of an odd rest)
        const uint32_t half = (dim - rotary + 1) / 2;
        a[n] = rotary + kVec * (j - turning);
        b[n] = a[n] + half;
        pair[n] = 0;
        in_a[n] = a[n] < rotary + half;
        turn_a[n] = turn_b[n] = false;
      }
      in_b[n] = in_a[n] && b[n] < dim;
    }
  }
};

template <class S, int kVec>
struct Raw {
  u32x4 v;
};
template <class S>
struct Raw<S, 1> {
  typename S::storage v;
};

// Streaming accesses (nothing is used twice) where the lanes of a row cover whole lines at a time, kWhole: 8 or more of
// them. 8,192 packed bf16 tokens of 32 + 8 heads of 128, backward: 90 us with ordinary accesses, 62 with streaming ones;
// 16,384 tokens of 64 heads of 64, whose accesses cover half lines: 58 and 66.
template <class S, int kVec, bool kWhole>
__device__ __forceinline__ Raw<S, kVec> ld(const char* base, int64_t elem) {
  const typename S::storage* p = reinterpret_cast<const typename S::storage*>(base) + elem;
  if constexpr (kVec == 1)
    return {*p};
  else
    return {kWhole ? ld_stream(p) : *reinterpret_cast<const u32x4_any*>(p)};
}

template <class S, int kVec>
__device__ __forceinline__ void widen(const Raw<S, kVec>& r, float (&f)[kVec]) {
  if constexpr (kVec == 1)
    f[0] = S::load1(&r.v);
  else
    S::unpack(r.v, f);
}

template <class S, int kVec, bool kWhole>
__device__ __forceinline__ void st(char* base, int64_t elem, const float (&f)[kVec]) {
  typename S::storage* p = reinterpret_cast<typename S::storage*>(base) + elem;
  if constexpr (kVec == 1)
    S::store1(p, f[0]);
  else if constexpr (kWhole)
    st_stream(p, S::pack(f));
  else
    *reinterpret_cast<u32x4_any*>(p) = S::pack(f);
}

template <int kVec, bool kBack>
__device__ __forceinline__ void turn_inside(float (&v)[kVec], const float2* cs) {
#pragma unroll
  for (int e = 0; e < kVec / 2; ++e) {
    const float2 t = cs[e];
    const float s = kBack ? -t.y : t.y, p = v[2 * e], q = v[2 * e + 1];
    v[2 * e] = p * t.x - q * s;
    v[2 * e + 1] = p * s + q * t.x;
  }
}

// A share's two vectors turned by the angles cs of a token (cosine and sine of each pair); kBack: by the opposite ones.
template <int kVec, bool kInside, bool kBack, class Sh>
__device__ __forceinline__ void turn_share(const Sh& sh, int n, float (&a)[kVec], float (&b)[kVec], const float2* cs) {
  if constexpr (kInside) {
    if (sh.turn_a[n]) turn_inside<kVec, kBack>(a, cs + sh.pair[n]);
    if (sh.turn_b[n]) turn_inside<kVec, kBack>(b, cs + sh.b[n] / 2);
  } else if (sh.turn_a[n]) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float2 t = cs[sh.pair[n] + e];
      const float s = kBack ? -t.y : t.y, p = a[e], q = b[e];
      a[e] = p * t.x - q * s;
      b[e] = p * s + q * t.x;
    }
  }
}

// Where rows of a token go: the element offset of its first head, or -1: nowhere.
__device__ __forceinline__ int64_t place_of(const Rotation& r, const Side& sd, uint32_t token, int32_t pos) {
  if (!sd.put) return static_cast<int64_t>(token) * sd.y_token;
  const uint32_t seq = r.seqs ? static_cast<uint32_t>(r.seqs[token]) : token;
  if (r.places && pos >= 0) pos = r.places[token];  // padding has no place
  if (pos < 0 || seq >= r.table_seqs) return -1;
  const uint32_t slot = static_cast<uint32_t>(pos) / r.page_tokens;
  if (slot >= r.table_width) return -1;
  const int32_t id = r.ids[static_cast<int64_t>(seq) * r.table_stride + slot];
  if (static_cast<uint32_t>(id) >= r.pages) return -1;
  return id * r.page_stride + static_cast<int64_t>(static_cast<uint32_t>(pos) - slot * r.page_tokens) * r.cache_token;
}

// Cosines and sines of the workgroup's tokens, its tokens' places and whether they are padding.
struct Tables {
  float2* cs;      // [slots][rotary / 2]
  int64_t* place;  // [slots]
  int32_t* live;   // [slots]
};

__device__ __forceinline__ Tables tables(const Rotation& r, char* lds, uint32_t half) {
  Tables t;
  t.cs = reinterpret_cast<float2*>(lds);
  t.place = reinterpret_cast<int64_t*>(lds + static_cast<size_t>(r.slots) * half * sizeof(float2));
  t.live = reinterpret_cast<int32_t*>(t.place + r.slots);
  return t;
}

__device__ __forceinline__ void fill_tables(const Rotation& r, const Side& sd, const Tables& t, uint32_t token0, uint32_t count) {
  for (uint32_t i = threadIdx.x; i < count; i += kThreads) {
    const int32_t pos = r.positions[token0 + i];
    t.live[i] = pos >= 0;
    t.place[i] = place_of(r, sd, token0 + i, pos);
  }
  const uint32_t half = sd.rotary / 2;
  for (uint32_t i = threadIdx.x; i < count * half; i += kThreads) {
    const uint32_t k = i / half, p = i - k * half;
    const double turns = static_cast<double>(r.positions[token0 + k]) * r.turns[p];
    const float part = static_cast<float>(turns - rint(turns));
    float s, c;
    sincospif(2.0f * part, &s, &c);
    t.cs[i] = make_float2(c * r.magnitude, s * r.magnitude);
  }
}

__device__ __forceinline__ uint32_t side_of(const Rotation& r, uint32_t block) {
  return block >= r.side[2].first_block ? 2 : block >= r.side[1].first_block ? 1 : 0;
}

// kRows rows for each group of L lanes: all of them are loaded before the angles are computed.
template <class S, int kVec, int L, int kPairs, bool kInside, int kRows>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const Rotation r, const uint32_t interleaved) {
  extern __shared__ __align__(16) char lds[];
  constexpr uint32_t kPerPass = kThreads / L, kBlockRows = kPerPass * kRows;
  const Side& sd = r.side[side_of(r, blockIdx.x)];
  const uint32_t row0 = (blockIdx.x - sd.first_block) * kBlockRows;
  const uint32_t rows = min(kBlockRows, sd.rows - row0);
  const uint32_t token0 = row0 / sd.heads, skip = row0 - token0 * sd.heads;
  const uint32_t count = (skip + rows - 1) / sd.heads + 1;

  Share<S, kVec, kPairs, kInside> sh;
  sh.place(threadIdx.x % L, L, r.dim, sd.rotary, interleaved);
  Raw<S, kVec> ra[kRows][kPairs] = {}, rb[kRows][kPairs] = {};
  uint32_t tok[kRows], head[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const uint32_t row = i * kPerPass + threadIdx.x / L;
    // (row + skip) / heads: row + skip < 2^17, so the product is off by less than the half's share
    tok[i] = static_cast<uint32_t>((static_cast<float>(row + skip) + 0.5f) * sd.inv_heads);
    head[i] = row + skip - tok[i] * sd.heads;
    if (row >= rows) continue;
    const int64_t at = static_cast<int64_t>(token0 + tok[i]) * sd.x_token + head[i] * sd.x_head;
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
      if (sh.in_a[n]) ra[i][n] = ld<S, kVec, (L >= 8)>(sd.x, at + sh.a[n]);
      if (sh.in_b[n]) rb[i][n] = ld<S, kVec, (L >= 8)>(sd.x, at + sh.b[n]);
    }
  }
  float ga[kPairs][kVec], gb[kPairs][kVec];
  if (sd.gamma) {
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
      Raw<S, kVec> va = {}, vb = {};
      if (sh.in_a[n]) va = ld<S, kVec, false>(sd.gamma, sh.a[n]);
      if (sh.in_b[n]) vb = ld<S, kVec, false>(sd.gamma, sh.b[n]);
      widen<S, kVec>(va, ga[n]);
      widen<S, kVec>(vb, gb[n]);
    }
  }
  const uint32_t half = sd.rotary / 2;
  const Tables t = tables(r, lds, half);
  fill_tables(r, sd, t, token0, count);
  __syncthreads();

  const float inv_dim = 1.0f / static_cast<float>(r.dim);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    float a[kPairs][kVec], b[kPairs][kVec];
    float ss = 0.0f;
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
      widen<S, kVec>(ra[i][n], a[n]);
      widen<S, kVec>(rb[i][n], b[n]);
    }
    if (sd.gamma) {
#pragma unroll
      for (int n = 0; n < kPairs; ++n)
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss += a[n][e] * a[n][e] + b[n][e] * b[n][e];
      const float s = 1.0f / sqrtf(sum_lanes<L>(ss) * inv_dim + r.eps);
#pragma unroll
      for (int n = 0; n < kPairs; ++n)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          a[n][e] *= s * ga[n][e];
          b[n][e] *= s * gb[n][e];
        }
    }
    if (i * kPerPass + threadIdx.x / L >= rows) continue;
    const int64_t place = t.place[tok[i]];
    if (place < 0) continue;
    const bool live = t.live[tok[i]] != 0;
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
      turn_share<kVec, kInside, false>(sh, n, a[n], b[n], t.cs + tok[i] * half);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        a[n][e] = live ? a[n][e] : 0.0f;
        b[n][e] = live ? b[n][e] : 0.0f;
      }
      const int64_t at = place + head[i] * sd.y_head;
      if (sh.in_a[n]) st<S, kVec, (L >= 8)>(sd.y, at + sh.a[n], a[n]);
      if (sh.in_b[n]) st<S, kVec, (L >= 8)>(sd.y, at + sh.b[n], b[n]);
    }
  }
}

// Backward: each workgroup walks over blocks of rows and keeps its share of the gamma gradient in
// registers; at its end the shares are added over the lanes of a wave and over the waves, and written
// to `partial` in the grid's order, which gamma_kernel adds. No atomics: the order is fixed.
template <class S, int kVec, int L, int kPairs, bool kInside>
__global__ void __launch_bounds__(kThreads) rotate_back_kernel(const Rotation r, const uint32_t interleaved, const uint32_t blocks0) {
  extern __shared__ __align__(16) char lds[];
  constexpr int kRows = 2;
  constexpr uint32_t kPerPass = kThreads / L, kBlockRows = kPerPass * kRows;
  const Side& sd = r.side[blockIdx.x >= blocks0 ? 1 : 0];
  const uint32_t block = blockIdx.x - sd.first_block;
  const uint32_t blocks = (blockIdx.x >= blocks0 ? gridDim.x : blocks0) - sd.first_block;
  const uint32_t half = sd.rotary / 2;
  const Tables t = tables(r, lds, half);
  const float inv_dim = 1.0f / static_cast<float>(r.dim);

  Share<S, kVec, kPairs, kInside> sh;
  sh.place(threadIdx.x % L, L, r.dim, sd.rotary, interleaved);
  float ga[kPairs][kVec], gb[kPairs][kVec], dga[kPairs][kVec], dgb[kPairs][kVec];
#pragma unroll
  for (int n = 0; n < kPairs; ++n) {
    Raw<S, kVec> va = {}, vb = {};
    if (sd.gamma && sh.in_a[n]) va = ld<S, kVec, false>(sd.gamma, sh.a[n]);
    if (sd.gamma && sh.in_b[n]) vb = ld<S, kVec, false>(sd.gamma, sh.b[n]);
    widen<S, kVec>(va, ga[n]);
    widen<S, kVec>(vb, gb[n]);
#pragma unroll
    for (int e = 0; e < kVec; ++e) dga[n][e] = dgb[n][e] = 0.0f;
  }

  const uint32_t chunks = (sd.rows - 1) / kBlockRows + 1;
  for (uint32_t c = block; c < chunks; c += blocks) {
    const uint32_t row0 = c * kBlockRows;
    const uint32_t rows = min(kBlockRows, sd.rows - row0);
    const uint32_t token0 = row0 / sd.heads, skip = row0 - token0 * sd.heads;
    const uint32_t count = (skip + rows - 1) / sd.heads + 1;
    Raw<S, kVec> xa[kRows][kPairs] = {}, xb[kRows][kPairs] = {}, ya[kRows][kPairs] = {}, yb[kRows][kPairs] = {};
    uint32_t tok[kRows], head[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const uint32_t row = i * kPerPass + threadIdx.x / L;
      tok[i] = static_cast<uint32_t>((static_cast<float>(row + skip) + 0.5f) * sd.inv_heads);
      head[i] = row + skip - tok[i] * sd.heads;
      if (row >= rows) continue;
      const int64_t at = static_cast<int64_t>(token0 + tok[i]) * sd.x_token + head[i] * sd.x_head;
      const int64_t dat = static_cast<int64_t>(token0 + tok[i]) * sd.dy_token + head[i] * sd.dy_head;
#pragma unroll
      for (int n = 0; n < kPairs; ++n) {
        if (sh.in_a[n]) ya[i][n] = ld<S, kVec, (L >= 8)>(sd.dy, dat + sh.a[n]);
        if (sh.in_b[n]) yb[i][n] = ld<S, kVec, (L >= 8)>(sd.dy, dat + sh.b[n]);
        if (sd.gamma && sh.in_a[n]) xa[i][n] = ld<S, kVec, (L >= 8)>(sd.x, at + sh.a[n]);
        if (sd.gamma && sh.in_b[n]) xb[i][n] = ld<S, kVec, (L >= 8)>(sd.x, at + sh.b[n]);
      }
    }
    __syncthreads();  // the tables of the rows before are read
    fill_tables(r, sd, t, token0, count);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const bool mine = i * kPerPass + threadIdx.x / L < rows;
      const uint32_t k = mine ? tok[i] : 0;
      const bool live = mine && t.live[k] != 0;
      float da[kPairs][kVec], db[kPairs][kVec];
#pragma unroll
      for (int n = 0; n < kPairs; ++n) {
        widen<S, kVec>(ya[i][n], da[n]);
        widen<S, kVec>(yb[i][n], db[n]);
        turn_share<kVec, kInside, true>(sh, n, da[n], db[n], t.cs + k * half);
      }
      if (sd.gamma) {
        float a[kPairs][kVec], b[kPairs][kVec];
        float ss = 0.0f, dot = 0.0f;
#pragma unroll
        for (int n = 0; n < kPairs; ++n) {
          widen<S, kVec>(xa[i][n], a[n]);
          widen<S, kVec>(xb[i][n], b[n]);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            ss += a[n][e] * a[n][e] + b[n][e] * b[n][e];
            dot += da[n][e] * ga[n][e] * a[n][e] + db[n][e] * gb[n][e] * b[n][e];
          }
        }
        const float s = 1.0f / sqrtf(sum_lanes<L>(ss) * inv_dim + r.eps);
        const float m = sum_lanes<L>(dot) * inv_dim * s * s;
#pragma unroll
        for (int n = 0; n < kPairs; ++n)
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (live) {
              dga[n][e] += da[n][e] * (a[n][e] * s);
              dgb[n][e] += db[n][e] * (b[n][e] * s);
            }
            da[n][e] = s * (da[n][e] * ga[n][e] - a[n][e] * m);
            db[n][e] = s * (db[n][e] * gb[n][e] - b[n][e] * m);
          }
      }
      if (!mine) continue;
      const int64_t at = static_cast<int64_t>(token0 + k) * sd.y_token + head[i] * sd.y_head;
#pragma unroll
      for (int n = 0; n < kPairs; ++n) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          da[n][e] = live ? da[n][e] : 0.0f;
          db[n][e] = live ? db[n][e] : 0.0f;
        }
        if (sh.in_a[n]) st<S, kVec, (L >= 8)>(sd.y, at + sh.a[n], da[n]);
        if (sh.in_b[n]) st<S, kVec, (L >= 8)>(sd.y, at + sh.b[n], db[n]);
      }
    }
  }
  if (!sd.gamma) return;
  // rows of one wave that end in the same dims: L, 2 L, .. lanes apart
  float* wave_sum = reinterpret_cast<float*>(lds);  // [4][dim]
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kPairs; ++n)
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
#pragma unroll
      for (int m = L; m < 64; m *= 2) {
        dga[n][e] += __shfl_xor(dga[n][e], m, 64);
        dgb[n][e] += __shfl_xor(dgb[n][e], m, 64);
      }
      if (threadIdx.x % 64 < L) {
        if (sh.in_a[n]) wave_sum[threadIdx.x / 64 * r.dim + sh.a[n] + e] = dga[n][e];
        if (sh.in_b[n]) wave_sum[threadIdx.x / 64 * r.dim + sh.b[n] + e] = dgb[n][e];
      }
    }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < r.dim; d += kThreads) {
    float sum = 0.0f;
    for (uint32_t w = 0; w < kThreads / 64; ++w) sum += wave_sum[w * r.dim + d];
    r.partial[static_cast<size_t>(blockIdx.x) * r.dim + d] = sum;
  }
}

// dgamma[d] = sum of the workgroups' shares: 16 dims by 64 slices of workgroups each.
__global__ void __launch_bounds__(1024) gamma_kernel(const float* partial, uint32_t blocks0, uint32_t blocks1, uint32_t dim, float* out0,
                                                     float* out1) {
  __shared__ float sums[64][17];
  const uint32_t side = blockIdx.y;
  float* out = side ? out1 : out0;
  if (out == nullptr) return;
  const uint32_t first = side ? blocks0 : 0, count = side ? blocks1 : blocks0;
  const uint32_t col = threadIdx.x % 16, slice = threadIdx.x / 16, d = blockIdx.x * 16 + col;
  float sum = 0.0f;
  if (d < dim)
    for (uint32_t b = slice; b < count; b += 64) sum += partial[static_cast<size_t>(first + b) * dim + d];
  sums[slice][col] = sum;
  __syncthreads();
  for (uint32_t m = 32; m > 0; m /= 2) {
    if (slice < m) sums[slice][col] += sums[slice + m][col];
    __syncthreads();
  }
  if (slice == 0 && d < dim) out[d] = sums[0][col];
}

// ---- launches

struct Shape {
  uint32_t lanes;   // of a row
  bool vectors;
};

// Vectors need every boundary of the row (its end, the rotated part and its middle) at a vector's.
template <class S>
Shape shape_of(uint32_t dim, uint32_t rotary) {
  constexpr uint32_t kPair = 2 * S::kVecElems;
  if (dim % kPair != 0 || rotary % kPair != 0) return {64, false};
  const uint32_t lanes = dim / kPair;
  return {lanes <= 4 ? 4u : lanes <= 8 ? 8u : lanes <= 16 ? 16u : 32u, true};
}

uint32_t slots_of(const Rotation& r, uint32_t block_rows, uint32_t sides) {
  uint32_t slots = 1;
  for (uint32_t i = 0; i < sides; ++i)
    if (r.side[i].rows > 0) slots = std::max(slots, (block_rows - 1) / r.side[i].heads + 2);
  return slots;
}

size_t lds_bytes(const Rotation& r, uint32_t rotary) {
  return static_cast<size_t>(r.slots) * (rotary / 2 * sizeof(float2) + sizeof(int64_t) + sizeof(int32_t));
}

template <class S, int kVec, int L, int kPairs, bool kInside, int kRows>
int launch_rows(Rotation& r, uint32_t rotary, uint32_t interleaved, hipStream_t st) {
  constexpr uint32_t kBlockRows = kThreads / L * kRows;
  uint64_t all = 0;
  for (const Side& sd : r.side) all += (sd.rows + uint64_t{kBlockRows} - 1) / kBlockRows;
  if (all >= (1u << 24)) return ZO_ERR_ARG;  // 2^32 threads at most in a launch
  uint32_t blocks = 0;
  for (Side& sd : r.side) {  // one without rows begins where the next does: no block finds it
    sd.first_block = blocks;
    blocks += (sd.rows + kBlockRows - 1) / kBlockRows;
  }
  r.slots = slots_of(r, kBlockRows, 3);
  rotate_kernel<S, kVec, L, kPairs, kInside, kRows><<<dim3(blocks), dim3(kThreads), lds_bytes(r, rotary), st>>>(r, interleaved);
  return launched();
}

// Four rows for each lane group once that still gives every CU two workgroups; else one, so that a
// few tokens spread over as many CUs as they can. One too where a workgroup's rows would span so many
// tokens (few heads) that their angles take more than 32 KiB of LDS.
template <class S, int kVec, int L, int kPairs, bool kInside>
int launch_forward(Rotation& r, uint32_t rotary, uint32_t interleaved, hipStream_t st) {
  uint64_t rows = 0;
  for (const Side& sd : r.side) rows += sd.rows;
  r.slots = slots_of(r, kThreads / L * 4, 3);
  if (rows >= 512ull * 4 * (kThreads / L) && lds_bytes(r, rotary) <= 32768) return launch_rows<S, kVec, L, kPairs, kInside, 4>(r, rotary, interleaved, st);
  return launch_rows<S, kVec, L, kPairs, kInside, 1>(r, rotary, interleaved, st);
}

template <class S, int kVec, int L, int kPairs, bool kInside>
int launch_back(Rotation& r, uint32_t rotary, uint32_t interleaved, const zo_rotate_back& b, hipStream_t st) {
  const uint32_t blocks0 = back_blocks(b.a.tokens, b.a.q_heads), blocks1 = back_blocks(b.a.tokens, b.a.k_heads);
  r.side[0].first_block = 0;
  r.side[1].first_block = blocks0;
  r.slots = slots_of(r, kThreads / L * 2, 2);
  const size_t lds = std::max(lds_bytes(r, rotary), 4 * r.dim * sizeof(float));
  if (blocks0 + blocks1 > 0) {
    rotate_back_kernel<S, kVec, L, kPairs, kInside><<<dim3(blocks0 + blocks1), dim3(kThreads), lds, st>>>(r, interleaved, blocks0);
    const int rc = launched();
    if (rc != ZO_OK) return rc;
  }
  float* out0 = b.a.q_gamma ? b.dq_gamma : nullptr;
  float* out1 = b.a.k_gamma ? b.dk_gamma : nullptr;
  if (out0 == nullptr && out1 == nullptr) return ZO_OK;
  gamma_kernel<<<dim3((r.dim + 15) / 16, 2), dim3(1024), 0, st>>>(r.partial, blocks0, blocks1, r.dim, out0, out1);
  return launched();
}

// The launcher `go` with the kernel's constants for these sizes: go(vec, lanes, pairs, inside).
template <class S, class Go>
int dispatch(uint32_t dim, uint32_t rotary, bool interleaved, Go go) {
  const Shape s = shape_of<S>(dim, rotary);
  using std::integral_constant;
  typedef integral_constant<int, S::kVecElems> Vec;
  typedef integral_constant<int, 1> One;
  if (!s.vectors) return go(One{}, integral_constant<int, 64>{}, integral_constant<int, 2>{}, std::false_type{});
  const auto lanes = [&](auto inside) {
    switch (s.lanes) {
      case 4: return go(Vec{}, integral_constant<int, 4>{}, One{}, inside);
      case 8: return go(Vec{}, integral_constant<int, 8>{}, One{}, inside);
      case 16: return go(Vec{}, integral_constant<int, 16>{}, One{}, inside);
      default:
        if constexpr (sizeof(typename S::storage) == 4) return go(Vec{}, integral_constant<int, 32>{}, One{}, inside);
        return static_cast<int>(ZO_ERR_ARG);
    }
  };
  return interleaved ? lanes(std::true_type{}) : lanes(std::false_type{});
}

Rotation rotation_of(const zo_rotate& a) {
  Rotation r;
  std::memset(&r, 0, sizeof r);
  r.positions = a.positions;
  r.dim = a.dim;
  r.eps = a.norm_eps;
  r.magnitude = a.magnitude;
  if (a.rotary > 0) std::memcpy(r.turns, a.turns, a.rotary / 2 * sizeof(double));
  return r;
}

Side side_rows(const zo_heads& x, const zo_heads& y, const void* gamma, uint32_t heads, uint32_t tokens, uint32_t rotary) {
  Side s;
  std::memset(&s, 0, sizeof s);
  s.x = static_cast<const char*>(x.data);
  s.y = static_cast<char*>(y.data);
  s.gamma = static_cast<const char*>(gamma);
  s.x_token = x.token_stride;
  s.x_head = x.head_stride;
  s.y_token = y.token_stride;
  s.y_head = y.head_stride;
  s.heads = std::max(heads, 1u);
  s.inv_heads = 1.0f / static_cast<float>(s.heads);
  s.rows = tokens * heads;
  s.rotary = rotary;
  return s;
}

int forward(Rotation& r, const zo_rotate& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const auto go = [&](auto storage) {
    typedef decltype(storage) S;
    return dispatch<S>(a.dim, a.rotary, a.interleaved != 0, [&](auto vec, auto lanes, auto pairs, auto inside) {
      return launch_forward<S, vec.value, lanes.value, pairs.value, inside.value>(r, a.rotary, a.interleaved != 0, st);
    });
  };
  return a.dtype == ZO_F32 ? go(F32{}) : go(BF16{});
}

}  // namespace
}  // namespace zo

extern "C" {

int zo_norm_rotate(const zo_rotate* a, void* stream) {
  using namespace zo;
  if (a == nullptr) return ZO_ERR_NULL;
  const int rc = check_rotate(*a, true);
  if (rc != ZO_OK) return rc;
  if (a->tokens == 0 || a->q_heads + a->k_heads == 0) return ZO_OK;
  Rotation r = rotation_of(*a);
  r.side[0] = side_rows(a->q, a->q_out, a->q_gamma, a->q_heads, a->tokens, a->rotary);
  r.side[1] = side_rows(a->k, a->k_out, a->k_gamma, a->k_heads, a->tokens, a->rotary);
  return forward(r, *a, stream);
}

int zo_norm_rotate_put_at(const zo_rotate_put* p, const int32_t* places, void* stream) {
  using namespace zo;
  if (p == nullptr) return ZO_ERR_NULL;
  const int rc = check_put(*p);
  if (rc != ZO_OK) return rc;
  if (reinterpret_cast<uintptr_t>(places) % 4 != 0) return ZO_ERR_ARG;
  const zo_rotate& a = p->a;
  if (a.tokens == 0 || a.q_heads + a.k_heads == 0) return ZO_OK;
  Rotation r = rotation_of(a);
  const zo_cache& c = p->cache;
  r.seqs = p->seqs;
  r.places = places;
  r.ids = p->table.ids;
  r.table_stride = p->table.stride;
  r.table_seqs = p->table.seqs;
  r.table_width = p->table.width;
  r.page_stride = c.page_stride;
  r.cache_token = c.token_stride;
  r.pages = c.pages;
  r.page_tokens = std::max(c.page_tokens, 1u);
  r.side[0] = side_rows(a.q, a.q_out, a.q_gamma, a.q_heads, a.tokens, a.rotary);
  r.side[1] = side_rows(a.k, zo_heads{c.k, 0, c.head_stride}, a.k_gamma, a.k_heads, a.tokens, a.rotary);
  r.side[2] = side_rows(p->v, zo_heads{c.v, 0, c.head_stride}, nullptr, a.k_heads, a.tokens, 0);
  r.side[1].put = r.side[2].put = 1;
  return forward(r, a, stream);
}

int zo_norm_rotate_put(const zo_rotate_put* p, void* stream) { return zo_norm_rotate_put_at(p, nullptr, stream); }

int zo_norm_rotate_back(const zo_rotate_back* b, void* stream) {
  using namespace zo;
  if (b == nullptr) return ZO_ERR_NULL;
  const int rc = check_back(*b);
  if (rc != ZO_OK) return rc;
  const zo_rotate& a = b->a;
  if (a.q_heads + a.k_heads == 0) return ZO_OK;
  Rotation r = rotation_of(a);
  r.partial = static_cast<float*>(b->work);
  r.side[0] = side_rows(a.q, b->dq, a.q_gamma, a.q_heads, a.tokens, a.rotary);
  r.side[1] = side_rows(a.k, b->dk, a.k_gamma, a.k_heads, a.tokens, a.rotary);
  const zo_heads* dy[2] = {&a.q_out, &a.k_out};
  for (int i = 0; i < 2; ++i) {
    r.side[i].dy = static_cast<const char*>(dy[i]->data);
    r.side[i].dy_token = dy[i]->token_stride;
    r.side[i].dy_head = dy[i]->head_stride;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const auto go = [&](auto storage) {
    typedef decltype(storage) S;
    return dispatch<S>(a.dim, a.rotary, a.interleaved != 0, [&](auto vec, auto lanes, auto pairs, auto inside) {
      return launch_back<S, vec.value, lanes.value, pairs.value, inside.value>(r, a.rotary, a.interleaved != 0, *b, st);
    });
  };
  return a.dtype == ZO_F32 ? go(F32{}) : go(BF16{});
}

}  // extern "C"
