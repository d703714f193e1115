// The deal of the tree attention's work, as its workgroups find it, on the host under AddressSanitizer and UBSan: every tile of every
// item is dealt out once, searches end, and each split item has one entry, behind parts that were written. Prints "tree_deal_check ok".
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "zo_tree_deal.h"

namespace {

using namespace zo;

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      std::exit(1);                               \
    }                                             \
  } while (0)

std::mt19937_64 rng(1);
uint32_t below(uint64_t n) { return static_cast<uint32_t>(rng() % n); }

template <uint32_t kRows>
struct OneLane {
  const Batch& batch;
  Seq seq(uint32_t n) const {
    CHECK(n < batch.seqs);
    return seq_of<kRows>(batch, n);
  }
  template <class F>
  uint64_t sum(uint32_t n, const F& f) const {
    uint64_t all = 0;
    for (uint32_t i = 0; i < n; ++i) all += f(i);
    return all;
  }
  template <class F>
  bool first_over(uint32_t n, uint64_t rest, const F& f, uint32_t& at, uint64_t& before) const {
    before = 0;
    for (at = 0; at < n; ++at) {
      if (before + f(at) > rest) return true;
      before += f(at);
    }
    return false;
  }
};

// The sequences' costs in front of each thread's, and in all.
template <uint32_t kRows, uint32_t kTile>
std::vector<uint64_t> deal(const Batch& b, uint32_t threads, uint32_t& each) {
  each = (b.seqs + threads - 1) / threads;
  std::vector<uint64_t> before(threads + 1, 0);
  for (uint32_t t = 0; t < threads; ++t) {
    uint64_t cost = 0;
    for (uint32_t seq = t * each; seq < (t + 1) * each && seq < b.seqs; ++seq)
      cost += head_cost<kRows, kTile>(b, seq_of<kRows>(b, seq), OneLane<kRows>{b});
    before[t + 1] = before[t] + cost * b.heads;
  }
  return before;
}

// All workers' runs. `stands`: the batch is the one that the runs were made from; otherwise every search has to end, inside the batch.
template <uint32_t kRows, uint32_t kTile>
void walk(const Batch& b, const std::vector<uint64_t>& before, uint32_t threads, uint32_t each, uint32_t most, bool stands) {
  const uint64_t total = before[threads];
  const OneLane<kRows> lanes{b};
  const Runs runs(total, most);
  if (total == 0) return;
  CHECK(runs.workers > 0 && runs.workers <= most && runs.first(0) == 0 && runs.first(runs.workers) == total);
  std::vector<uint64_t> first_item(b.seqs + 1, 0);  // of each sequence, in the list of items
  for (uint32_t s = 0; s < b.seqs; ++s) first_item[s + 1] = first_item[s] + uint64_t{seq_of<kRows>(b, s).blocks} * b.heads;
  struct Tiles {
    uint32_t done = 0, all = 0, first = ~0u, last = 0;
  };
  std::vector<Tiles> items(first_item[b.seqs]);
  std::vector<int> parts(2 * runs.workers, 0), entries(runs.workers, 0);
  struct Entry {
    uint32_t first, last;
  };
  std::vector<Entry> split;
  for (uint32_t w = 0; w < runs.workers; ++w) {
    const uint64_t begin = runs.first(w), end = runs.first(w + 1);
    CHECK(begin < end && runs.worker_of(begin) == w && runs.worker_of(end - 1) == w);
    uint64_t at = begin;
    uint32_t chunk = 0;
    for (uint32_t step = threads / 2; step > 0; step /= 2)
      if (before[chunk + step] <= at) chunk += step;
    Item item;
    if (!seek<kRows, kTile>(b, chunk * each, before[chunk], at, lanes, item)) {
      CHECK(!stands);
      continue;
    }
    while (at < end && item.first < end) {
      CHECK(item.seq < b.seqs && item.head < b.heads && item.block < item.s.blocks);
      const uint32_t tiles = tiles_of<kRows, kTile>(b, item.s, item.block);
      CHECK(item.block * kRows < item.s.count * b.group && item.s.token + item.s.count <= b.tokens);
      const Share share(at, end, item.first, tiles);
      CHECK(share.end >= 1 && share.end <= tiles);
      if (stands) {
        CHECK(share.begin < share.end);
        Tiles& t = items[first_item[item.seq] + uint64_t{item.head} * item.s.blocks + item.block];
        CHECK(t.done == share.begin);
        t.done = share.end;
        t.all = tiles;
        const bool whole = share.begin == 0 && share.end == tiles;
        if (share.begin == 0) t.first = w;
        t.last = w;
        if (!whole) ++parts[2 * w + (share.begin == 0 ? 1 : 0)];
        if (share.end == tiles && !whole) {
          const uint32_t owner = runs.worker_of(item.first);
          CHECK(owner == t.first && owner < w);
          ++entries[owner];
          split.push_back({owner, w});
        }
      }
      at = item.first + share.end;
      if (share.end == tiles && !next_item(b, at, end, lanes, item)) break;
    }
    if (!leaves_open(begin, at, item.first)) ++entries[w];
  }
  if (!stands) return;
  for (const Tiles& t : items) CHECK(t.all > 0 && t.done == t.all);
  for (int n : entries) CHECK(n == 1);
  for (int n : parts) CHECK(n <= 1);
  std::vector<int> read(2 * runs.workers, 0);
  for (const Entry& e : split)
    for (uint32_t w = e.first; w <= e.last; ++w) ++read[2 * w + (w == e.first ? 1 : 0)];
  CHECK(read == parts);
}

template <uint32_t kRows, uint32_t kTile>
void form(Batch b, uint32_t threads, std::vector<int32_t>& lengths) {
  for (uint32_t visit : {0u, 1u, 4u}) {
    b.visit = visit;
    uint32_t each;
    const std::vector<uint64_t> before = deal<kRows, kTile>(b, threads, each);
    for (uint32_t most : {8u, 256u, 512u}) walk<kRows, kTile>(b, before, threads, each, most, true);
    // lengths that another call changes meanwhile
    const std::vector<int32_t> kept = lengths;
    for (int32_t& n : lengths)
      if (below(2) != 0) n = static_cast<int32_t>(below(2000));
    walk<kRows, kTile>(b, before, threads, each, 256, false);
    lengths = kept;
  }
}

void batch(std::vector<int32_t> lengths, std::vector<int32_t> starts, uint32_t tokens, uint32_t heads, uint32_t group, uint32_t width, uint32_t page,
           bool masks) {
  static const uint64_t seen = 0;
  const uint32_t seqs = static_cast<uint32_t>(lengths.size());
  Batch b = {lengths.data(), starts.data(), masks ? &seen : nullptr, 1.0 / group, tokens, seqs, width, page, heads, group, 0};
  form<32, 128>(b, 256, lengths);
  form<128, 64>(b, 256, lengths);
  form<128, 32>(b, 256, lengths);
  form<256, 64>(b, 512, lengths);
}

void batches() {
  // a batch whose call of a kernel that is no more did not end: 30 and 9 tokens of 24 heads on one behind 70 and 20
  for (bool masks : {false, true}) batch({70, 20}, {0, 30, 39}, 39, 1, 24, 194, 16, masks);
  for (int round = 0; round < 400; ++round) {
    const uint32_t seqs = 1 + below(round % 8 == 0 ? 1500 : round % 3 == 0 ? 60 : 6), heads = 1 + below(12), group = 1 + below(round % 5 ? 8 : 30);
    const uint32_t page = 16 * (1 + below(5)), width = 1 + below(200);
    const uint32_t longest = round % 4 == 0 ? 400 : 1 + below(40), context = below(2) ? 100 : 5000;
    std::vector<int32_t> lengths(seqs), starts(seqs + 1);
    starts[0] = static_cast<int32_t>(below(4));
    for (uint32_t s = 0; s < seqs; ++s) {
      lengths[s] = below(20) == 0 ? -3 : below(20) == 0 ? 0x7FFFFFFF : static_cast<int32_t>(below(context));
      starts[s + 1] = starts[s] + static_cast<int32_t>(below(4) == 0 ? 0 : below(longest + 1));
    }
    uint32_t tokens = static_cast<uint32_t>(starts[seqs]) + below(3);
    if (below(4) == 0) tokens -= below(tokens + 1) / 2;  // starts behind the rows
    if (below(8) == 0) starts[0] = -5;
    if (below(8) == 0) starts[below(seqs + 1)] = static_cast<int32_t>(below(tokens + 9));  // falls, perhaps
    batch(lengths, starts, tokens, heads, group, width, page, below(2) != 0);
  }
}

// Quotients next to whole numbers, and tokens of rows, are exact.
void numbers() {
  for (int round = 0; round < 2000000; ++round) {
    const uint64_t d = 1 + rng() % (uint64_t{1} << (1 + below(51))), most = (uint64_t{1} << 52) - 1, k = rng() % (most / d + 1);
    CHECK(quotient(k * d, d) == k);
    if (k > 0) CHECK(quotient(k * d - 1, d) == k - 1);
  }
  for (uint32_t group = 1; group < 70; ++group) {
    Batch b = {};
    b.inv_group = 1.0 / group;
    for (uint32_t i = 0; i < 4000; ++i) {
      const uint32_t row = i < 2000 ? i : below(1u << 24);
      CHECK(node_of(b, row) == row / group);
    }
  }
}

}  // namespace

int main() {
  numbers();
  batches();
  std::printf("tree_deal_check ok\n");
}
