// How the tree attention's work is dealt out to its workgroups: whole numbers alone, for the kernel and for checks on the host.
//
// An item is a sequence, a key head and kRows rows (a new token and a query head of the key head's group); it is cut into tiles of kTile
// tokens up to the last one that a row of it can see, and costs `visit` tiles more. The costs of all items, in order (sequence, key
// head, rows), are dealt out in equal runs. Every workgroup finds its run by itself from lengths and starts, which have to stand still.
#ifndef ZO_TREE_DEAL_H_
#define ZO_TREE_DEAL_H_

#include <cstdint>

#ifdef __HIPCC__
#define ZO_DEAL __host__ __device__ __forceinline__
#else
#define ZO_DEAL inline
#endif

namespace zo {

struct Batch {
  const int32_t *lengths, *starts;
  const uint64_t* seen;
  double inv_group;  // of a group's query heads
  uint32_t tokens, seqs, width, page_tokens, heads, group, visit;
};

ZO_DEAL uint32_t less(uint32_t a, uint32_t b) { return a < b ? a : b; }

// Floor of n / d for n below 2^52: exact, since quotients of neighbours are further apart than an fp64 rounding.
ZO_DEAL uint64_t quotient(uint64_t n, uint64_t d) { return static_cast<uint64_t>(static_cast<double>(n) / static_cast<double>(d)); }

struct Seq {
  uint32_t token, count;  // its new tokens
  uint32_t cached, len;   // tokens before them, and with them: as many as the table holds
  uint32_t blocks;        // items of each key head
};

template <uint32_t kRows>
ZO_DEAL Seq seq_of(const Batch& b, uint32_t seq) {
  const int64_t room = static_cast<int64_t>(b.width) * b.page_tokens, most = b.tokens;
  int64_t first = b.starts[seq], last = b.starts[seq + 1], cached = b.lengths[seq];
  first = first < 0 ? 0 : first > most ? most : first;
  last = last < first ? first : last > most ? most : last;
  cached = cached < 0 ? 0 : cached > room ? room : cached;
  Seq s;
  s.token = static_cast<uint32_t>(first);
  s.count = static_cast<uint32_t>(last - first);
  s.cached = static_cast<uint32_t>(cached);
  s.len = static_cast<uint32_t>(cached + s.count < room ? cached + s.count : room);
  s.blocks = (s.count * b.group + kRows - 1) / kRows;
  return s;
}

// The new token of a row (rows below 2^24: the product's error stays below the half's share).
ZO_DEAL uint32_t node_of(const Batch& b, uint32_t row) { return static_cast<uint32_t>((static_cast<double>(row) + 0.5) * b.inv_group); }

// How many tokens the rows of a sequence up to (and without) `row` can see.
ZO_DEAL uint32_t visible(const Batch& b, const Seq& s, uint32_t row) {
  if (b.seen) return s.len;
  return less(s.len, s.cached + node_of(b, less(row, s.count * b.group) - 1) + 1);
}

// Tiles of an item; at least one, which writes the rows that see nothing. Its cost is b.visit tiles more.
template <uint32_t kRows, uint32_t kTile>
ZO_DEAL uint32_t tiles_of(const Batch& b, const Seq& s, uint32_t block) {
  const uint32_t tiles = (visible(b, s, (block + 1) * kRows) + kTile - 1) / kTile;
  return tiles > 1 ? tiles : 1;
}
template <uint32_t kRows, uint32_t kTile>
ZO_DEAL uint32_t cost_of(const Batch& b, const Seq& s, uint32_t block) {
  return tiles_of<kRows, kTile>(b, s, block) + b.visit;
}

// The cost of one key head of a sequence. lanes.sum(n, f): f(0) + .. + f(n - 1), by all lanes together.
template <uint32_t kRows, uint32_t kTile, class Lanes>
ZO_DEAL uint64_t head_cost(const Batch& b, const Seq& s, const Lanes& lanes) {
  if (s.blocks == 0) return 0;
  if (b.seen) return static_cast<uint64_t>(s.blocks) * cost_of<kRows, kTile>(b, s, 0);
  return lanes.sum(s.blocks, [&](uint32_t block) { return cost_of<kRows, kTile>(b, s, block); });
}

// The run of each worker: the total cost in equal parts, the first ones longer by one.
struct Runs {
  uint64_t each, longer;
  uint32_t workers;
  ZO_DEAL Runs(uint64_t total, uint32_t most) {
    workers = total < most ? static_cast<uint32_t>(total) : most;
    if (workers == 0) workers = 1;
    each = quotient(total, workers);
    longer = total - each * workers;
  }
  ZO_DEAL uint64_t first(uint32_t w) const { return w * each + (w < longer ? w : longer); }
  ZO_DEAL uint32_t worker_of(uint64_t place) const {
    const uint64_t head = longer * (each + 1);  // of the longer runs
    return static_cast<uint32_t>(place < head ? quotient(place, each + 1) : longer + quotient(place - head, each));
  }
};

struct Item {
  Seq s;
  uint32_t seq, head, block;
  uint64_t first;  // where its first tile is, behind its own cost
};

// The item that `at` lies in; `seq` begins at `before` and not behind it. lanes.seq(n) is sequence n, lanes.first_over(n, rest, f, block,
// cost) the first block whose f and all before it add up to more than the rest, and what those before it add up to. False: none, which needs
// other lengths or starts than the runs were made from.
template <uint32_t kRows, uint32_t kTile, class Lanes>
ZO_DEAL bool seek(const Batch& b, uint32_t seq, uint64_t before, uint64_t at, const Lanes& lanes, Item& item) {
  uint64_t cost = 0;
  for (;; ++seq) {
    if (seq >= b.seqs) return false;
    item.s = lanes.seq(seq);
    cost = head_cost<kRows, kTile>(b, item.s, lanes);
    if (at < before + cost * b.heads) break;
    before += cost * b.heads;
  }
  item.seq = seq;
  item.head = static_cast<uint32_t>(quotient(at - before, cost));
  before += cost * item.head;
  if (b.seen) {
    const uint32_t each = cost_of<kRows, kTile>(b, item.s, 0);
    item.block = static_cast<uint32_t>(quotient(at - before, each));
    before += static_cast<uint64_t>(item.block) * each;
  } else {
    uint64_t blocks_before;
    if (!lanes.first_over(item.s.blocks, at - before, [&](uint32_t block) { return cost_of<kRows, kTile>(b, item.s, block); }, item.block, blocks_before))
      return false;
    before += blocks_before;
  }
  item.first = before + b.visit;
  return true;
}

// The tiles begin .. end - 1 of an item of which the run at .. end has some (item.first < end).
struct Share {
  uint32_t begin, end;
  ZO_DEAL Share(uint64_t at, uint64_t run_end, uint64_t item_first, uint32_t tiles) {
    begin = at <= item_first ? 0u : static_cast<uint32_t>(at - item_first);
    end = run_end - item_first < tiles ? static_cast<uint32_t>(run_end - item_first) : tiles;
  }
};

// Behind an item's last tile, at `at`: the next one. False: the run ends here, or no sequence follows (as in seek()).
template <class Lanes>
ZO_DEAL bool next_item(const Batch& b, uint64_t at, uint64_t run_end, const Lanes& lanes, Item& item) {
  item.first = at + b.visit;
  if (++item.block == item.s.blocks) {
    item.block = 0;
    if (++item.head == b.heads) {
      item.head = 0;
      if (at >= run_end) return false;
      do {
        if (++item.seq >= b.seqs) return false;
        item.s = lanes.seq(item.seq);
      } while (item.s.blocks == 0);
    }
  }
  return at < run_end;
}

// Whether a run that began at `first` and has come to `at` leaves the item open that it began last: then the run that ends the item
// writes the entry for both, otherwise this one its own (empty) one.
ZO_DEAL bool leaves_open(uint64_t first, uint64_t at, uint64_t item_first) { return item_first >= first && item_first < at; }

}  // namespace zo

#endif  // ZO_TREE_DEAL_H_
