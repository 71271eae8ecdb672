// How sp_attn_cross divides chunks of more than a few tokens over the chip, from the host-side hints alone.  Without a mask all query
// tiles of a sequence are equally long, so the causal calls' rules (cut_plan.h), made for triangles, are not its own.  Plain code
// that compiles for the host as well: the CPU tests run it.
//
// Times are estimated in us from constants that leave the least behind on 960 batches drawn at random (eight head shards, 1 to 24
// sequences, up to 1600 workgroups of 128 columns, 20 to 8192 keys; equal lengths, unequal ones of both sides, unequal keys only;
// all forms but solo workgroups timed): 2.3 % over the best form of each batch, where the causal rules leave 7 %.  Both sides of it: 1 x 1137
// queries on 4580 keys at 32q/4kv in halves 112 us (a second round of workgroups for the last tenth), whole tiles 88; 2 x 206 on 2284 at
// 16q/2kv 28 and 44; 12 x 17..600 on 65..2500 at 12q/3kv, head_dim 64, 27 and 38.
#pragma once
#include <stddef.h>

#include "cut_plan.h"

namespace sp {

constexpr int kCus = 256;

struct CrossShape {
  bool halves;  // 128 columns, whose keys two wave groups share; else whole tiles of 256 (head_dim 64: 128, three workgroups a CU)
  bool solo;    // head_dim 128: 128 columns, two workgroups a CU
  bool ranked;  // workgroups take their items by keys plus the tile's place in its chunk, most first (the causal calls' weight); else in (tile, sequence) order
  int pieces;   // of the key ranges (halves only)
};

inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

// Pieces for launches that leave CUs idle: a key tile of a piece costs 0.4 us, the merge 2 us and 0.4 us per thousand partial rows of
// 128 channels.
// 4 x 14 queries on 2967 keys at 8q/1kv 31.6 us in one piece, 14.7 in 16; 1 x 168 on 1819 22.7, 19.1 in 4; 2 x 206 on 2284 at
// 16q/2kv 27.7, 28.8 in 4.  All of them in one round of workgroups, with some room for the estimate.
inline int cross_piece_count(long rows, long wgs, long max_kv_len, int head_dim) {
  const long tiles = ceil_div(max_kv_len, 64);
  const int cap = kv_split_cap(rows);
  double least = 0.4 * tiles;
  int best = 1;
  for (int p = 2; p <= cap && p * wgs <= 240 && 2 * p <= tiles; ++p) {
    const double t = 0.4 * ceil_div(tiles, p) + 2 + 0.4e-3 * rows * p * head_dim / 128;
    if (t < least) {
      least = t;
      best = p;
    }
  }
  return best;
}

// Keys that stay in LDS (attn_cross_resident.hip), 32 per block: two workgroups of four waves a CU where both fit, else one of eight.  One
// round of them, if that is up to eleven times 32 columns a wave (16 with eight waves); beyond, and where chunks are uneven, shorter ones,
// whose ends leave less idle (191 even batches of 4 to 40: three instead of up to 16 times 1.1 to 1.18 times as fast from 12 on, 0.85 to 1.03
// before; 69 uneven ones 1.2 times, with eight waves 102 more 1.05; but 2 x 65039 queries on 236 at 8q/1kv, 16 times with eight waves,
// 204 us, five 268).
//
// Up to 128 keys (329 batches of 9 to 5000 queries: 1.3 times as fast as query tiles at head_dim 64 in the mean, 1.7 at 128, one of
// them slower, by 7 %; 14 x 1844 queries on 129 at 32q/8kv 252 us in tiles, 137 so); up to 256 where there are enough queries (8 x 1749 on
// 229 at 16q/2kv 74 and 59, but 1 x 78 on 251 at 8q/1kv 11.7 and 16), at head_dim 128 and even chunks up to 320 (25 batches on more than 256:
// 1.13 times as fast as any tiles in the mean; uneven chunks 0.6 to 1.4).  At head_dim 64 the weights are the work there: 0.57 to 1.15.
constexpr int kResidentLds = 160 * 1024, kResidentPair = 128 * 1024;
struct CrossResident {
  int blocks;  // 0: not taken
  int waves;
  int rounds;  // of 32 columns per wave
};
inline CrossResident cross_resident(long rows, long streams, int columns, long max_q_len, long max_kv_len, int head_dim) {
  CrossResident r = {0, 0, 0};
  const bool uneven = 10.0 * rows < 9.0 * streams * columns * max_q_len;
  if (max_kv_len < 1 || max_kv_len > (head_dim == 128 && !uneven ? 320 : 256) || (max_kv_len > 128 && rows < 48000) || max_q_len > (1 << 24) || streams > 0x7fffffffL) return r;
  const long blocks = ceil_div(max_kv_len, 32), lds = blocks * 2 * 32 * head_dim * 2;
  r.waves = 2 * lds <= kResidentPair ? 4 : 8;
  const long wgs = (r.waves == 4 ? 2 : 1) * kCus, rounds = ceil_div(rows, 32 * r.waves * wgs);
  const long most = uneven ? 3 : r.waves == 4 ? 11 : 16;
  r.rounds = (int)(rounds < 1 ? 1 : rounds <= most ? rounds : uneven || r.waves == 4 ? 3 : 8);
  const long least = ceil_div(max_q_len * columns, 32L * r.waves * 65535);  // what the grid holds
  if (r.rounds < least) r.rounds = (int)least;
  r.blocks = (int)blocks;
  return r;
}

// Whether it also serves chunks of a few tokens, as against the decode kernel (160 batches of 1 to 120 sequences): up to 64 keys (means of
// 1.1 to 1.2 times as fast at head_dim 128, 1.0 to 1.1 at 64), and up to 128 where the rows are more than a round of the decode kernel's
// workgroups (1.2 to 1.8 times; otherwise as fast or up to 9 % slower).  99 x 2 tokens on 17 keys at 32q/8kv 17.2 and 8.9 us; 50 x 1 on 66
// at 8q/1kv 5.5 and 6.7.
inline bool cross_resident_for_few(long streams, long max_kv_len, int head_dim) {
  return max_kv_len <= 64 || (max_kv_len <= 128 && streams > (head_dim == 128 ? 1 : 2) * kCus);
}

// Chunks of a few column tiles of a wave (q_cap tokens each): every tile in a workgroup of the decode kernel of its own, which reads the
// keys again but begins in a third of the time that a query tile takes.  Up to 512 keys each in one launch, where the workgroups are
// one round (240 batches: 1.28 times as fast in the mean, the worst 0.93); longer ranges
// in splits that are merged, for few workgroups and keys (about 170 batches: 1.12 times, six of them more than 5 % slower; 1 x 64 tokens on
// 2000 at 32q/4kv 18.6 -> 16.1, 1 x 32 on 2616 16.2 -> 14.8, but 15 x 33 on 516 at 12q/3kv, head_dim 64, 9.5 and 13.4).
struct CrossTiles {
  int tiles;  // 0: not taken
  int splits, chunk;
};
inline CrossTiles cross_tiles(int batch, int n_hgroups, int q_cap, long max_q_len, long max_kv_len, int head_dim, bool can_split) {
  CrossTiles t = {0, 0, 0};
  const double rows = (double)batch * n_hgroups * ceil_div(max_q_len, q_cap);
  const int resident = head_dim == 128 ? kCus : 2 * kCus;
  if (max_kv_len < 1 || max_q_len <= q_cap || rows > resident || (max_kv_len > 512 && (!can_split || rows > (head_dim == 128 ? 64 : 96) || rows * max_kv_len > 131072))) return t;
  t.chunk = max_kv_len <= 512 ? 512 : 256;
  while (max_kv_len > 512 && rows * ceil_div(max_kv_len, t.chunk) > resident) t.chunk += 128;  // ends at 768: the product above
  t.splits = (int)ceil_div(max_kv_len, t.chunk);
  t.tiles = (int)ceil_div(max_q_len, q_cap);
  return t;
}
// Bytes of its partials.
inline size_t cross_tiles_bytes(const CrossTiles &t, int batch, int num_q_heads, long max_q_len, int head_dim) {
  return t.tiles == 0 || t.splits == 1 ? 0 : (size_t)batch * num_q_heads * max_q_len * t.splits * (head_dim + 2) * sizeof(float);
}

// columns: query columns of a token (heads that share a KV head's column dimension); streams: sequences x head groups.
inline CrossShape cross_shape(long rows, int batch, long streams, int columns, long total_q, long max_q_len, long max_kv_len, int head_dim,
                              bool can_cut) {
  const long tiles = ceil_div(max_kv_len, 64);
  const long found = rows / 128 + (streams + 1) / 2, wgs = found > streams ? found : streams;  // workgroups of 128 columns that find work
  const bool uneven = 10.0 * total_q < 9.0 * batch * max_q_len;
  // The search for an item by its rank costs a microsecond per workgroup.  It pays where there is more than one round and the
  // lengths differ: those of the queries are known; the keys' are taken to differ where they are not the queries' own, if the key
  // ranges are long (8 x 270..1089 queries on 470..1891 keys at 16q/2kv, head_dim 64: 60 us by order, 45 ranked; 2 x 1904 on 101 at
  // 32q/4kv 28.5 and 39.6).
  auto rank = [&](int cols) { return batch >= 2 && (double)streams * ceil_div(max_q_len * columns, cols) > kCus && (uneven ? tiles >= 2 : max_q_len != max_kv_len && tiles >= 30); };
  CrossShape s;
  s.solo = false;
  s.pieces = can_cut ? cross_piece_count(rows, wgs, max_kv_len, head_dim) : 1;
  const bool rank_halves = rank(128), rank_whole = rank(head_dim == 128 ? 256 : 128);
  if (s.pieces > 1) {
    s.halves = true;
    s.ranked = rank_halves;
    return s;
  }
  // Workgroups that find work: of even batches as many as the longest chunk has (8 x 550 queries on 1328 keys at 12q/2kv are 288 whole tiles,
  // two rounds: 70 us, halves 50).
  auto items = [&](int cols) {
    const double all = (double)streams * ceil_div(max_q_len * columns, cols);
    return uneven ? found * 128.0 / cols : all < 1e15 ? all : 1e15;
  };
  // A tile of an item: 0.55 us in halves, 1 whole; at head_dim 64 0.9, or 0.42 times the workgroups on its CU.  Starts, merges and
  // stores: 10 us a round in halves, 9 whole.  Uneven batches: the mean item at 0.4 of the longest, and half of that (all of it by
  // order) for the end.
  const double n = items(128);
  auto span = [&](double items, double t, double start, bool ranked) {
    if (!uneven) return (double)(long)((items + kCus - 1) / kCus) * (t + start);
    const double even = items * (0.4 * t + start) / kCus + (ranked ? 0.5 : 1.0) * t;
    return even > t + start ? even : t + start;
  };
  double whole;
  if (head_dim == 128) {
    whole = span(items(256), 1.0 * tiles, 9, rank_whole);
  } else if (uneven) {
    const double even = n / kCus * 0.4 * 0.42 * tiles + 0.21 * tiles;
    whole = 9 + (even > 0.9 * tiles ? even : 0.9 * tiles);
  } else {
    const long full = (long)n / (3 * kCus), left = ceil_div((long)n % (3 * kCus), kCus);  // rounds of three workgroups a CU, and the last
    whole = full * (3 * 0.42 * tiles + 9);
    if (left > 0) whole += (0.42 * left > 0.9 ? 0.42 * left : 0.9) * tiles + 9;
  }
  const double halves = span(n, 0.55 * tiles, 10, rank_halves);
  s.halves = halves <= whole;
  s.ranked = s.halves ? rank_halves : rank_whole;
  if (head_dim == 64 || max_kv_len <= 256 || n <= kCus) return s;
  // Two workgroups of 128 columns on a CU, whose starts and stores are behind each other's multiplications: a tile takes 0.62 us per workgroup
  // there, one alone 0.8; starts 4 us a round.  Where every workgroup of 128 columns has a CU to itself the halves are faster (500 batches: by
  // 2 to 25 %, the more keys the more).  On more tiles than about 32 whole tiles, which load every key once per 256 columns,
  // are as fast or faster.  873 batches on 257 to 6000 keys: 2 % over the best of all forms, 10 % without this one; 12 x 1212 queries on 340
  // keys at 32q/4kv 163 -> 121 us, 7 x 313 on 529 46 -> 36; but 6 x 714 on 2014 at 8q/1kv 45.6 and 51.9.
  const long full = (long)n / (2 * kCus), left = ceil_div((long)n % (2 * kCus), kCus);
  double solo;
  if (uneven) {
    const double even = n / kCus * (0.4 * 0.62 * tiles + 3) + 0.5 * 0.8 * tiles, longest = 0.8 * tiles + 4;
    solo = even > longest ? even : longest;
  } else {
    solo = full * (2 * 0.62 * tiles + 4);
    if (left > 0) solo += (0.62 * left > 0.8 ? 0.62 * left : 0.8) * tiles + 4;
  }
  if (solo < (halves < whole ? halves : whole)) {
    s.solo = true;
    s.halves = false;
    s.ranked = rank_halves;
  }
  return s;
}

}  // namespace sp
