// How an attention over a paged cache is cut for the chip and what memory that takes: arithmetic of host and device.
#pragma once

#include <algorithm>

#include "treekv_internal.h"

namespace tkv {

constexpr int PA_THREADS = 256, PA_WAVES = PA_THREADS / 64;
constexpr int TILE = 64, TILED_ROWS = PA_WAVES * 32;       // many rows: columns of a tile, rows of a workgroup

// A second sequence in a share costs a workgroup about what STRADDLE more columns do.  Up to SHORT columns a share,
// a size that is larger by no more and gives every sequence shares of its own, no more of them than were to be, is taken (8
// sequences of 2048 columns and one token, 8 KV heads: 22.0 -> 18.9 us); sequences that are more than the shares take one or
// two each (64 of 500: 29.5 -> 24.2 us; of 2048 columns 67 either way).  Row tiles: what 128 rows write and read again for
// another share costs about what it gains up to TILED_SHARE columns (200 tokens behind 1000, groups of 4: 33.3 -> 27.1 us).
constexpr int MIN_SHARE = 128;               // columns: a block for each wave
constexpr int STRADDLE = 256, SHORT = 1024, TILED_SHARE = 1024;
// A share is no larger than a sequence can be.  Where that leaves more shares than were to be, they are a sequence's own, one each:
// then nothing has to be merged, and nothing is needed for partial results.
constexpr int MAX_SHARE = 1 << 30;
struct Cut {
  int size;                                  // columns of a share
  bool own;                                  // each share is of one sequence, whose first one starts at its first token
};
// `total` columns (of all sequences, each one's rounded up to whole blocks; `wide`: past 32 bits) in `shares` of them, or a few more
// where they are a sequence's own: `count(size)` says how many those would be of the first 64 sequences.
template <class Count>
__host__ __device__ inline Cut cut_columns(long long total, int shares, int batch, bool tiled, bool wide, Count count) {
  const long long each = wide ? (total + shares - 1) / shares : (int)(((unsigned)total + shares - 1) / (unsigned)shares);
  const long long up = (each + 31) / 32 * 32, least = up > MIN_SHARE ? up : MIN_SHARE;
  Cut c;
  c.size = (int)(least < MAX_SHARE ? least : MAX_SHARE);
  if (tiled && c.size <= TILED_SHARE / 2) c.size *= 2;
  c.own = tiled || c.size == MIN_SHARE || least > MAX_SHARE;
  if (!c.own && c.size <= SHORT && !wide && shares > 1) {
    c.own = batch > shares;
    if (batch <= (shares < 64 ? shares : 64))
      for (int size = c.size; size <= c.size + STRADDLE; size += 64)
        if (count(size) <= shares) { c.size = size; c.own = true; break; }
  }
  return c;
}
__host__ __device__ inline int shares_in(int length, int size) { return (int)(((unsigned)length + (unsigned)size - 1) / (unsigned)size); }
// Sequence b's shares, `start` its first column among all (or its first share among all: `own`).
struct Runs {
  int first, count;                          // its first share, how many
};
__host__ __device__ inline Runs runs_of(const Cut& c, bool wide, long long start, int length) {
  if (c.own) return {(int)start, shares_in(length, c.size)};
  const int first = wide ? (int)(start / c.size) : (int)start / c.size;
  return {first, !length ? 0 : (wide ? (int)((start + length - 1) / c.size) : ((int)start + length - 1) / c.size) - first + 1};
}
// Where the partial results of a sequence's shares lie.
//   dense   every share of every sequence has one: shares + batch of them.
//   sparse  sequences of several shares have them.  Counted in columns, each of their shares goes on from, or is the first before, a
//           border between two of `size`, and a border has one sequence before it and one behind: two places for
//           each are enough, however many sequences there are.
// That of its first share, `column` columns into all (asked for if sparse), and from there to that of its k-th.
__host__ __device__ inline int part_of_first(const Cut& c, bool wide, bool sparse, const Runs& r, long long column, int b) {
  if (!sparse) return c.own ? r.first : r.first + b;
  return 2 * (!c.own ? r.first : wide ? (int)(column / c.size) : (int)column / c.size) + 1;
}
__host__ __device__ inline int part_at(bool sparse, int k) { return sparse ? (k ? 2 * k - 1 : 0) : k; }
inline bool is_sparse(int shares, int batch, bool keep) { return !keep && shares < batch; }
inline size_t parts(int shares, int batch, bool keep) { return shares == 1 && !keep ? 0 : is_sparse(shares, batch, keep) ? 2 * (size_t)shares : (size_t)shares + batch; }
inline bool past_32_bits(const treekv_paged_cache& c) { return (long long)c.batch * ((long long)c.table_width * c.page_size + 31) > 1 << 30; }

// ---- a call's shape, on the host ---------------------------------------------------------------
struct AttendShape {
  int rows, tiles, shares;                   // rows of a tile
  int weigh_splits;                          // parts of the rows that a column's weights are summed in
  int short_shares;                          // of the sequences with up to 16 rows, where they are taken by themselves
  bool tiled, keep, short_keep, weigh_tiled; // many rows through LDS; logits kept for the weights; weights of many rows through LDS
  size_t part, short_part, logits, stat, gains;     // bytes of scratch: shares' results, logits, rows' references and sums, splits' sums
};
inline AttendShape attend_shape(const treekv_paged_cache& c, int tokens, int longest, int weigh) {
  const long long rows = (long long)longest * (c.q_heads / c.kv_heads), cap = (long long)c.table_width * c.page_size;
  const long long units = (long long)c.batch * c.kv_heads;
  AttendShape s;
  s.tiled = rows > 64 && c.dtype == TREEKV_BF16;
  s.rows = rows <= 16 ? 16 : s.tiled ? TILED_ROWS : 32;
  s.tiles = (int)((rows + s.rows - 1) / s.rows);
  const long long groups = (long long)c.kv_heads * s.tiles, want = s.tiled ? 512 : 256;
  // (few rows: one workgroup a compute unit has enough on its way, and leaves fewer shares to add: 16 sequences of 16000 columns
  // and one token 118 us, with two 121, with three or four 123 to 134; row tiles: two, 168 us for 512 tokens behind 16000, with
  // one 186, but no more of them than are at work together, 768 tokens 275 us, with a third more 305)
  const long long most = ((long long)c.batch * cap + MIN_SHARE - 1) / MIN_SHARE;
  s.shares = (int)(s.tiled ? max(want / groups, 1ll) : (want + groups - 1) / groups);
  if (s.shares > most) s.shares = (int)most;
  // A few chunks among many sequences of a token or two: those are attended by the kernel for few rows, in a launch of its own
  // (512 tokens and 31 single ones behind 8000 each, 8 groups of 4: 268 us in place of 596, with weights 374 in place of 855).  From
  // where the longest is four times the average: 4 of 64 tokens and 12 single ones (3.8) take 139 us together, 137 apart, and 16
  // single ones (4.7) 236 and 164; one of 64 and three (3.8) 45 and 56, four (4.7) 63 and 64.  (Chunks of 512 would gain
  // before: 4 and 8, 3 times, 443 and 369.)
  s.short_shares = s.tiled && (long long)tokens * 4 <= (long long)longest * c.batch && c.q_heads / c.kv_heads <= 16
                       ? (int)std::min<long long>((256 + c.kv_heads - 1) / c.kv_heads, most) : 0;
  // keys once more cost d elements a column, kept logits two words for each row: up to 1 GiB of them, for up to 32 rows (8 sequences
  // of 8000 columns, groups of 4, 5 tokens: 54 us against 76 with the keys read again, 8 tokens 58 against 78, fp32 alike).  They are
  // counted by the table's width and whole tiles of rows, for lengths are on the device.
  s.weigh_tiled = s.tiled && c.q_heads / c.kv_heads <= TILE;     // (what that asks of the query rows' distance, the launch adds)
  s.keep = weigh && rows <= 32 && (size_t)units * s.rows * cap * 4 <= (size_t)1 << 30;
  s.short_keep = weigh && s.short_shares && (size_t)units * 16 * cap * 4 <= (size_t)1 << 30;
  s.part = align_up(parts(s.shares, c.batch, s.keep) * groups * s.rows * (c.head_dim + 4) * 4);
  s.short_part = s.short_shares ? align_up(parts(s.short_shares, c.batch, s.short_keep) * c.kv_heads * 16 * (c.head_dim + 4) * 4) : 0;
  s.logits = s.keep || s.short_keep ? align_up((size_t)units * (s.keep ? s.rows : 16) * cap * 4) : 0;
  // few column tiles: each one's rows are shared between up to 16 workgroups, with two tiles of them at least, and their sums added
  // in a launch of its own (attention and weights of 2048 tokens behind 2000, one group of 8: 297 -> 90 us, 512 of 8 groups of 4
  // alone 65 -> 41; four tiles at least: 100 tokens behind 1000 37 us, with two 34).  By the table's width too: the first of these
  // takes 218 us with a table for 32768.
  s.weigh_splits = 1;
  if (weigh && !s.keep && s.weigh_tiled) {
    const long long tiles = (cap + PA_WAVES * 32 - 1) / (PA_WAVES * 32) * units;
    s.weigh_splits = (int)std::max(std::min({512 / tiles, rows / (2 * TILE), 16ll}), 1ll);
  }
  s.gains = s.weigh_splits > 1 ? align_up((size_t)s.weigh_splits * units * cap * 4) : 0;
  s.stat = weigh && !s.keep ? align_up((size_t)tokens * c.q_heads * 8) : 0;
  return s;
}

// A launch has fewer than 2^32 threads.
constexpr long long MAX_GROUPS = (1ll << 32) / PA_THREADS - 1;
// The merge's workgroups, `at_once` rows each: so many of every (sequence, KV head), or of every KV head for all sequences one after
// the other (`packed`, where the longest sequence has many more than the others).  `rows`: the most of a sequence.  Where that would be
// more than a launch can have, a sequence gets as many as there can be, which go on to its next rows.
struct MergeGrid {
  int groups;
  bool packed;
};
inline MergeGrid merge_grid(int batch, int kv_heads, int G, int tokens, int rows, int at_once) {
  const int all = (rows + at_once - 1) / at_once;
  const long long packed = (long long)tokens * G / at_once + batch;
  if (2 * packed < (long long)all * batch && packed * kv_heads <= MAX_GROUPS) return {(int)packed, true};
  return {(int)std::min<long long>(all, MAX_GROUPS / ((long long)batch * kv_heads)), false};
}

}  // namespace tkv
