// Work plan of the attention over paged caches: which blocks every workgroup takes, for which query rows.
//
// A run is a stretch of blocks that some query tokens see together: the common prefix of several sequences, with the query tokens of
// all of them, or the rest of one sequence, with its own.  A run's query tokens are cut into tiles, and every (kv head, tile) of a run is a
// unit of the run's n_blk blocks; in short runs, where the end of a unit would cost its workgroup more than the blocks, four kv heads are one
// unit, a wavefront each.  All units are laid end to end and the list is divided evenly over the workgroups.  An entry of the list is a
// stretch of time, not of blocks: a block takes `cost` entries, by what its workgroup does with it, and a unit ends with `pad` entries more (states
// merged, a partial result stored, the next one's first blocks waited for).  A block belongs to the workgroup that has its first entry.  Units of a shared run are in the order of
// the kv heads: the tiles of a kv head read the same blocks at about the same time.  (Consecutive shares on one XCD, so that these tiles meet in one L2: as
// long with a prefix of 16 384 tokens for 64 sequences of 8, 159 us, though a quarter of the bytes came from behind the L2s; 47 instead of 46 us with three
// prefixes and contexts of their own, whose reads then fall on few XCDs.)
#pragma once
#include "paged.h"

namespace bass {

constexpr int kPagedWaves = 4;      // wavefronts of a workgroup
constexpr int kPagedShares = 256;   // workgroups of the attention launch: one per compute unit
// An entry is 1/8 us.  Of a block: up to 32 and 64 rows (four blocks at a time, a wavefront each); tiles of 128 and 256 rows (a block at a time, all
// wavefronts) over bf16 and INT8 pages.  Of the end of a unit, with the beginning of the next: by a wavefront per head, by all four, and of a tile.
// All of it fitted to heads of 128; heads of 64, with half the bytes and products per block and the same beginnings, are divided by the same numbers.
// Fitted to kernel times, us per layer before and with these: INT8, 6 sequences of 5 tokens behind 32 768, 32/8 heads 54 -> 35 (the workgroups without a tile had been given too
// much); 16 sequences of 6 behind 8192, 32 heads 47 -> 41, over INT8 51 -> 39; 64 of 8 behind 16 384, 32/8 heads, INT8 222 -> 200; three prompts 46 -> 42.
// The end of a tile at 76 / 108: 16 sequences of 4 behind 4096, 32/8 heads 24.7 / 21.1, 32 of 4 behind 1024, 64/8 heads 26.9 / 24.4; 32 of 4 behind 512, 32 heads, with the merge 31.3 / 34.2, 8 behind
// 4096, 64/8 heads, 28.3 / 30.5; the others level.
constexpr int kCostRows1 = 4, kCostRows2 = 6, kCostTile1 = 5, kCostTile2 = 7, kCostTile1Int8 = 5, kCostTile2Int8 = 10;
constexpr int kPadHeads = 64, kPadRows = 56, kPadTile = 108;
constexpr int kTileStart = 48;  // a workgroup that begins with a tile loses so much more than one that begins with few rows (see tile_cost)
// Short runs give each wavefront a kv head of its own: nothing is merged, but a workgroup has four partial results, and the list has fewer, longer
// units.  Worth it where units are many.  us per layer, heads of 128, 4 tokens, without -> with: 32/8 heads, 32 sequences of 40 / 100 / 200 / 400 tokens
// 15.4 / 16.3 / 18.7 / 21.7 -> 14.2 / 16.6 / 18.6 / 23.9; 128 sequences 33.2 / 37.4 / 45.2 / 55.5 -> 23.4 / 29.2 / 37.2 / 52.7; 4 sequences 9.1 / 10.9 / 12.7 / 13.4 ->
// 11.7 / 12.3 / 13.7 / 14.2; 64 rows, 128 sequences 54.8 / 59.6 / 68.6 / 80.8 -> 40.9 / 48.8 / 55.3 / 75.7; 24 sequences of 40 / 200 / 400 tokens, 16 rows
// 10.9 / 16.1 / 19.3 -> 13.9 / 17.2 / 21.2.  So where there is about a unit per workgroup, up to 8 blocks, and twice as many with more than 32 rows, whose states
// are twice as large to merge, or with four times the units.
constexpr int kHeadUnits = 240, kHeadBlocks = 8;
BASS_HD inline int head_blocks(int units, int rows) { return units < kHeadUnits ? 0 : rows > 32 || units >= 4 * kHeadUnits ? 2 * kHeadBlocks : kHeadBlocks; }
constexpr int kLeastEntries = 40;   // of a workgroup, as long as there are fewer workgroups than kPagedShares
// The merge adds up a partial result of every workgroup between the first and the last one that have a block of a unit, so each of them has to have one: a
// share must not be shorter than a block's entries.  At most that many: few rows, a kv head per wavefront; tiles, up to three times the plain cost (tile_cost:
// the quotient stays below it, because per < 3 (per / 3 + 1)).
constexpr int kCostTileMost = imax(imax(kCostTile1, kCostTile2), imax(kCostTile1Int8, kCostTile2Int8));
static_assert(kLeastEntries >= kPagedWaves * imax(kCostRows1, kCostRows2), "a share has a block of every unit that it lies in");
static_assert(kLeastEntries >= 3 * kCostTileMost, "a share has a block of every unit that it lies in");
constexpr int kTileRows = 256;      // most query rows of a tile
constexpr int kSlotRows = kTileRows;  // rows between the partial results of two workgroups (see partial_row)

struct PagedRun {
  int32_t row;       // whose table is read
  int32_t tok;       // shared: first entry of the token list; else: first query token b * kmax
  int32_t n_tok;     // query tokens
  int32_t tile_tok;  // query tokens of a tile
  int32_t n_tiles;
  int32_t first;     // first block
  int32_t n_blk;     // blocks
  int32_t L;         // tokens cached before the step; -1: shared (all of it is visible to all rows)
  int32_t start;     // entries of the list before this run
  int32_t row_base;  // partial rows before this run
  int32_t whole;     // 1: the sequence has no shared part, so a unit that is not cut is the final result
  int32_t cost;      // entries of a block
  int32_t pad;       // entries of the unit's end
  int32_t heads;     // kv heads of a unit: 1, or one for each wavefront
  int32_t reserved[2];
  BASS_HD int entries() const { return n_blk * cost + pad; }                                // of a unit
  BASS_HD int block_at(int entry) const { return imin((entry + cost - 1) / cost, n_blk); }  // first block that starts at `entry` or behind it
};

constexpr int kTileFrom = 32;  // shared runs: tiles where a tile has more rows
BASS_HD inline bool is_tile(bool shared, int rows) { return shared && rows > kTileFrom; }
BASS_HD inline int block_cost(bool shared, int rows, int heads, bool int8) {
  if (!is_tile(shared, rows)) return (rows <= 32 ? kCostRows1 : kCostRows2) * heads;
  return rows <= kTileRows / 2 ? (int8 ? kCostTile1Int8 : kCostTile1) : int8 ? kCostTile2Int8 : kCostTile2;
}
BASS_HD inline int unit_pad(bool shared, int rows, int heads) { return is_tile(shared, rows) ? kPadTile : heads > 1 ? kPadHeads : kPadRows; }
// Whether a common prefix is computed for all of its sequences together.  Separate sequences read it again from the caches; together, a workgroup has one
// more beginning and end, and every row one more partial result.  us per layer, separate / together, prefixes of 256 / 512 / 1024 / 2048 / 4096 tokens, 200
// of their own, 4 query tokens: 32 heads, 2 sequences 13.5 / 13.9 / 14.9 / 18.5 / 24.1 and 13.2 / 13.7 / 14.5 / 16.6 / 21.6, 4 sequences 13.8 / 16.0 / 18.6 / 23.1 / 32.8 and 13.7 /
// 15.4 / 16.7 / 18.6 / 22.8, 8 sequences 19.2 / 23.2 / 31.4 / 49.2 / 83.2 and 16.3 / 16.5 / 18.0 / 20.1 / 25.5; 32/8 heads, 8 sequences 14.0 / 14.7 / 15.7 / 20.3 / 29.5 and 13.9 / 15.7 / 17.3 /
// 20.4 / 24.2, 32 sequences 21.7 / 25.0 / 33.2 / 54.2 / 94.1 and 24.4 / 26.6 / 27.5 / 28.3 / 33.3; 64/8 heads, 8 sequences 14.6 / 15.5 / 17.0 / 21.7 / 31.4 and 18.8 / 21.9 / 25.9 / 27.1 /
// 30.5, 32 sequences 24.1 / 27.8 / 36.2 / 58.7 / 98.1 and 26.1 / 27.3 / 31.1 / 35.7 / 44.0.  In entries saved per workgroup: from about 12 on, or 55 with tiles, whose
// beginnings are long; but those are paid once for all prefixes of a batch.
// (32 sequences, 32/8 heads, 512 tokens are just beyond that line, with 57, and 1.6 us longer together.)
constexpr int kSavedRows = 12, kSavedTile = 55;
BASS_HD inline int saved_by_sharing(int members, int tokens, int tiles, int tile_tok, int n_blk, int g, int Hkv, bool int8) {
  const int64_t apart = (int64_t)members * block_cost(false, tokens * g / members, 1, int8), together = (int64_t)tiles * block_cost(true, tile_tok * g, 1, int8);
  const int64_t saved = (apart - together) * n_blk * Hkv / kPagedShares;
  return saved < 0 ? 0 : (int)(saved < (1 << 16) ? saved : 1 << 16);
}
BASS_HD inline bool worth_sharing(int saved, int saved_by_all, bool tile) { return saved >= kSavedRows && saved_by_all >= (tile ? kSavedTile : kSavedRows); }
// Every workgroup pays for a beginning, those with tiles more; in short lists that is much of their time, so that a tile's block counts for more there.
// per: entries of a workgroup by the plain costs.
BASS_HD constexpr int tile_cost(int cost, int per) { return (int)((int64_t)cost * per / imax(per - kTileStart, per / 3 + 1)) + 1; }

struct PagedHeader {
  int32_t signature, n_runs, total, per, rem, used;
  int32_t reserved[10];
};

// What a workgroup starts with; it goes on through the units (and runs) that follow until its entries are used up.
struct PagedShare {
  int32_t signature, run, unit, off, entries;  // first run, unit of the run, entry of the unit
  int32_t reserved[3];
  PagedRun first;  // the run itself: one trip to memory less
};

// A sequence, for the merge of its rows: both of its runs as they are, one trip to memory.
struct PagedSeq {
  int32_t nq;        // query tokens
  int32_t pos;       // its first token's place among the shared run's
  int32_t reserved[2];
  PagedRun own, shared;  // n_blk = 0: there is none
};

struct PagedLayout {
  size_t shares, runs, seqs, tokens, bytes;
};
inline PagedLayout paged_layout(const bass_paged_desc* d) {
  PagedLayout l;
  l.shares = sizeof(PagedHeader);
  l.runs = l.shares + sizeof(PagedShare) * kPagedShares;
  l.seqs = l.runs + sizeof(PagedRun) * 2 * (size_t)d->B;  // a shared run has two sequences at least
  l.tokens = l.seqs + sizeof(PagedSeq) * (size_t)d->B;
  l.bytes = (l.tokens + 4 * (size_t)d->B * d->kmax + 15) / 16 * 16;
  return l;
}

// Even division of `total` entries over `used` shares.
struct PagedSplit {
  int per, rem, total;
  BASS_HD int first(int w) const { return imin(w * per + imin(w, rem), total); }
  BASS_HD int owner(int x) const {
    const int big = rem * (per + 1);
    return x < big ? x / (per + 1) : rem + (x - big) / imax(per, 1);
  }
};

// Place of a unit's first row among the partial results of workgroup w.  Workgroups and units both come in the order of the list: with
// the next pair of them at least a unit's rows, or kSlotRows, are added, so that no two pairs overlap.
BASS_HD inline size_t partial_row(const PagedRun& r, int g, int kvh, int tile, int w) {
  return (size_t)r.row_base + (size_t)kvh * r.n_tok * g + (size_t)tile * r.tile_tok * g + (size_t)w * kSlotRows;
}
inline size_t partial_rows(const bass_paged_desc* d) { return 2 * (size_t)d->B * d->kmax * d->Hq + (size_t)kPagedShares * kSlotRows; }

inline int32_t paged_signature(const bass_paged_desc* d) {
  uint32_t h = 2166136261u;
  const int32_t v[] = {d->B, d->kmax, d->Hq, d->Hkv, d->D, d->page_tokens, d->max_pages, d->dtype, kPagedShares, kTileRows};
  for (int32_t x : v)
    for (int i = 0; i < 4; ++i) h = (h ^ ((uint32_t)x >> (8 * i) & 0xFFu)) * 16777619u;
  return (int32_t)(h | 1u);  // never the zero of an empty buffer
}

// The list counts in 32 bits.  Most entries of a sequence and kv head with n blocks, by the costs above:
//   own run           6 n + 56; a kv head per wavefront (n <= 16): a unit of 4 (6 n + 16) entries for at least two heads, 12 n + 32 <= 6 n + 128
//   its part of a shared run of s blocks, which its own run is shorter by: the rule for sharing asks that the tiles take less than the sequences apart, so less
//                     than 6 s, and a tile per sequence at most: 108 more; in a tile's cost in effect (tile_cost) at most 6 / 5 of that, from 480 entries per
//                     workgroup on.  (Lists with less stay below 3 * 256 * 481 entries.)
// Together less than 7.2 n + 236.
constexpr int kEntriesPerBlock = 8, kEntriesPerUnit = 256;
static_assert(kCostRows1 <= kCostRows2 && kCostRows2 <= 6 && kPadRows <= 56 && kPadHeads <= 64 && kPadTile <= 108 && 2 * kHeadBlocks <= 16, "bound of the list");
constexpr bool tile_cost_bounded(int cost) { return 5 * tile_cost(cost, 480) <= 6 * cost; }
static_assert(tile_cost_bounded(kCostTile1) && tile_cost_bounded(kCostTile2) && tile_cost_bounded(kCostTile1Int8) && tile_cost_bounded(kCostTile2Int8), "bound of the list");

// Workgroups of the merge: one for a query token and this many of its heads.
constexpr int kMergeElems = 1024;
inline int64_t merge_groups(const bass_paged_desc* d) { return (int64_t)d->B * d->kmax * ((d->Hq + (int64_t)(kMergeElems / d->D) - 1) / (kMergeElems / d->D)); }

inline int check_paged_attention(const bass_paged_desc* d) {
  const int rc = check_paged(d);
  if (rc != BASS_OK) return rc;
  if (d->B > kMaxPagedBatch || (int64_t)d->kmax * (d->Hq / d->Hkv) > 64) return BASS_ERR_UNSUPPORTED;
  const int64_t blocks = (int64_t)d->max_pages * (d->page_tokens / kBlockTokens);
  // divided, because the product may need more than 64 bits.  Partial rows, 2 B kmax Hq <= 128 B Hkv (partial_rows), are then below 2^31 too.
  if (kEntriesPerBlock * blocks + kEntriesPerUnit > ((1ll << 31) - 1) / ((int64_t)d->B * d->Hkv)) return BASS_ERR_UNSUPPORTED;
  if (!grid_fits(merge_groups(d))) return BASS_ERR_UNSUPPORTED;
  return BASS_OK;
}

}  // namespace bass
