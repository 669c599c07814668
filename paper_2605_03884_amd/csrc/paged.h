// paged.h — a cache in pages as the kernels see it, and the integer work they share: which tokens a query sees, how those
// are cut into tiles and the tiles into shares, where a sequence's queries stand in a ragged batch.
// The integer functions compile for the host too, so that a host program can go through them.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define QKV_HD __host__ __device__ inline
#else
#define QKV_HD inline
#endif

#include "../../include/qkvcard.h"

namespace qkv {

constexpr uint32_t kAttendTile = 32;         // tokens a wave of the decode kernel takes at a time
constexpr uint32_t kAttendWhole = 4;         // tiles of the longest sequence there is room for, up to which items are not cut at all
constexpr uint32_t kAttendSingle = 1024;     // tiles in all, up to which a share has one where items are cut; otherwise two at least
constexpr uint32_t kMaxRows = 65536;         // sequences of a table

// The tokens a query at the last position of `length` sees: [0, sink_end) and [begin, length).
struct Seen {
  uint32_t sink_end, begin, length;
};

QKV_HD Seen seen_by_last(uint32_t length, uint32_t window, uint32_t sinks) {
  Seen s{0u, 0u, length};
  if (window != 0u && length > window) {
    s.begin = length - window;
    s.sink_end = sinks < s.begin ? sinks : s.begin;
    if (s.sink_end == s.begin) s.sink_end = s.begin = 0u;       // nothing lies between the two
  }
  return s;
}

// Tiles of such a range: those of the sinks first, then those of the window, which start at whole tiles.  A sequence without tokens has
// one tile with nothing in it, so that somebody writes its result.
QKV_HD uint32_t sink_tiles(const Seen& s) { return (s.sink_end + kAttendTile - 1u) / kAttendTile; }
QKV_HD uint32_t seen_tiles(const Seen& s) {
  const uint32_t n = sink_tiles(s) + (s.length + kAttendTile - 1u) / kAttendTile - s.begin / kAttendTile;
  return n == 0u ? 1u : n;
}

// Tile `i` of the range: the token it starts at, and the tokens [lo, hi) that count in it.
struct TileRange {
  uint32_t first, lo, hi;
};
QKV_HD TileRange tile_range(const Seen& s, uint32_t i) {
  const uint32_t head = sink_tiles(s);
  TileRange t;
  if (i < head) {
    t.first = i * kAttendTile;
    t.lo = t.first;
    t.hi = s.sink_end < t.first + kAttendTile ? s.sink_end : t.first + kAttendTile;
  } else {
    t.first = (s.begin / kAttendTile + (i - head)) * kAttendTile;
    t.lo = s.begin > t.first ? s.begin : t.first;
    t.hi = s.length < t.first + kAttendTile ? s.length : t.first + kAttendTile;
  }
  if (t.hi < t.lo) t.hi = t.lo;
  return t;
}

// `total` tiles dealt to at most `most` shares in a row: one each up to kAttendSingle tiles, two each while that is enough, then in equal parts, the first ones one
// more than the last ones.  Few tiles end sooner apart (1500 tokens of 8 heads 11.3 us, with two a share 12.9; 8 rows of up to 120 9.9, 12.9), but parts have to be
// joined (7000 tokens 16.5, with one a share 18.1).
struct Shares {
  uint32_t shares, each, more, total;      // share i has each + (i < more) tiles
};
QKV_HD Shares deal(uint32_t total, uint32_t most) {
  if (total <= kAttendSingle && total <= most) return Shares{total, 1u, 0u, total};
  if (total <= 2u * most) return Shares{(total + 1u) / 2u, 2u, 0u, total};
  return Shares{most, total / most, total % most, total};
}
// Items that are not cut: share i has the items [i * each, (i + 1) * each).
QKV_HD uint32_t items_each(uint32_t items, uint32_t most) { return (items + most - 1u) / most; }
QKV_HD uint32_t share_begin(const Shares& s, uint32_t i) {
  const uint32_t at = i * s.each + (i < s.more ? i : s.more);
  return at < s.total ? at : s.total;
}
QKV_HD uint32_t share_of(const Shares& s, uint32_t tile) {
  if (s.more == 0u) return tile / s.each;
  const uint32_t big = s.more * (s.each + 1u);
  return tile < big ? tile / (s.each + 1u) : s.more + (tile - big) / s.each;
}

// Lengths are taken as they come from the device: below 0 counts as 0, and no length reaches past the row's entries.
QKV_HD uint32_t held(int32_t length, uint32_t row_pages, uint32_t page_shift) {
  const uint32_t most = row_pages << page_shift;
  return length < 0 ? 0u : (uint32_t)length > most ? most : (uint32_t)length;
}

// Work of the prompt kernel: query tiles of a ragged batch without a look at all sequences.  Sequence b, whose queries are
// [starts[b], starts[b + 1]), has the places starts[b] / per + b and on; that is room for ceil(n / per) tiles, since
// floor((a + n) / per) + 1 - floor(a / per) >= ceil(n / per).
QKV_HD uint32_t first_place(uint32_t start, uint32_t b, uint32_t per) { return start / per + b; }
QKV_HD uint32_t places(uint32_t tokens, uint32_t rows, uint32_t per) { return tokens / per + rows; }

// The keys that the queries at places [base, base + here) see, in tiles of `keys`: those of the sinks, [0, sink_end), are `head` tiles, the others the tiles
// `body` and on, `tiles` in all.  Nobody sees a key of [sink_end, win_lo).
struct KeyTiles {
  int32_t win_lo;
  uint32_t sink_end, head, body, tiles;
};
QKV_HD KeyTiles key_tiles_of(int32_t base, uint32_t here, int32_t window, int32_t sinks, uint32_t keys) {
  KeyTiles k;
  const int32_t reach = base + (int32_t)here;
  k.win_lo = window != 0 && base >= window ? base - window + 1 : 0;
  k.sink_end = (uint32_t)(sinks < k.win_lo ? sinks : k.win_lo);
  k.head = (k.sink_end + keys - 1u) / keys;
  k.body = (uint32_t)k.win_lo / keys;
  if (k.body < k.head) k.body = k.head;
  const uint32_t stop = reach > 0 ? ((uint32_t)reach + keys - 1u) / keys : 0u;
  k.tiles = k.head + (stop > k.body ? stop - k.body : 0u);
  return k;
}
// Parts the keys of a query tile are cut into: as many as there may be, of at least `least` keys (512 where there are few query tiles: six prompts of up to 450 keys 17.4 us, with 256 keys a part 20.3; 61 tokens
// behind 32768 take 67 - 69 with 256, 512 or 1024).
QKV_HD uint32_t prompt_splits(uint32_t keys, uint32_t most, uint32_t least = 512u) {
  const uint32_t n = keys / least;
  return n < 2u ? 1u : n < most ? n : most;
}

// One layer of a cache in pages.
struct PageLayer {
  const uint8_t *k, *v;
  uint64_t page_stride, head_stride, token_stride;       // bytes
  const int32_t* table;
  const int32_t* lens;
  uint32_t rows, row_pages, pages, page_shift, kv_heads;
};

#ifdef __HIPCC__

struct PageCache {
  uint8_t* k[QKV_INJECT_MAX_LAYERS];
  uint8_t* v[QKV_INJECT_MAX_LAYERS];
  uint64_t page_stride, head_stride, token_stride;       // bytes
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  uint32_t layers, kv_heads, head_dim, page_shift, pages, rows, row_pages;
};

struct AppendArgs {
  const uint8_t *k, *v;
  uint64_t layer_stride, head_stride, token_stride;      // bytes, of the new rows
  const int32_t* starts;                                 // or null: one token a row
  uint32_t tokens, layer_begin, layer_count;
  uint32_t first;                                        // of the tokens a launch takes
  uint32_t* status;
};

struct PagedAttendArgs {
  PageLayer p;
  const uint8_t* q;
  uint64_t q_token_stride, q_head_stride;                // bytes
  uint32_t rep, blocks;                                  // query heads per kv head, groups of 16 of them
  uint32_t window, sinks;
  float scale_log2;                                      // softmax scale times log2(e), never 0
  float nothing;                                         // a score that weighs nothing: -inf, or +inf where the scale is negative
  const float *prior_out, *prior_lse;
  float *out, *lse;
  float *part_o, *part_ml;                               // [items + most shares][heads of a block][dim], [...][2]
  uint32_t most;                                         // shares at most
  uint32_t cut;                                          // items may be cut: tiles are dealt, otherwise items
  uint32_t* status;
};

struct PagedPromptArgs {
  PageLayer p;
  const uint8_t* q;
  uint64_t q_token_stride, q_head_stride;                // bytes
  const int32_t* starts;
  uint32_t tokens, rep, per, waves;                      // per: query tokens of a tile; waves: of a workgroup, 32 (token, head) pairs each
  uint32_t window, sinks;
  float scale_log2;                                      // the softmax scale's absolute value times log2(e), above 0
  uint32_t flip;                                         // the scale is negative: q's signs are turned instead
  uint8_t* out;
  float* lse;
  float *part_o, *part_ml;                               // [splits][tokens][q heads][dim], [...][2]
  uint32_t splits, least;                                // parts of a query tile's keys at most, keys of a part at least
  uint32_t* status;
};

hipError_t launch_pages_append(const PageCache& c, const AppendArgs& a, hipStream_t stream);
hipError_t launch_pages_reserve(const PageCache& c, const int32_t* more, uint32_t* status, hipStream_t stream);
hipError_t launch_pages_fork(const PageCache& c, const int32_t* source, const int32_t* target, uint32_t n, uint32_t* status, hipStream_t stream);
hipError_t launch_pages_free(const PageCache& c, const int32_t* rows, uint32_t n, uint32_t window, uint32_t sinks, uint32_t* status, hipStream_t stream);
hipError_t launch_pages_compact(const PageCache& c, int32_t* live, int32_t* workspace, uint32_t* status, hipStream_t stream);
hipError_t launch_paged_attend(const PagedAttendArgs& a, uint32_t head_dim, bool bf16, bool may_split, hipStream_t stream);
hipError_t launch_paged_prompt(const PagedPromptArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream);

// The largest b < rows with fits(b), which holds up to some row and for none behind it; 0 if it holds nowhere.  A wave looks at 64 rows at a
// time; every lane gets the answer.
template <typename Fits>
__device__ inline uint32_t find_row(uint32_t rows, uint32_t lane, Fits fits) {
  uint32_t lo = 0u, n = rows;                            // the answer is in [lo, lo + n)
  while (n > 1u) {
    const uint32_t step = (n + 63u) / 64u;
    const uint32_t i = lane * step;
    const uint64_t hit = __builtin_amdgcn_ballot_w64(i < n && fits(lo + i));
    const uint32_t last = hit ? 63u - (uint32_t)__builtin_clzll(hit) : 0u;
    lo += last * step;
    n = n - last * step < step ? n - last * step : step;
  }
  return lo;
}

__device__ inline void flag(uint32_t* status, uint32_t bits) {
  if (status) atomicOr(status, bits);
}

#endif

}  // namespace qkv
