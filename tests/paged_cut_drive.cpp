// Goes through the integer work of paged.h on the host: every share of every batch reads tiles that exist, all tiles are dealt once, the tokens
// that count are those a query sees, parts have slots of their own, and every query tile of a ragged batch has a place.
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>

#include "../paper_2605_03884_amd/csrc/paged.h"

using namespace qkv;

static uint32_t state = 12345u;
static uint32_t draw(uint32_t below) {
  state = state * 1664525u + 1013904223u;
  return (uint32_t)(((uint64_t)state * below) >> 32);
}
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static int ranges() {
  for (int round = 0; round < 4000; ++round) {
    const uint32_t length = draw(round % 3 ? 300 : 5), window = draw(4) ? draw(320) : 0u, sinks = window ? draw(round % 5 ? 70 : 500) : 0u;
    const Seen s = seen_by_last(length, window, sinks);
    std::vector<int> count(length, 0);
    const uint32_t tiles = seen_tiles(s);
    CHECK(tiles >= 1u && tiles <= (length + kAttendTile - 1u) / kAttendTile + 2u);
    for (uint32_t i = 0; i < tiles; ++i) {
      const TileRange t = tile_range(s, i);
      CHECK(t.first % kAttendTile == 0u && t.lo >= t.first && t.hi <= t.first + kAttendTile && t.hi >= t.lo);
      CHECK(t.lo == t.hi || t.hi <= length);
      for (uint32_t k = t.lo; k < t.hi; ++k) ++count[k];
    }
    for (uint32_t k = 0; k < length; ++k) {
      const bool seen = window == 0u || (int64_t)k > (int64_t)length - 1 - window || k < sinks;
      CHECK(count[k] == (seen ? 1 : 0));
    }
  }
  CHECK(held(-5, 7, 4) == 0u && held(200, 7, 4) == 112u && held(111, 7, 4) == 111u && held(0x7FFFFFFF, 1, 0) == 1u);
  return 0;
}

static int deals() {
  for (int round = 0; round < 4000; ++round) {
    const uint32_t items = 1u + draw(40), most = 1u + draw(round % 2 ? 64 : 4096);
    std::vector<uint32_t> tiles(items);
    uint32_t total = 0u;
    for (auto& t : tiles) total += t = 1u + draw(round % 4 ? 9 : 300);
    const Shares s = deal(total, most);
    CHECK(s.shares >= 1u && s.shares <= most && share_begin(s, 0) == 0u && share_begin(s, s.shares) == total);
    std::set<uint32_t> slots;
    uint32_t item = 0u, in_item = 0u;
    for (uint32_t i = 0; i < s.shares; ++i) {
      const uint32_t begin = share_begin(s, i), end = share_begin(s, i + 1u);
      CHECK(end > begin || total < s.shares);
      for (uint32_t at = begin; at < end; ++at) CHECK(share_of(s, at) == i);
      uint32_t at = begin;
      while (at < end) {
        const uint32_t upto = in_item + (end - at) < tiles[item] ? in_item + (end - at) : tiles[item];
        if (!(in_item == 0u && upto == tiles[item])) {
          CHECK(item + i < items + most);
          CHECK(slots.insert(item + i).second);
        }
        at += upto - in_item;
        in_item = upto;
        if (in_item == tiles[item]) { ++item; in_item = 0u; }
      }
    }
    CHECK(item == items);
    const uint32_t each = items_each(items, most);          // items that are not cut: every one in one of `most` shares
    CHECK(each >= 1u && (uint64_t)each * most >= items && each * ((items + each - 1u) / each) >= items && (items + each - 1u) / each <= most);
  }
  return 0;
}

static int query_places() {
  for (int round = 0; round < 4000; ++round) {
    const uint32_t rows = 1u + draw(30), per = 1u + draw(130);
    std::vector<uint32_t> starts(rows + 1, 0u);
    for (uint32_t b = 0; b < rows; ++b) starts[b + 1] = starts[b] + (draw(3) ? draw(round % 2 ? 400 : 3) : 0u);
    const uint32_t all = places(starts[rows], rows, per);
    std::set<std::pair<uint32_t, uint32_t>> done;
    for (uint32_t at = 0; at < all; ++at) {
      uint32_t b = 0u;
      while (b + 1u < rows && first_place(starts[b + 1], b + 1u, per) <= at) ++b;
      const uint32_t count = starts[b + 1] - starts[b], skip = (at - first_place(starts[b], b, per)) * per;
      if (skip >= count) continue;
      CHECK(done.insert({b, skip}).second);
    }
    for (uint32_t b = 0; b < rows; ++b)
      for (uint32_t skip = 0; skip < starts[b + 1] - starts[b]; skip += per) CHECK(done.count({b, skip}) == 1u);
  }
  return 0;
}

static int keys_of_queries() {
  for (int round = 0; round < 4000; ++round) {
    const int32_t base = (int32_t)draw(500) - (round % 7 ? 0 : 40), window = draw(3) ? (int32_t)draw(300) + 1 : 0, sinks = window ? (int32_t)draw(round % 5 ? 70 : 600) : 0;
    const uint32_t here = 1u + draw(130), keys = draw(2) ? 32u : 64u;
    const int32_t reach = base + (int32_t)here;
    const KeyTiles k = key_tiles_of(base, here, window, sinks, keys);
    std::vector<int> count(reach > 0 ? reach : 0, 0);
    for (uint32_t i = 0; i < k.tiles; ++i) {
      const uint32_t t = (i < k.head ? i : k.body + (i - k.head)) * keys;
      CHECK(reach > 0 && t < (uint32_t)reach);
      for (uint32_t j = t; j < t + keys && j < (uint32_t)reach; ++j) ++count[j];
    }
    for (int32_t t = 0; t < reach; ++t) {
      bool seen = false;
      for (int32_t p = base; p < reach; ++p) seen = seen || (p >= 0 && t <= p && (window == 0 || t > p - window || t < sinks));
      CHECK(count[t] <= 1 && (!seen || count[t] == 1));
      CHECK(!seen || t >= k.win_lo || t < (int32_t)k.sink_end);
    }
    CHECK(prompt_splits(k.tiles * keys, 7u) >= 1u && prompt_splits(k.tiles * keys, 7u) <= (k.tiles > 1u ? k.tiles : 1u));
  }
  return 0;
}

int main() {
  if (ranges() || deals() || query_places() || keys_of_queries()) return 1;
  std::printf("ok\n");
  return 0;
}
