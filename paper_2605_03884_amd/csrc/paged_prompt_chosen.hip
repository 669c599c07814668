// paged_prompt_chosen.hip — attention of many new tokens over the pages chosen for each: a token sees what stands up to its own place in the pages whose bit is set.
//
// Work: a workgroup of 4 waves takes a tile of 128 (query token, query head) pairs of one kv head, 32 a wave.  Neighbouring tokens choose much the same pages, so the
// workgroup goes through those that any of its tokens has chosen, and a page is read once for all of them.  They stand in a list in LDS, made from the tokens' bits
// for a stretch of the sequence at a time; a lane holds the place of one of the next 64 entries, and a wave has any of them by reading a lane.  Where there are few query
// tiles the list is split as well, and a second kernel joins the parts.
//
// A tile of 64 keys, two halves of 32 that lie one after the other where a page holds as many and are any two of the list otherwise:
//   staging  rows of K and V go from memory into registers and on into LDS, two tiles ahead of their use; entries are looked up a tile before that.
//   half     a wave none of whose pairs has chosen it leaves it out.  Otherwise scores S^T = K Q^T on v_mfma_f32_32x32x16 (a lane gets 16 scores of its own pair, the
//            lane 32 further on the other 16), what a pair has not chosen or does not see set to -inf, weights relative to a maximum that follows the true
//            one only when that has grown by 2^8, O^T = V^T P^T with the weights where the product wants them and V^T through the transposing read of LDS.
// Weights are rounded to the cache's type, which is what the matrix instruction takes; a second part for what that leaves off would be half as many products again.  Off by half
// a step each, they are no further off than the result itself, which is rounded to the same type (the three shapes below against 64 bits: 2.7e-4, 2.8e-4 and, bf16, 2.2e-3
// of the result, where rounding it alone gives 2.1e-4, 2.1e-4 and 1.7e-3).  Maxima, sums and results are in 32 bits.
//
// What bounds it: a wave's own chain of scores, maximum, weights and values, with two waves a SIMD (256 registers each).  8192 tokens of 32 heads and 128 dimensions, each at 16 pages of 64: 307 - 315 us; the
// choices ask for 125 GFLOP, a wave's 8 tokens together for 181 (22 pages of the 64 in sight on average, the workgroup's 32 tokens for 27), so matrix units see 0.58 PFLOP/s, busy 24 % of the
// cycles, vector instructions issuing in 37 %, waves waiting 38 % (of launches under a profiler, which take 328 - 350 us).  Not memory: with every entry naming the same page it takes as long.  Staging alone takes 155 us, lists, queries and results 48.
// 1000 tokens of 64 heads of 64 dimensions behind 32768, 64 pages of 32 each: 148 - 152 us in three parts, of which 11 join them (33 GFLOP asked for, 46 done).  38 - 150 tokens of six short
// sequences: 25 us, about 9 and 3 more for each 64 keys that follow each other; attention over all of their pages (up to 368 tokens) takes 17, as it works on the next 32 keys' scores beside these.
// Registers: two variants of 64 dimensions keep 6 and 12 of a lane's values in memory (pages of 64 tokens and more, pages of 16 and 32), one of 128 two (pages of 16 and 32), those of 256 dimensions 14 to 28;
// staging holds 16, 32 or 64 registers beside the addresses and three tiles' places.
// What was worth it: waves leave out halves and 64 keys a tile in place of 32 with all waves at all of them 376 -> 315 and 207 -> 176 (the six short ones stayed at 25), then parts 149.  And what was not: 8 waves for 256 pairs 348, two
// tiles' halves in one stream of instructions 332, the next half's scores beside these weights 333, staging between halves 321, four halves deep 733 (registers in memory), 16 pairs
// a wave on the 16x16 instruction with four waves a SIMD, which read every key and value twice as often, 2 % slower there and 13 % with 64 dimensions; priorities of waves make no difference.
#include "paged_prompt.h"

namespace qkv {
namespace {

constexpr uint32_t kWaves = 4, kThreads = kWaves * kWaveSize;
constexpr uint32_t kKeys = 64;                           // of a tile
constexpr uint32_t kListWords = 64;                      // words of a choice that are made into a list at a time, a lane each
constexpr uint32_t kListSpans = kListWords * 32u;        // a span: a page, or the 32 keys of as many pages as hold them
constexpr uint32_t kEvery = 0x8000u;                     // in the list: all tokens of the workgroup have chosen it
constexpr int32_t kNowhere = -32;                        // a half behind the list: keys that nobody sees, in unsigned numbers behind every place

// Waves a SIMD holds at once: what its 512 registers allow.
constexpr uint32_t waves_a_simd(int D) { return D == 256 ? 1u : D == 128 ? 2u : 3u; }

// Bits of pages as bits of the 32 keys that start in the page `first` names: pages of 2^shift keys, a bit each, as often as they have keys.
__device__ inline uint32_t keys_of_pages(uint32_t word, uint32_t first, uint32_t shift) {
  uint32_t x = word >> (first & 31u);
  if (shift >= 5u) return 0u - (x & 1u);
  if (shift == 4u) return (x & 1u ? 0xFFFFu : 0u) | (x & 2u ? 0xFFFF0000u : 0u);
  if (shift == 3u) {
    x &= 0xFu;
    x = (x | x << 14) & 0x00030003u;
    return ((x | x << 7) & 0x01010101u) * 0xFFu;
  }
  if (shift == 2u) {
    x &= 0xFFu;
    x = (x | x << 12) & 0x000F000Fu;
    x = (x | x << 6) & 0x03030303u;
    return ((x | x << 3) & 0x11111111u) * 0xFu;
  }
  if (shift == 1u) {
    x &= 0xFFFFu;
    x = (x | x << 8) & 0x00FF00FFu;
    x = (x | x << 4) & 0x0F0F0F0Fu;
    x = (x | x << 2) & 0x33333333u;
    return ((x | x << 1) & 0x55555555u) * 3u;
  }
  return x;
}

// RUN: tokens of a tile that surely lie in one page, one after the other: 64, 16, or 1.
template <typename T, int D, uint32_t RUN>
__global__ __launch_bounds__(kThreads, waves_a_simd(D)) void prompt_chosen_kernel(PagedPromptArgs a) {
  constexpr uint32_t kChunks = D / 8;                                  // 16-byte pieces of a row
  constexpr uint32_t kLoads = kKeys * kChunks / kThreads;              // of them a thread loads, of K and of V
  constexpr uint32_t kRowsAtOnce = kThreads / kChunks;
  constexpr uint32_t kSteps = D / 16, kSlabs = D / 32, kProducts = 2u * kSlabs;
  constexpr uint32_t kKeyPlace = kKeys * key_row(D), kValuePlace = kKeys * value_row(D);
  __shared__ __attribute__((aligned(256))) uint8_t k_place[2][kKeyPlace], v_place[2][kValuePlace];
  __shared__ uint16_t spans[kListSpans];                               // counted from the stretch's first one on, with kEvery
  __shared__ uint32_t by_some[kListWords], by_all[kListWords], list_size;
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 32u, h = lane / 32u;
  const uint32_t q_heads = a.p.kv_heads * a.rep;

  // the tile: sequence, queries
  const uint32_t kv_head = blockIdx.x % a.p.kv_heads;
  const uint32_t at = gridDim.x / a.p.kv_heads - 1u - blockIdx.x / a.p.kv_heads;      // tiles with many keys first
  uint32_t row;
  int32_t start, end, raw_length;
  if (a.p.rows < kWaveSize) {                                          // one trip to memory: lane l has row l's start and length
    const int32_t mine = a.starts[min(lane, a.p.rows)], long_is = a.p.lens[min(lane, a.p.rows - 1u)];
    const uint64_t fits = __builtin_amdgcn_ballot_w64(lane < a.p.rows && first_place((uint32_t)mine, lane, a.per) <= at);
    row = fits ? 63u - (uint32_t)__builtin_clzll(fits) : 0u;
    start = __builtin_amdgcn_readlane(mine, (int)row);
    end = __builtin_amdgcn_readlane(mine, (int)row + 1);
    raw_length = __builtin_amdgcn_readlane(long_is, (int)row);
  } else {
    row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return first_place((uint32_t)a.starts[b], b, a.per) <= at; }));
    start = a.starts[row];
    end = a.starts[row + 1u];
    raw_length = a.p.lens[row];
  }
  if (start < 0 || end < start || (uint32_t)end > a.tokens) {
    if (threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_ROW);
    return;
  }
  const uint32_t count = (uint32_t)(end - start), skip = (at - first_place((uint32_t)start, row, a.per)) * a.per;
  if (at < first_place((uint32_t)start, row, a.per) || skip >= count) return;
  const uint32_t here = min(a.per, count - skip);                      // query tokens
  const int32_t length = (int32_t)held(raw_length, a.p.row_pages, a.p.page_shift);
  const int32_t base = length - (int32_t)count + (int32_t)skip;        // place of the tile's first query
  if (base < 0 && threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_ROW);
  const int32_t reach = base + (int32_t)here;                          // keys below it are seen by somebody
  const uint32_t in_sight = reach > 0 ? ((uint32_t)(reach - 1) >> a.p.page_shift) + 1u : 0u;      // pages
  const uint32_t page_shift = a.p.page_shift, in_page = (1u << page_shift) - 1u;

  // the lane's pair
  const uint32_t pair = wave * 32u + n, token = pair / a.rep, hq = kv_head * a.rep + pair % a.rep;
  const bool live = token < here;
  const int32_t mine = live ? base + (int32_t)token : -1;
  const int32_t wave_first = base + (int32_t)(wave * 32u / a.rep);     // place of the wave's first query
  const uint64_t first_query = (uint64_t)(uint32_t)start + skip, query = first_query + token;
  const uint32_t* words = a.choice + ((live ? query : first_query) * a.p.kv_heads + kv_head) * a.words;
  typename T::x8 q[kSteps];
#pragma unroll
  for (uint32_t k = 0; k < kSteps; ++k) {
    u32x4 x = (u32x4)(0u);
    if (live) x = *reinterpret_cast<const u32x4*>(a.q + query * a.q_token_stride + (uint64_t)hq * a.q_head_stride + (k * 16u + h * 8u) * 2u);
    if (a.flip) x ^= (u32x4)(0x80008000u);
    q[k] = __builtin_bit_cast(typename T::x8, x);
  }
  f32x16 acc[kSlabs];
#pragma unroll
  for (uint32_t d = 0; d < kSlabs; ++d) acc[d] = (f32x16)(0.0f);
  float m = -INFINITY, l = 0.0f, less = 0.0f;                          // less: what is taken off in the exponent
  float scale = a.scale_log2, slack = kSlack;                          // 1 and 0 once a maximum was beyond kFar
  uint32_t special = 0u;                                               // bits, the same for all lanes: kLost, kScaled

  const uint8_t* keys = a.p.k + (uint64_t)kv_head * a.p.head_stride;
  const uint8_t* values = a.p.v + (uint64_t)kv_head * a.p.head_stride;
  const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
  const uint32_t my_row = threadIdx.x / kChunks, my_chunk = threadIdx.x % kChunks;
  u32x4 kx[kLoads], vx[kLoads];

  // The list.  A unit is what a lane of the window stands for: a tile where a page holds whole ones (RUN 64), otherwise half of one.
  constexpr uint32_t kUnitShift = RUN == 64u ? 6u : 5u, kTileUnits = RUN == 64u ? 1u : 2u;
  const uint32_t span_pages = RUN != 64u && page_shift < 5u ? 32u >> page_shift : 1u, span_mask = span_pages == 32u ? 0xFFFFFFFFu : (1u << span_pages) - 1u;
  const uint32_t span_shift = max(page_shift, 5u), units_shift = span_shift - kUnitShift;      // keys and units of a span
  uint32_t first_word = 0u, units = 0u, window_from = 0u;
  int32_t window = 0;                                                  // the lane's unit: its first key, a multiple of 32, and in the lowest bit kEvery
  const auto fill_window = [&](uint32_t from) {
    window_from = from;
    const uint32_t i = from + lane;
    if (i < units) {
      const uint32_t x = spans[i >> units_shift];
      window = (int32_t)((first_word * 32u << page_shift) + ((x & (kEvery - 1u)) << span_shift) + ((i & ((1u << units_shift) - 1u)) << kUnitShift)) | (x & kEvery ? 1 : 0);
    } else {
      window = kNowhere;
    }
  };
  // A tile as the pipeline carries it: the first keys of its halves, with kEvery's bit in the lowest.
  struct Tile {
    int32_t half[2];
  };
  const auto tile_of = [&](uint32_t i) -> Tile {
    if constexpr (RUN == 64u) {
      const int32_t x = __builtin_amdgcn_readlane(window, (int)(i - window_from));
      return Tile{{x, x + 32}};
    }
    const int one = (int)(2u * i - window_from);
    return Tile{{__builtin_amdgcn_readlane(window, one), __builtin_amdgcn_readlane(window, one + 1)}};
  };
  const auto first_key = [](int32_t half) { return half & ~1; };
  // Whether all pairs whose first query stands at `place` see all of a half.
  const auto whole = [&](int32_t half, int32_t place) { return (half & 1) != 0 && first_key(half) <= place - 31; };
  const auto make_list = [&]() {
    const uint32_t count = min(kListWords, (in_sight + 31u) / 32u - first_word);
    __syncthreads();                                                   // nobody is at the last stretch's list any more
    if (threadIdx.x < kListWords) {
      by_some[threadIdx.x] = 0u;
      by_all[threadIdx.x] = 0xFFFFFFFFu;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < here * count; i += kThreads) {
      const uint32_t of = i / count, w = i % count;
      const int32_t place = base + (int32_t)of;
      const uint32_t front = place < 0 ? 0u : ((uint32_t)place >> page_shift) + 1u, from = (first_word + w) * 32u;      // pages in the token's sight
      uint32_t x = front > from ? a.choice[((first_query + of) * a.p.kv_heads + kv_head) * a.words + first_word + w] : 0u;
      if (front > from && front - from < 32u) x &= (1u << (front - from)) - 1u;
      if (x != 0u) atomicOr(&by_some[w], x);
      if (x != 0xFFFFFFFFu) atomicAnd(&by_all[w], x);
    }
    __syncthreads();
    if (wave == 0u) {                                                  // a lane a word: a bit for each span, at its first page
      uint32_t has = lane < count ? by_some[lane] : 0u, full = by_all[lane];
      for (uint32_t by = 1; by < span_pages; by *= 2u) {
        has |= has >> by;
        full &= full >> by;
      }
      if (span_pages != 1u) has &= (uint32_t)(0xFFFFFFFFull / ((1ull << span_pages) - 1ull));
      const uint32_t mine_too = (uint32_t)__builtin_popcount(has), upto = wave_inclusive_scan(mine_too);
      uint32_t to = upto - mine_too;
      for (; has != 0u; has &= has - 1u) {
        const uint32_t bit = (uint32_t)__builtin_ctz(has);
        spans[to++] = (uint16_t)((lane * 32u + bit) / span_pages | (full >> bit & 1u ? kEvery : 0u));
      }
      if (lane == kWaveSize - 1u) list_size = upto;
    }
    __syncthreads();
    const uint32_t all = (uint32_t)__builtin_amdgcn_readfirstlane((int)list_size);
    units = all << units_shift;
    if (all != 0u) {                                                   // of the last span, those units that somebody sees
      const uint32_t last = (uint32_t)__builtin_amdgcn_readfirstlane((int)((first_word * 32u << page_shift) + ((spans[all - 1u] & (kEvery - 1u)) << span_shift)));
      const uint32_t rest = ((uint32_t)reach - last + (1u << kUnitShift) - 1u) >> kUnitShift;
      if (rest < 1u << units_shift) units -= (1u << units_shift) - rest;
    }
  };

  // A tile goes through four hands: its entries are looked up, its rows are loaded, stored to LDS, worked on.  Lane l has the entry of key l of the tile.
  const auto key_of = [&](const Tile& t, uint32_t of) -> int32_t { return first_key(of < 32u ? t.half[0] : t.half[1]) + (int32_t)(of % 32u); };
  const auto lanes_key = [&](const Tile& t) -> int32_t { return first_key(lane < 32u ? t.half[0] : t.half[1]) + (int32_t)(lane % 32u); };
  const auto seen_by_some = [&](int32_t key) {
    if (RUN == 64u || span_pages == 1u) return (uint32_t)key < (uint32_t)reach;      // a half is one page's
    const uint32_t page = (uint32_t)key >> page_shift;
    return (uint32_t)key < (uint32_t)reach && (by_some[page / 32u - first_word] >> (page % 32u) & 1u) != 0u;
  };
  const auto look_up = [&](const Tile& t) -> uint32_t { return (uint32_t)entries[min((uint32_t)lanes_key(t), (uint32_t)reach - 1u) >> page_shift]; };
  // Where the thread's rows of a tile are, in head 0: with pages of at least RUN tokens a place for each load that is the same for the wave, to which `own` is
  // added, otherwise the thread's own.  Rows that nobody sees, and those without a page (`lost`, a bit a key), are read from page 0.
  constexpr uint32_t kSpots = RUN == 64u ? 1u : kLoads;
  struct Spots {
    uint64_t at[kSpots];
  };
  const uint32_t own = my_row % RUN * (RUN == 1u ? 0u : (uint32_t)a.p.token_stride) + my_chunk * 16u;
  uint64_t lost = 0ull;
  const auto settle = [&](const Tile& t, uint32_t entry) -> Spots {
    const bool wanted = seen_by_some(lanes_key(t)), known = entry < a.p.pages;
    const uint64_t there = __builtin_amdgcn_ballot_w64(wanted && known);
    lost = __builtin_amdgcn_ballot_w64(wanted && !known);
    special |= lost != 0ull ? kLost : 0u;
    const uint32_t page = wanted && known ? entry : 0u;
    Spots to;
#pragma unroll
    for (uint32_t j = 0; j < kSpots; ++j) {
      const uint32_t of = j * kRowsAtOnce + my_row;                    // the row
      if constexpr (RUN == 1u) {
        to.at[j] = (uint64_t)(uint32_t)__shfl((int)page, (int)of) * a.p.page_stride + (uint64_t)((uint32_t)key_of(t, of) & in_page) * a.p.token_stride;
      } else {
        // any key of the run that is there names the page; rows of a run lie one after the other
        const uint32_t first = RUN == 64u ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)(of / RUN * RUN));
        const uint64_t in_run = there >> first & (RUN == 64u ? ~0ull : (1ull << (RUN % 64u)) - 1ull);
        const uint32_t number = (uint32_t)__builtin_amdgcn_readlane((int)page, (int)(first + (in_run ? (uint32_t)__builtin_ctzll(in_run) : 0u)));
        const uint32_t key = (uint32_t)key_of(t, first);
        to.at[j] = (uint64_t)number * a.p.page_stride + (key & in_page) * (uint32_t)a.p.token_stride +
                   (RUN == 16u && kRowsAtOnce < RUN ? j * kRowsAtOnce % RUN * (uint32_t)a.p.token_stride : 0u);
      }
    }
    return to;
  };
  const auto load = [&](const uint8_t* pool, const Spots& from, u32x4 (&x)[kLoads]) {
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j)
      x[j] = *reinterpret_cast<const u32x4*>(pool + from.at[RUN == 64u ? 0u : j] + (own + (RUN == 64u ? j * kRowsAtOnce * (uint32_t)a.p.token_stride : 0u)));
  };
  const auto store_keys = [&](uint32_t place) {
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(k_place[place] + (my_row + j * kRowsAtOnce) * key_row(D) + my_chunk * 16u) = kx[j];
  };
  const auto store_values = [&](const Tile& t, uint32_t place) {
    // Rows that nobody sees may hold anything: behind the sequence nothing has been written yet.
    const bool cut = (uint32_t)first_key(t.half[1]) + 31u >= (uint32_t)reach || (RUN != 64u && span_pages != 1u);
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) {
      if (cut && !seen_by_some(key_of(t, j * kRowsAtOnce + my_row))) vx[j] = (u32x4)(0u);
      *reinterpret_cast<u32x4*>(v_place[place] + (my_row + j * kRowsAtOnce) * value_row(D) + my_chunk * 16u) = vx[j];
    }
  };

  // The pieces of the work on 32 keys, in the order in which they are to be issued: reads of LDS come kAhead matrix instructions in front of their use.
  constexpr uint32_t kAhead = D == 64 ? 4u : 6u;
  static_assert(kAhead <= kSteps && kAhead <= kProducts && kProducts == kSteps);
  typename T::x8 piece[kSteps], v_piece[kProducts];
  const auto read_key = [&](const uint8_t* from, uint32_t k) { piece[k] = __builtin_bit_cast(typename T::x8, *reinterpret_cast<const u32x4*>(from + n * key_row(D) + (k * 2u + h) * 16u)); };
  const auto read_value = [&](const uint8_t* from, uint32_t k) {
    const uint8_t* p = from + (4u * h + (lane % 16u) / 4u) * value_row(D) + (lane / 16u % 2u) * 32u + (lane % 4u) * 8u;
    const u32x2 lo = read_turned(p + (k / kSlabs) * 16u * value_row(D) + (k % kSlabs) * 64u), hi = read_turned(p + ((k / kSlabs) * 16u + 8u) * value_row(D) + (k % kSlabs) * 64u);
    v_piece[k] = __builtin_bit_cast(typename T::x8, (u32x4){lo.x, lo.y, hi.x, hi.y});
  };
  typename T::x8 w[2];
  const auto weigh = [&](const f32x16& s, uint32_t first, uint32_t many) {
    float e[16], sum = 0.0f;
#pragma unroll
    for (uint32_t j = first; j < first + many; ++j) e[j] = exp2f_(__builtin_fmaf(s[j], scale, -less));
#pragma unroll
    for (uint32_t j = first; j < first + many; ++j) {
      sum = j == first ? e[j] : sum + e[j];
      w[j / 8u][j % 8u] = (typename T::one)e[j];
    }
    l += sum;
  };
  // what the lane's pair does not see of 32 keys scores -inf; `word` has the bits of their pages
  const auto mask = [&](const Tile& tile, uint32_t half, uint32_t word, f32x16& s) {
    const int32_t t = first_key(tile.half[half]);
    if constexpr (RUN != 1u) {
      // all in front of the wave's first query: 16 keys at least are one page's, and a bit that is the same for all of them is a mask of lanes
      if (special == 0u && t <= wave_first - 31) {
        const bool one = word >> ((uint32_t)t >> page_shift) % 32u & 1u, two = RUN == 64u ? one : word >> ((uint32_t)(t + 16) >> page_shift) % 32u & 1u;
        if (__builtin_amdgcn_ballot_w64(!one || !two) == 0ull) return;
#pragma unroll
        for (uint32_t j = 0; j < 16u; ++j) s[j] = (j < 8u ? one : two) ? s[j] : -INFINITY;
        return;
      }
    }
    uint32_t seen = (uint32_t)((1ull << (uint32_t)min(max(mine - t + 1, 0), 32)) - 1ull) & keys_of_pages(word, (uint32_t)t >> page_shift, page_shift);
    if (special != 0u) {
      if ((special & kLost) != 0u) {
        settle(tile, look_up(tile));
        seen &= ~(uint32_t)(lost >> (32u * half));
      }
      if ((special & kScaled) != 0u) s *= a.scale_log2;
    }
    seen >>= 4u * h;
#pragma unroll
    for (uint32_t j = 0; j < 16u; ++j) s[j] = seen >> (8u * (j / 4u) + j % 4u) & 1u ? s[j] : -INFINITY;
  };
  // m, which is -inf at first, to the largest of the scores s
  const auto follow = [&](f32x16& s) {
    float top = s[0];
#pragma unroll
    for (uint32_t j = 1; j < 16u; ++j) top = fmaxf(top, s[j]);
    const float most = max32(top) * scale;
    if (__builtin_amdgcn_ballot_w64(most > m + slack) != 0ull) {
      // a pair that sees none of these keys has a maximum of -inf, which is not far: its weights are 0 whatever is rounded
      if (__builtin_amdgcn_ballot_w64(__builtin_fabsf(most) > kFar && most != -INFINITY) != 0ull && (special & kScaled) == 0u) {
        s *= scale;
        scale = uniform(1.0f);
        slack = uniform(0.0f);
        special = (uint32_t)__builtin_amdgcn_readfirstlane((int)(special | kScaled));
      }
      const float next = fmaxf(m, most);
      const float shrink = m == -INFINITY ? 0.0f : exp2f_(m - next);
      l *= shrink;
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) acc[d] *= shrink;
      m = next;
      less = m == -INFINITY ? 0.0f : m - kLift;
    }
  };

  for (; first_word * 32u < in_sight; first_word += kListWords) {
    make_list();
    const uint32_t tiles = (units + kTileUnits - 1u) / kTileUnits;
    uint32_t i = (uint32_t)((uint64_t)tiles * blockIdx.y / a.splits);
    const uint32_t last = (uint32_t)((uint64_t)tiles * (blockIdx.y + 1u) / a.splits);
    if (i >= last) continue;
    fill_window(i * kTileUnits);
    const auto no_further = [&](uint32_t tile) { return min(tile, last - 1u); };      // what is read ahead behind the last tile is the last tile
    const auto word_of = [&](int32_t half) -> uint32_t { return words[min((uint32_t)first_key(half) >> page_shift, in_sight - 1u) / 32u]; };
    Tile tile = tile_of(i), next = tile_of(no_further(i + 1u)), then = tile_of(no_further(i + 2u));
    const uint32_t entries_ahead[2] = {look_up(tile), look_up(next)};
    uint32_t entry = look_up(then);
    uint32_t word[2] = {word_of(tile.half[0]), RUN == 64u ? 0u : word_of(tile.half[1])}, word_next[2] = {word_of(next.half[0]), RUN == 64u ? 0u : word_of(next.half[1])};
    Spots spots = settle(tile, entries_ahead[0]);
    load(keys, spots, kx);
    load(values, spots, vx);
    store_keys(0u);
    store_values(tile, 0u);
    spots = settle(next, entries_ahead[1]);
    load(keys, spots, kx);
    load(values, spots, vx);
    __syncthreads();
    for (uint32_t place = 0u;; place ^= 1u) {
      const bool more = i + 1u < last;
      const Tile now = tile;
      const uint32_t bits[2] = {word[0], RUN == 64u ? word[0] : word[1]};
      if (more) {
        // the next tile takes the place of the last one, which nobody reads any more; the one after it is asked for
        if ((i + 4u) * kTileUnits - window_from > kWaveSize) fill_window(i * kTileUnits);
        store_keys(place ^ 1u);
        store_values(next, place ^ 1u);
        spots = settle(then, entry);
        load(keys, spots, kx);
        load(values, spots, vx);
        tile = next;
        next = then;
        then = tile_of(no_further(i + 3u));
        entry = look_up(then);
        word[0] = word_next[0];
        word_next[0] = word_of(next.half[0]);
        if constexpr (RUN != 64u) {
          word[1] = word_next[1];
          word_next[1] = word_of(next.half[1]);
        }
      }
#pragma unroll
      for (uint32_t half = 0; half < 2u; ++half) {
        const int32_t t = first_key(now.half[half]);
        if ((uint32_t)t >= (uint32_t)reach || __builtin_amdgcn_ballot_w64(live && (bits[half] >> ((uint32_t)t >> page_shift) % 32u & span_mask) != 0u) == 0ull) continue;
        const uint8_t *const k_at = k_place[place] + half * 32u * key_row(D), *const v_at = v_place[place] + half * 32u * value_row(D);
        f32x16 s = (f32x16)(0.0f);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) read_key(k_at, k);
#pragma unroll
        for (uint32_t k = 0; k < kSteps; ++k) {
          if (k + kAhead < kSteps) read_key(k_at, k + kAhead);
          else read_value(v_at, k + kAhead - kSteps);
          s = T::mfma32(piece[k], q[k], s);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (!whole(now.half[half], wave_first) || special != 0u) mask(now, half, bits[half], s);
        follow(s);
        weigh(s, 0u, 8u);
#pragma unroll
        for (uint32_t k = 0; k < kProducts; ++k) {
          if (k + kAhead < kProducts) read_value(v_at, k + kAhead);
          acc[k % kSlabs] = T::mfma32(v_piece[k], w[k / kSlabs], acc[k % kSlabs]);
          if (k < kSlabs) weigh(s, 8u + k * (8u / kSlabs), 8u / kSlabs);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (!more) break;
      ++i;
      __syncthreads();
    }
  }
  if ((special & kLost) != 0u && lane == 0u) flag(a.status, QKV_STATUS_BAD_PAGE);

  // Values that are infinite or no number have spoilt their dimension for all pairs that met them, with a weight of nothing too.  Where that has happened a pair goes
  // through its keys once more: values that are numbers count with their weights, the others as they are.  Scores are the same products as before, to the bit: m and l
  // are made of those, and two sums in another order are a factor of 2^several apart where scores are beyond 2^24.
  f32x16 zero = (f32x16)(0.0f);                                        // stays that only where all are numbers
#pragma unroll
  for (uint32_t d = 0; d < kSlabs; ++d) zero += acc[d] * 0.0f;
  float zeros = 0.0f;
#pragma unroll
  for (uint32_t j = 0; j < 16u; ++j) zeros += zero[j];
  const bool spoilt = live && !(sum32(zeros) == 0.0f);
  if (__builtin_expect(__syncthreads_or(spoilt), 0)) {
    if (spoilt) {
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) acc[d] = (f32x16)(0.0f);
    }
    static_assert(kWaves * 32u * 32u * 4u <= sizeof(v_place));
    float* const weights = reinterpret_cast<float*>(v_place[0]) + wave * 1024u;      // the wave's: of 32 keys, 32 pairs each; nobody reads values there any more
    for (first_word = 0u; first_word * 32u < in_sight; first_word += kListWords) {
      make_list();
      const uint32_t tiles = (units + kTileUnits - 1u) / kTileUnits, last = (uint32_t)((uint64_t)tiles * (blockIdx.y + 1u) / a.splits);
      for (uint32_t i = (uint32_t)((uint64_t)tiles * blockIdx.y / a.splits); i < last; ++i) {
        fill_window(i * kTileUnits);
        const Tile tile = tile_of(i);
#pragma unroll 1
        for (uint32_t half = 0; half < 2u; ++half) {
          const int32_t t = first_key(tile.half[half]);
          if ((uint32_t)t >= (uint32_t)reach) continue;
          const uint32_t key = min((uint32_t)t + n, (uint32_t)reach - 1u), entry = (uint32_t)entries[key >> page_shift];      // the lane's row of K
          const uint8_t* from = keys + (uint64_t)(entry < a.p.pages ? entry : 0u) * a.p.page_stride + (uint64_t)(key & in_page) * a.p.token_stride + h * 16u;
          f32x16 s = (f32x16)(0.0f);
#pragma unroll
          for (uint32_t k = 0; k < kSteps; ++k) {
            u32x4 y = (u32x4)(0u);
            if (live) y = *reinterpret_cast<const u32x4*>(a.q + query * a.q_token_stride + (uint64_t)hq * a.q_head_stride + (k * 16u + h * 8u) * 2u);
            if (a.flip) y ^= (u32x4)(0x80008000u);
            s = T::mfma32(__builtin_bit_cast(typename T::x8, *reinterpret_cast<const u32x4*>(from + k * 32u)), __builtin_bit_cast(typename T::x8, y), s);
          }
          if ((special & kScaled) != 0u) s *= a.scale_log2;
#pragma unroll
          for (uint32_t j = 0; j < 16u; ++j) weights[(8u * (j / 4u) + 4u * h + j % 4u) * 32u + n] = (float)(typename T::one)exp2f_(__builtin_fmaf(s[j], scale, -less));
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
#pragma unroll 1
          for (uint32_t of = 0; of < 32u && (uint32_t)t + of < (uint32_t)reach; ++of) {
            const uint32_t at_key = (uint32_t)t + of, page = at_key >> page_shift, number = (uint32_t)entries[page];
            if (number >= a.p.pages) continue;
            if (!spoilt || (int32_t)at_key > mine || (words[page / 32u] >> (page % 32u) & 1u) == 0u) continue;
            const uint64_t row_at = (uint64_t)number * a.p.page_stride + (uint64_t)(at_key & in_page) * a.p.token_stride;
            const float weight = weights[of * 32u + n];
#pragma unroll
            for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
              for (uint32_t j = 0; j < 4u; ++j) {
                const typename T::x4 v = *reinterpret_cast<const typename T::x4*>(values + row_at + (d * 32u + j * 8u + h * 4u) * 2u);
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e) acc[d][4u * j + e] += __builtin_fabsf((float)v[e]) < INFINITY ? (float)v[e] * weight : (float)v[e];
              }
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // the next half's weights take these ones' place
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
  }
  if (!live) return;
  const uint64_t out_at = query * q_heads + hq;
  const float sum = sum32(l);
  if (a.splits != 1u) {
    const uint64_t slot = (uint64_t)blockIdx.y * a.tokens * q_heads + out_at;
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j)
        *reinterpret_cast<f32x4*>(a.part_o + slot * D + d * 32u + j * 8u + h * 4u) = (f32x4){acc[d][4 * j], acc[d][4 * j + 1], acc[d][4 * j + 2], acc[d][4 * j + 3]};
    if (h == 0u) *reinterpret_cast<f32x2*>(a.part_ml + slot * 2u) = (f32x2){m, sum};
  } else {
    const float share = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) {
        typename T::x4 o;
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) o[e] = (typename T::one)(acc[d][4u * j + e] * share);
        *reinterpret_cast<typename T::x4*>(a.out + (out_at * D + d * 32u + j * 8u + h * 4u) * 2u) = o;
      }
    if (a.lse && h == 0u) a.lse[out_at] = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
}

// Joins the parts of the query heads of one token, D / 4 lanes each.
constexpr uint32_t kJoinThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void prompt_chosen_join_kernel(PagedPromptArgs a) {
  constexpr uint32_t kLanes = D / 4, kAtOnce = 8;
  const uint32_t lane = threadIdx.x % kWaveSize, q_heads = a.p.kv_heads * a.rep, token = blockIdx.x;
  const uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return (uint32_t)a.starts[b] <= token; }));
  const int32_t start = a.starts[row], end = a.starts[row + 1u];
  if (start < 0 || (uint32_t)start > token || end <= (int32_t)token || (uint32_t)end > a.tokens) return;      // nobody's token has no parts
  const uint32_t at = threadIdx.x % kLanes, hq = blockIdx.y * (kJoinThreads / kLanes) + threadIdx.x / kLanes;
  if (hq >= q_heads) return;
  const uint64_t all = (uint64_t)a.tokens * q_heads, pair = (uint64_t)token * q_heads + hq;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = (f32x4)(0.0f);
  for (uint32_t s = 0; s < a.splits; s += kAtOnce) {
    f32x2 ml[kAtOnce];
    f32x4 x[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint64_t slot = min(s + k, a.splits - 1u) * all + pair;    // past the last one: the last one, without weight
      ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
      x[k] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
    }
    float top = m;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k)
      if (s + k < a.splits) top = fmaxf(top, ml[k].x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top);
    l *= keep;
    o *= keep;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      if (s + k >= a.splits) continue;
      const float take = ml[k].x == -INFINITY ? 0.0f : exp2f_(ml[k].x - top);
      l += ml[k].y * take;
      o += x[k] * take;
    }
    m = top;
  }
  keep_odd(o, a.splits, [&](uint32_t s) { return *reinterpret_cast<const f32x4*>(a.part_o + (s * all + pair) * D + at * 4u); });
  const float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
  typename T::x4 r;
#pragma unroll
  for (uint32_t e = 0; e < 4u; ++e) r[e] = (typename T::one)(o[e] * scale);
  *reinterpret_cast<typename T::x4*>(a.out + (pair * D + at * 4u) * 2u) = r;
  if (a.lse && at == 0u) a.lse[pair] = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D>
hipError_t launch_of(const PagedPromptArgs& a, hipStream_t stream) {
  const dim3 grid(places(a.tokens, a.p.rows, a.per) * a.p.kv_heads, a.splits);
  if (a.p.page_shift >= 6u) prompt_chosen_kernel<T, D, 64u><<<grid, kThreads, 0, stream>>>(a);
  else if (a.p.page_shift >= 4u) prompt_chosen_kernel<T, D, 16u><<<grid, kThreads, 0, stream>>>(a);
  else prompt_chosen_kernel<T, D, 1u><<<grid, kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1u) return e;
  const uint32_t together = kJoinThreads / (D / 4);
  prompt_chosen_join_kernel<T, D><<<dim3(a.tokens, (a.p.kv_heads * a.rep + together - 1u) / together), kJoinThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const PagedPromptArgs& a, uint32_t head_dim, hipStream_t stream) {
  if (head_dim == 64u) return launch_of<T, 64>(a, stream);
  if (head_dim == 128u) return launch_of<T, 128>(a, stream);
  return launch_of<T, 256>(a, stream);
}

}  // namespace

hipError_t launch_paged_prompt_chosen(const PagedPromptArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  return bf16 ? launch_type<BFloat>(a, head_dim, stream) : launch_type<Half>(a, head_dim, stream);
}

}  // namespace qkv
