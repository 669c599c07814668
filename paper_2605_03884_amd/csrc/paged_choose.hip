// paged_choose.hip — which pages a query reads: scores of all pages in whole numbers, and the highest of them.
//
//     P_d = sum_r max(q_rd, 0),  N_d = sum_r min(q_rd, 0),  x = max_d (floor log2 max(P_d, -N_d) + e_d)
//     p_d = min(127, rne(P_d 2^(e_d - x + 6))),  n_d likewise;   score_j = sum_d p_d hi_jd + n_d lo_jd
//
// A score is a product of two rows of 2 D codes, so the scores of 16 pages with 16 tokens are one chain of v_mfma_i32_16x16x64_i8, which reads the digests as they lie
// in memory.  It is below 2^23 (127 * 128 * 2 * 256) and exact.
//
// Where scores fit LDS one kernel does: a workgroup takes one token, or a tile of 16 or 32 tokens of one sequence, with a kv head.  Its waves work the tokens' codes
// out into LDS, go through the pages in sight, 64 a wave at a time with the digests of 32 on their way, and put the scores into LDS.  Then a token is a wave's, or the one token
// all waves': its scores stay in registers while counting finds the last one that is chosen, and a ballot writes 64 bits of the choice at once.  Otherwise one kernel
// writes the scores of stretches of pages to the workspace and a second one picks.
//
// What bounds it: many tokens, instructions.  6583 tokens of two prompts behind up to 8000, pages of 32, 8 kv heads of 128 dimensions: 54.6 us for 58 MB (12 us of a copy) and 7.4 G
// operations; vector instructions issue in 53 % of the cycles, 373 for each of 52664 choices.  Single tokens, one chain: lengths, entries, digests, scores, picks.  48 rows of up to 8192
// tokens in pages of 16: 11.6 us for 26 MB; 131071 tokens of one row: 13.3 us for 16.8 MB, 6.2 for the scores and 7 for the picks, which are those of 8 workgroups.
// What steps were worth, these three: scores in LDS and counting (8 bits a look) in place of bisection over the workspace (a bit a look) 128.6 -> 59, 19.5 -> 12.8 and 22.4 -> 14.6 us; of it no
// branches in a wave's blocks 70 -> 57 (with 16 tokens a tile 71 where 32 have 57).  With 256 dimensions the codes of four tokens at once do not fit the registers: tiles of 32 and of 64 tokens keep 224
// bytes a lane in memory then.  A wave or two for each of many choices, in place of 16 that wait for each other: 3000 tokens of 4000 pages 347 -> 202.
#include <algorithm>

#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kScoreThreads = 256, kScoreWaves = kScoreThreads / kWaveSize;
constexpr int32_t kAbsent = INT32_MIN, kAlways = INT32_MAX;

// The query tokens of a tile: of one row, `here` of them from token `query` of the batch on, the first at place `base`.
struct QueryTile {
  uint32_t row, here, query;
  int32_t base;
};
__device__ inline QueryTile query_tile(const ChooseArgs& a, uint32_t at, uint32_t lane, bool tell) {
  QueryTile t{at, 0u, at, -1};
  if (!a.starts) {
    t.here = 1u;
    t.base = (int32_t)held(a.p.lens[at], a.p.row_pages, a.p.page_shift) - 1;
    return t;
  }
  int32_t start, end, length;
  if (a.p.rows < kWaveSize) {                                          // one trip to memory: lane l has row l's start and length
    const int32_t mine = a.starts[min(lane, a.p.rows)], long_is = a.p.lens[min(lane, a.p.rows - 1u)];
    const uint64_t fits = __builtin_amdgcn_ballot_w64(lane < a.p.rows && first_place((uint32_t)mine, lane, a.per) <= at);
    t.row = fits ? 63u - (uint32_t)__builtin_clzll(fits) : 0u;
    start = __builtin_amdgcn_readlane(mine, (int)t.row);
    end = __builtin_amdgcn_readlane(mine, (int)t.row + 1);
    length = __builtin_amdgcn_readlane(long_is, (int)t.row);
  } else {
    t.row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return first_place((uint32_t)a.starts[b], b, a.per) <= at; }));
    start = a.starts[t.row];
    end = a.starts[t.row + 1u];
    length = a.p.lens[t.row];
  }
  if (start < 0 || end < start || (uint32_t)end > a.tokens) {
    if (tell) flag(a.status, QKV_STATUS_BAD_ROW);
    return t;
  }
  const uint32_t count = (uint32_t)(end - start), first = first_place((uint32_t)start, t.row, a.per), skip = (at - first) * a.per;
  if (at < first || skip >= count) return t;
  t.here = min(a.per, count - skip);
  t.query = (uint32_t)start + skip;
  t.base = (int32_t)held(length, a.p.row_pages, a.p.page_shift) - (int32_t)count + (int32_t)skip;
  if (t.base < 0 && tell) flag(a.status, QKV_STATUS_BAD_ROW);
  return t;
}

// Extremes over a wave, in moves between lanes only; in the last lane's register, and from there the same for all.
template <typename Join>
__device__ inline int32_t over_wave(int32_t x, int32_t nothing, Join join) {
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x111, 0xF, 0xF, false));      // row_shr:1
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x112, 0xF, 0xF, false));      // row_shr:2
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x114, 0xF, 0xF, false));      // row_shr:4
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x118, 0xF, 0xF, false));      // row_shr:8
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x142, 0xA, 0xF, false));      // row_bcast:15 -> rows 1, 3
  x = join(x, __builtin_amdgcn_update_dpp(nothing, x, 0x143, 0xC, 0xF, false));      // row_bcast:31 -> rows 2, 3
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ inline int32_t wave_max(int32_t x) { return over_wave(x, INT32_MIN, [](int32_t y, int32_t z) { return max(y, z); }); }
__device__ inline int32_t wave_min(int32_t x) { return over_wave(x, INT32_MAX, [](int32_t y, int32_t z) { return min(y, z); }); }

// Bytes between the codes of a tile's tokens: 16 lanes that read one piece of theirs meet every bank once.
constexpr uint32_t code_row(int D) { return 2u * D + 16u; }

// Codes of queries to LDS, a wave: those of up to AT_ONCE tokens, `by` apart, so that their reads are on their way together.  Lane l has the channels l D / 64 and on.
template <typename T, int D, uint32_t AT_ONCE>
__device__ inline void query_codes(const ChooseArgs& a, const QueryTile& t, uint32_t head, uint32_t lane, uint32_t first, uint32_t by, int8_t* codes) {
  constexpr int kEach = D / 64, kHeads = 4;
  struct Values {
    typename T::one v[kEach];
  };
  int32_t e[kEach];
  const int8_t* exponents = a.exponents + (uint64_t)head * D + lane * kEach;
#pragma unroll
  for (int i = 0; i < kEach; ++i) e[i] = exponents[i];
  for (; first < t.here; first += AT_ONCE * by) {
    float above[AT_ONCE][kEach], below[AT_ONCE][kEach];
    const uint8_t* q[AT_ONCE];
#pragma unroll
    for (uint32_t k = 0; k < AT_ONCE; ++k) {
      q[k] = a.q + (uint64_t)(t.query + min(first + k * by, t.here - 1u)) * a.q_token_stride + (uint64_t)head * a.rep * a.q_head_stride + lane * kEach * 2u;
#pragma unroll
      for (int i = 0; i < kEach; ++i) above[k][i] = below[k][i] = 0.0f;
    }
    for (uint32_t r = 0; r < a.rep; r += kHeads) {
      Values x[AT_ONCE][kHeads];
#pragma unroll
      for (uint32_t k = 0; k < AT_ONCE; ++k)
#pragma unroll
        for (uint32_t h = 0; h < kHeads; ++h) x[k][h] = *reinterpret_cast<const Values*>(q[k] + (uint64_t)min(r + h, a.rep - 1u) * a.q_head_stride);
#pragma unroll
      for (uint32_t k = 0; k < AT_ONCE; ++k)
#pragma unroll
        for (uint32_t h = 0; h < kHeads; ++h)
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const float v = r + h < a.rep ? (float)x[k][h].v[i] : 0.0f;
            above[k][i] += fmaxf(v, 0.0f);               // no number: 0
            below[k][i] += fminf(v, 0.0f);
          }
    }
#pragma unroll
    for (uint32_t k = 0; k < AT_ONCE; ++k) {
      int32_t height = INT32_MIN;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        above[k][i] = fminf(above[k][i], 3.40282347e38f);
        below[k][i] = fmaxf(below[k][i], -3.40282347e38f);
        const float most = fmaxf(above[k][i], -below[k][i]);
        if (most > 0.0f) height = max(height, __builtin_amdgcn_frexp_expf(most) - 1 + e[i]);
      }
      height = wave_max(height);
      if (first + k * by >= t.here) break;
      int8_t* to = codes + (first + k * by) * code_row(D) + lane * kEach;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int32_t up = height == INT32_MIN ? 0 : e[i] - height + 6;
        to[i] = (int8_t)fminf(__builtin_rintf(__builtin_amdgcn_ldexpf(above[k][i], up)), 127.0f);
        to[D + i] = (int8_t)fmaxf(__builtin_rintf(__builtin_amdgcn_ldexpf(below[k][i], up)), -127.0f);
      }
    }
  }
}

// Scores of the pages [begin, end), begin a multiple of 64 and what they are put to with room up to the next one, with the codes of a tile's tokens, a workgroup of WAVES: `put(token, page, four scores of that page and on)`.
// A wave takes 64 pages at a time: a lane looks up an entry, then come the digests of all four 16, loads ahead of products.  GROUPS: 16 tokens each.
// `prepare` makes the codes, while the first digests are on their way.
template <int D, uint32_t GROUPS, uint32_t WAVES, typename Prepare, typename Put>
__device__ inline void score_pages(const ChooseArgs& a, const QueryTile& t, uint32_t head, uint32_t lane, uint32_t wave, const int8_t* codes, uint32_t begin, uint32_t end,
                                   Prepare prepare, Put put) {
  constexpr uint32_t kSteps = 2u * D / 64u, kTurns = 2u;      // of 16 pages, in flight at a time
  const uint32_t n = lane % 16u, g = lane / 16u;
  const int32_t* entries = a.p.table + (uint64_t)t.row * a.p.row_pages;
  const int8_t* digests = a.digest + (uint64_t)head * (2u * D) + g * 16u;
  const uint64_t page_bytes = (uint64_t)a.p.kv_heads * (2u * D);
  uint32_t at = begin + wave * 64u;
  uint32_t page = at + lane < end ? (uint32_t)entries[at + lane] : 0xFFFFFFFFu, next_page = 0xFFFFFFFFu;
  i32x4 x[kTurns][kSteps];
  const auto load = [&](uint32_t turn) {                               // kTurns times 16 pages of the 64 whose entries there are; page 0 for what is not there
    const uint32_t here = page < a.p.pages ? page : 0u;
#pragma unroll
    for (uint32_t i = 0; i < kTurns; ++i) {
      const int8_t* row = digests + (uint64_t)(uint32_t)__shfl((int)here, (int)((turn + i) * 16u + n)) * page_bytes;
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) x[i][k] = *reinterpret_cast<const i32x4*>(row + k * 64u);
    }
  };
  if (at < end) {
    const uint32_t next = at + WAVES * 64u + lane;
    next_page = next < end ? (uint32_t)entries[next] : 0xFFFFFFFFu;
    load(0u);
  }
  prepare();
  i32x4 q[GROUPS][kSteps];
#pragma unroll
  for (uint32_t c = 0; c < GROUPS; ++c)
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
      q[c][k] = (i32x4)(0);
      if (c * 16u + n < t.here) q[c][k] = *reinterpret_cast<const i32x4*>(codes + (c * 16u + n) * code_row(D) + k * 64u + g * 16u);
    }
  while (at < end) {
    const uint64_t there = __builtin_amdgcn_ballot_w64(page < a.p.pages);
#pragma unroll
    for (uint32_t turn = 0; turn < 4u; turn += kTurns) {
      if (turn != 0u) {
        if (at + turn * 16u >= end) break;
        load(turn);
      }
#pragma unroll
      for (uint32_t i = 0; i < kTurns; ++i)
#pragma unroll
        for (uint32_t c = 0; c < GROUPS; ++c) {
          i32x4 s = (i32x4)(0);
#pragma unroll
          for (uint32_t k = 0; k < kSteps; ++k) s = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[i][k], q[c][k], s, 0, 0, 0);
          const uint32_t known = (uint32_t)(there >> ((turn + i) * 16u + 4u * g));
#pragma unroll
          for (uint32_t j = 0; j < 4u; ++j) s[j] = known >> j & 1u ? s[j] : kAbsent;
          if (c * 16u + n < t.here) put(c * 16u + n, at + (turn + i) * 16u + 4u * g, s);
        }
    }
    at += WAVES * 64u;
    if (at >= end) break;
    page = next_page;
    const uint32_t next = at + WAVES * 64u + lane;
    next_page = next < end ? (uint32_t)entries[next] : 0xFFFFFFFFu;
    load(0u);
  }
}

// The pages of one (token, kv head) by their scores, which stand in `scores` (LDS or the workspace, with room for whole blocks of 64, one at least): those from
// `first` on and in front of the last ones; `without(j)`: kAlways or kAbsent, what a page counts as that has none.  WAVES share them, in stretches of whole blocks of
// 64, and keep up to KEEP blocks each in registers; with KEEP 0 they are read again for every look at them.
//
// The last score that is chosen is found by counting: how far scores lie below the highest one, in 256 steps that are powers of two, then the step in which the place
// `most` falls in 256 steps of its own, until all of a step are chosen or the step is a single score.  At most 3 rounds, mostly 1 or 2.  What a wave does with a block
// is written without branches: a wave that has few of them spends its time on issuing instructions.
constexpr uint32_t kOutOfRange = 16;                     // places for what is out of range, so that lanes do not wait for each other at one
template <uint32_t WAVES>
struct PickSpace {
  uint32_t counts[256 + kOutOfRange];
  int32_t shared[2][WAVES];
};
template <uint32_t WAVES, uint32_t KEEP, bool CHEAP, typename Without>
__device__ inline void pick(const ChooseArgs& a, uint32_t lane, uint32_t wave, uint32_t all, PickSpace<WAVES>& space, const int32_t* scores, uint32_t* choice, Without without) {
  const uint32_t scored = all > a.last ? all - a.last : 0u, span = scored > a.first ? scored - a.first : 0u;       // pages with scores: `first` and on
  const uint32_t blocks = (all + 63u) / 64u, each = (blocks + WAVES - 1u) / WAVES, from = min(wave * each, blocks), upto = min(from + each, blocks);
  const uint32_t last_block = max(blocks, 1u) - 1u, end = min(all, upto * 64u);
  uint32_t turn = 0u;
  const auto sync = [&]() {
    if constexpr (WAVES != 1u) {
      __syncthreads();
    } else {                                                           // a wave's own accesses of LDS are in order; nothing is waited for
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  // sums and extremes over the waves that share; the same in all lanes
  const auto together = [&](int32_t x, auto join) -> int32_t {
    if constexpr (WAVES != 1u) {
      if (lane == 0u) space.shared[turn][wave] = x;
      __syncthreads();
      x = space.shared[turn][0];
#pragma unroll
      for (uint32_t w = 1; w < WAVES; ++w) x = join(x, space.shared[turn][w]);
      turn ^= 1u;
    }
    return __builtin_amdgcn_readfirstlane(x);
  };
  int32_t low = kAlways, high = kAbsent;
  const auto settled = [&](uint32_t block, int32_t x) -> int32_t {
    const uint32_t j = block * 64u + lane;
    const bool has = j - a.first < span;
    low = min(low, has ? x : kAlways);                                 // (with a page that is not there it is far below: steps are wider then)
    high = max(high, has ? x : kAbsent);
    if constexpr (CHEAP) {
      x = has ? x : without(j);
    } else {
      if (block * 64u < a.first || block * 64u + 64u > scored) x = has ? x : without(min(j, all - 1u));
    }
    return j < end ? x : kAbsent;
  };
  int32_t keep[KEEP == 0u ? 1u : KEEP];
  if constexpr (KEEP != 0u) {
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i) keep[i] = scores[min(from + i, last_block) * 64u + lane];
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i) {
      if (CHEAP || from + i < upto) keep[i] = settled(from + i, keep[i]);
      else keep[i] = kAbsent;
    }
  } else {
    for (uint32_t i = from; i < upto; ++i) settled(i, scores[i * 64u + lane]);
  }
  low = together(wave_min(low), [](int32_t x, int32_t y) { return min(x, y); });
  high = together(wave_max(high), [](int32_t x, int32_t y) { return max(x, y); });
  // what is always chosen, no more than `most`, comes one above the highest score; what is not there is further below it than any score
  int32_t top = (high == kAbsent ? 0 : high) + 1;
  const auto each_block = [&](auto look) {
    if constexpr (KEEP != 0u) {
#pragma unroll
      for (uint32_t i = 0; i < KEEP; ++i) look(i, keep[i]);
    } else {
      for (uint32_t i = 0; from + i < upto; ++i) look(i, settled(from + i, scores[(from + i) * 64u + lane]));
    }
  };
  uint32_t left = a.most - 1u, shift = min(16u, (uint32_t)max(0, 24 - (int)__builtin_clz(((uint32_t)top - (uint32_t)low) | 1u)));
  int32_t least;                                                       // chosen: what is above, and ...
  uint32_t equal = 0xFFFFFFFFu;                                        // ... so many of those that are equal, from the front; all of them by default
  const int32_t highest = top;
  for (;;) {
    if (WAVES == 1u || wave == 0u) *reinterpret_cast<u32x4*>(&space.counts[4u * lane]) = (u32x4)(0u);
    sync();
    each_block([&](uint32_t, int32_t x) {
      const uint32_t step = ((uint32_t)top - (uint32_t)min(x, highest)) >> shift;      // what is out of range either way is beyond 255
      atomicAdd(&space.counts[min(step, 256u + lane % kOutOfRange)], 1u);
    });
    sync();
    // lane l: the steps 4 l .. 4 l + 3
    const u32x4 c = *reinterpret_cast<const u32x4*>(&space.counts[4u * lane]);
    const uint32_t four = (c.x + c.y) + (c.z + c.w), upto_here = wave_inclusive_scan(four);
    const uint64_t over = __builtin_amdgcn_ballot_w64(upto_here > left);
    if (over == 0ull) {                                                // there are no more than that
      least = kAbsent + 1;
      break;
    }
    const uint32_t who = (uint32_t)__builtin_ctzll(over);
    uint32_t step = 4u * who;
    left -= (uint32_t)__builtin_amdgcn_readlane((int)(upto_here - four), (int)who);
    uint32_t here = 0u;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
      here = (uint32_t)__builtin_amdgcn_readlane((int)c[i], (int)who);
      if (left < here) break;
      left -= here;
      ++step;
    }
    if (left + 1u == here) {                                           // the whole step
      least = top - (int32_t)((step + 1u) << shift) + 1;
      break;
    }
    top -= (int32_t)(step << shift);
    if (shift == 0u) {
      least = top;
      equal = left + 1u;
      break;
    }
    shift = shift > 8u ? shift - 8u : 0u;
    sync();                                                            // everybody has read them
  }
  uint32_t words = 0u;                                                 // lane 2 i + k: word k of block i, of 32 blocks
  const auto write = [&](uint32_t i, uint64_t bits) {
    if constexpr (KEEP != 0u) {
      words = lane == 2u * i ? (uint32_t)bits : lane == 2u * i + 1u ? (uint32_t)(bits >> 32) : words;
    } else {
      const uint32_t word = 2u * (from + i) + lane;
      if (lane < 2u && word < a.words) choice[word] = (uint32_t)(bits >> (32u * lane));
    }
  };
  if (equal == 0xFFFFFFFFu) {
    each_block([&](uint32_t i, int32_t x) { write(i, __builtin_amdgcn_ballot_w64(x >= least)); });
  } else {                                                             // equal ones are taken from the front
    uint32_t taken = 0u;
    if constexpr (WAVES != 1u) {
      uint32_t mine = 0u;
      each_block([&](uint32_t, int32_t x) { mine += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(x == least)); });
      if (lane == 0u) space.shared[turn][wave] = (int32_t)mine;
      __syncthreads();
      for (uint32_t w = 0; w < wave; ++w) taken += (uint32_t)space.shared[turn][w];
    }
    each_block([&](uint32_t i, int32_t x) {
      const uint64_t same = __builtin_amdgcn_ballot_w64(x == least);
      const uint32_t in_front = taken + (uint32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
      taken += (uint32_t)__builtin_popcountll(same);
      write(i, __builtin_amdgcn_ballot_w64(x > least || (x == least && in_front < equal)));
    });
  }
  if constexpr (KEEP != 0u) {
    static_assert(KEEP <= 32u);
    if (lane < 2u * (upto - from) && 2u * from + lane < a.words) choice[2u * from + lane] = words;
  }
  for (uint32_t word = 2u * blocks + wave * kWaveSize + lane; word < a.words; word += WAVES * kWaveSize) choice[word] = 0u;
}

// Pages in sight of a place.
__device__ inline uint32_t in_sight(const ChooseArgs& a, int32_t place) { return place < 0 ? 0u : ((uint32_t)place >> a.p.page_shift) + 1u; }

// One kernel for a tile of up to 16 GROUPS tokens of a kv head, where their scores fit LDS: tokens are taken by a wave each, or (ONE: a tile is one token) by all.
template <typename T, int D, uint32_t GROUPS, uint32_t KEEP, bool ONE, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * kWaveSize) void choose_tile_kernel(ChooseArgs a) {
  constexpr uint32_t kTileThreads = WAVES * kWaveSize, kTileWaves = WAVES;
  constexpr uint32_t kTokens = ONE ? 1u : GROUPS * 16u;
  __shared__ __attribute__((aligned(16))) int8_t codes[kTokens * code_row(D)];
  __shared__ __attribute__((aligned(16))) PickSpace<ONE ? kTileWaves : 1u> space[ONE ? 1u : kTileWaves];
  // four words between the tokens, so that 16 of them with four scores each meet every bank once
  constexpr uint32_t kNext = KEEP * kWaveSize * (ONE ? kTileWaves : 1u) + 4u;
  __shared__ __attribute__((aligned(16))) int32_t scores[kTokens * kNext];
  __shared__ int32_t without[kNext];                                   // what a page counts as that has no score
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t tile = blockIdx.x / a.p.kv_heads, head = blockIdx.x % a.p.kv_heads;
  const QueryTile t = query_tile(a, tile, lane, head == 0u && threadIdx.x == 0u);
  if (t.here == 0u) return;
  const uint32_t all = in_sight(a, t.base + (int32_t)t.here - 1), begin = a.first & ~63u, end = all > a.last ? all - a.last : 0u;
  const int32_t* entries = a.p.table + (uint64_t)t.row * a.p.row_pages;
  for (uint32_t j = threadIdx.x; j < kNext; j += kTileThreads) without[j] = j < all && (uint32_t)entries[min(j, a.p.row_pages - 1u)] < a.p.pages ? kAlways : kAbsent;
  score_pages<D, GROUPS, kTileWaves>(
      a, t, head, lane, wave, codes, begin, end,
      [&]() {
        if (begin < end) query_codes<T, D, ONE ? 1u : kTokens / WAVES>(a, t, head, lane, wave, kTileWaves, codes);
        __syncthreads();
      },
      [&](uint32_t token, uint32_t j, i32x4 s) { *reinterpret_cast<i32x4*>(scores + token * kNext + j) = s; });
  __syncthreads();
  for (uint32_t token = ONE ? 0u : wave; token < t.here; token += kTileWaves)
    pick<ONE ? kTileWaves : 1u, KEEP, true>(a, lane, ONE ? wave : 0u, in_sight(a, t.base + (int32_t)token), space[ONE ? 0u : wave], scores + token * kNext,
                                      a.choice + ((uint64_t)(t.query + token) * a.p.kv_heads + head) * a.words, [&](uint32_t j) { return without[j]; });
}

// Two kernels where there are few tiles, whose pages are scored in stretches, or where scores do not fit LDS: they go through the workspace.
template <typename T, int D, uint32_t GROUPS>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ChooseArgs a, uint32_t chunk) {
  __shared__ __attribute__((aligned(16))) int8_t codes[GROUPS * 16u * code_row(D)];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t tile = blockIdx.x / a.p.kv_heads, head = blockIdx.x % a.p.kv_heads;
  const QueryTile t = query_tile(a, a.first_tile + tile, lane, false);
  if (t.here == 0u) return;
  const uint32_t all = in_sight(a, t.base + (int32_t)t.here - 1);
  const uint32_t begin = max(blockIdx.y * chunk, a.first & ~63u), end = min((blockIdx.y + 1u) * chunk, all > a.last ? all - a.last : 0u);
  if (begin >= end) return;                                            // what has no score is chosen anyway
  int32_t* scores = a.scores + (((uint64_t)tile * a.per) * a.p.kv_heads + head) * a.stride;
  const uint64_t next_token = (uint64_t)a.p.kv_heads * a.stride;
  score_pages<D, GROUPS, kScoreWaves>(
      a, t, head, lane, wave, codes, begin, end,
      [&]() {
        query_codes<T, D, GROUPS == 1u ? 1u : 4u>(a, t, head, lane, wave, kScoreWaves, codes);
        __syncthreads();
      },
      [&](uint32_t token, uint32_t j, i32x4 s) { *reinterpret_cast<i32x4*>(scores + token * next_token + j) = s; });
}

template <uint32_t WAVES, uint32_t KEEP>
__global__ __launch_bounds__(WAVES * kWaveSize) void choose_kernel(ChooseArgs a) {
  __shared__ __attribute__((aligned(16))) PickSpace<WAVES> space;
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t pairs = a.per * a.p.kv_heads, tile = blockIdx.x / pairs, in_tile = blockIdx.x % pairs;
  const uint32_t token = in_tile / a.p.kv_heads, head = in_tile % a.p.kv_heads;
  const QueryTile t = query_tile(a, a.first_tile + tile, lane, in_tile == 0u && threadIdx.x == 0u);
  if (token >= t.here) return;
  const int32_t* entries = a.p.table + (uint64_t)t.row * a.p.row_pages;
  pick<WAVES, KEEP, false>(a, lane, wave, in_sight(a, t.base + (int32_t)token), space, a.scores + (((uint64_t)tile * a.per + token) * a.p.kv_heads + head) * a.stride,
                         a.choice + ((uint64_t)(t.query + token) * a.p.kv_heads + head) * a.words, [&](uint32_t j) { return (uint32_t)entries[j] < a.p.pages ? kAlways : kAbsent; });
}

template <uint32_t WAVES, uint32_t KEEP>
hipError_t launch_pick_of(const ChooseArgs& a, uint32_t units, hipStream_t stream) {
  choose_kernel<WAVES, KEEP><<<units, WAVES * kWaveSize, 0, stream>>>(a);
  return hipGetLastError();
}
// Blocks of 64 pages a wave keeps: those it has not are looked at too (8193 pages of one token: 5.9 us with 9, 7.6 with 16).  Where there are many (token, kv head)
// pairs each has as few waves as can keep its scores: less is waited for.
hipError_t launch_pick(const ChooseArgs& a, uint32_t units, hipStream_t stream) {
  const uint32_t blocks = a.stride / 64u;
  if (units >= 2048u && blocks <= 256u) {
    if (blocks <= 16u) return launch_pick_of<1u, 16u>(a, units, stream);
    if (blocks <= 24u) return launch_pick_of<1u, 24u>(a, units, stream);
    if (blocks <= 32u) return launch_pick_of<2u, 16u>(a, units, stream);
    if (blocks <= 48u) return launch_pick_of<2u, 24u>(a, units, stream);
    if (blocks <= 64u) return launch_pick_of<2u, 32u>(a, units, stream);
    if (blocks <= 96u) return launch_pick_of<4u, 24u>(a, units, stream);
    if (blocks <= 128u) return launch_pick_of<4u, 32u>(a, units, stream);
    if (blocks <= 192u) return launch_pick_of<8u, 24u>(a, units, stream);
    return launch_pick_of<8u, 32u>(a, units, stream);
  }
  if (blocks <= 64u) return launch_pick_of<16u, 4u>(a, units, stream);
  if (blocks <= 144u) return launch_pick_of<16u, 9u>(a, units, stream);
  if (blocks <= 256u) return launch_pick_of<16u, 16u>(a, units, stream);
  return launch_pick_of<16u, 0u>(a, units, stream);
}

template <typename T, int D, uint32_t GROUPS, uint32_t KEEP, bool ONE, uint32_t WAVES>
void launch_tile(const ChooseArgs& a, hipStream_t stream) {
  choose_tile_kernel<T, D, GROUPS, KEEP, ONE, WAVES><<<a.tiles * a.p.kv_heads, WAVES * kWaveSize, 0, stream>>>(a);
}
// Waves of a workgroup and blocks of 64 pages each of them keeps: 2048 pages for a token that all waves share, 384 for 32 tokens, up to 1536 for 16.  16 waves, a token each, where
// only one workgroup fits a CU or there are no more than two for each (120 tokens of 700 pages 12.7 us, with 8 waves 14.5; 6000 tokens 87, with 8 71).
template <typename T, int D, uint32_t GROUPS, bool ONE>
hipError_t launch_tiles(const ChooseArgs& a, hipStream_t stream) {
  if constexpr (ONE) {
    launch_tile<T, D, GROUPS, 4u, ONE, 8u>(a, stream);
  } else if constexpr (GROUPS == 2u) {
    launch_tile<T, D, GROUPS, 6u, ONE, 8u>(a, stream);
  } else {
    if (a.stride > 1024u) launch_tile<T, D, GROUPS, 24u, ONE, 16u>(a, stream);
    else if (a.stride > 768u) launch_tile<T, D, GROUPS, 16u, ONE, 16u>(a, stream);
    else if (a.tiles * a.p.kv_heads <= 512u) launch_tile<T, D, GROUPS, 12u, ONE, 16u>(a, stream);
    else launch_tile<T, D, GROUPS, 12u, ONE, 8u>(a, stream);
  }
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_choose_of(const ChooseArgs& given, hipStream_t stream) {
  ChooseArgs a = given;
  if (!a.scores) return !a.starts ? launch_tiles<T, D, 1u, true>(a, stream) : a.per == 16u ? launch_tiles<T, D, 1u, false>(a, stream) : launch_tiles<T, D, 2u, false>(a, stream);
  const uint32_t all = a.starts ? places(a.tokens, a.p.rows, a.per) : a.p.rows, at_once = a.tiles;
  for (a.first_tile = 0u; a.first_tile < all; a.first_tile += at_once) {
    a.tiles = std::min(at_once, all - a.first_tile);
    // Few tiles: their pages in stretches, until there are four workgroups to a CU, of 64 pages at least (131071 tokens in pages of 16, 8 kv heads: 4.8 us, with two 5.7).
    const uint32_t groups = a.tiles * a.p.kv_heads, pages = (a.p.row_pages + 63u) / 64u;
    const uint32_t cuts = std::min(pages, groups >= 1024u ? 1u : (1023u + groups) / groups), chunk = (pages + cuts - 1u) / cuts * 64u;
    const dim3 grid(groups, (a.p.row_pages + chunk - 1u) / chunk);
    if (!a.starts || a.per == 16u) score_kernel<T, D, 1u><<<grid, kScoreThreads, 0, stream>>>(a, chunk);
    else score_kernel<T, D, 4u><<<grid, kScoreThreads, 0, stream>>>(a, chunk);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t units = a.tiles * a.per * a.p.kv_heads;
    e = launch_pick(a, units, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_paged_choose(const ChooseArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  if (head_dim == 64u) return bf16 ? launch_choose_of<BFloat, 64>(a, stream) : launch_choose_of<Half, 64>(a, stream);
  if (head_dim == 128u) return bf16 ? launch_choose_of<BFloat, 128>(a, stream) : launch_choose_of<Half, 128>(a, stream);
  return bf16 ? launch_choose_of<BFloat, 256>(a, stream) : launch_choose_of<Half, 256>(a, stream);
}

}  // namespace qkv
