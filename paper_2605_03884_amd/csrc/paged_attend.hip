// paged_attend.hip — attention of one new token of every sequence over its pages, in one pass over what the token sees.
//
//     s_t = scale * <q, K_t>,   out = sum_t softmax(s)_t V_t,   lse = log sum_t exp s_t,   t in [0, sinks) and (p - window, p], p = length - 1
//
// Work: an item is a (sequence, kv head, group of up to 16 query heads); its tokens are cut into tiles of 32.  All items' tiles stand in
// one row and are dealt to the waves in equal shares, whatever the lengths: a wave reads the lengths, finds its share, and goes through
// the tiles with a running maximum m, sum l and sum of p.V.  An item that lies within one share is finished there; parts of
// an item go to a workspace and are joined by a second kernel.
//
// A tile, one wave (lane = 16 g + n):
//   scores   S^T = K Q^T on v_mfma_f32_16x16x32: a lane's operand of K is 8 dimensions of one token, as they lie in memory, so K goes from
//            memory straight into the operand; the result gives lane (g, n) the scores of tokens 4 g .. 4 g + 3 (and 16 more on) with head n.
//   softmax  over the lane's 8 scores and, for the maximum, the four lanes with the same n.
//   values   O^T = V^T P^T: the weights are already where the product wants them (a lane's 8 tokens, in an order of the tokens that V
//            follows); V^T wants 4 tokens of one dimension in a lane, which the transposing read of LDS gives.
//            Rows of V stand in LDS with their 32-byte pieces exchanged by token, so that neither side meets a bank twice.
// The sum of a head that sees anything is at least 1, so the hardware's reciprocal and logarithm, which know no subnormals, serve (1 step each).
// The weights are held to 22 bits (fp16: high part and remainder; bf16, 8 bits each, high part and two remainders, 24 bits), in fp16 scaled by 2^15: those
// below 2^-18 of the largest lose bits, and are off by 2^-40 of it at most, 2^-23 over 131072 of them.  Maxima, sums and results are in 32 bits.
//
// What bounds it: memory, and the chain lengths - entries - K, V - two tiles where little is read.  48 rows of up to 8192 tokens, 8 kv heads of 128 dimensions: 152 us, 146 of
// them here (5.8 TB/s; reads alone reach 6.9), 131071 tokens of one row 92 - 96 with 84 here (6.4 TB/s); 37 tokens 6.4 - 8.  Loads that pass the
// caches by: 175 -> 152 and 106 -> 97, K and V are read once and rows that share pages are read at the same time.  The next tile's loads fill the registers of this
// one's as they get free; three waves a SIMD in place of two would leave 24 registers of them in memory.
#include <algorithm>

#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr uint32_t kAttendThreads = 256;
constexpr uint32_t kAttendWaves = kAttendThreads / kWaveSize;

__device__ inline uint32_t sum64(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readlane((int)wave_inclusive_scan(x), 63);
}

__device__ inline uint32_t row_length(const PagedAttendArgs& a, uint32_t row) { return held(a.p.lens[row], a.p.row_pages, a.p.page_shift); }

// The rows' tiles: lane l has row l's length, of the first 64 rows, and (one query head group of one kv head) its tiles; `total` is of all rows.
// With up to 64 rows nothing more has to be read to find a share.
struct Lengths {
  uint32_t length, tiles, total;
};
__device__ inline Lengths read_lengths(const PagedAttendArgs& a, uint32_t lane) {
  Lengths n;
  n.length = lane < a.p.rows ? row_length(a, lane) : 0u;
  n.tiles = lane < a.p.rows ? seen_tiles(seen_by_last(n.length, a.window, a.sinks)) : 0u;
  uint32_t sum = n.tiles;
  for (uint32_t row = lane + kWaveSize; row < a.p.rows; row += kWaveSize) sum += seen_tiles(seen_by_last(row_length(a, row), a.window, a.sinks));
  n.total = sum64(sum);
  return n;
}

// The row that tile `at` of all items falls into, the tiles in front of that row, and its length.  `inner`: items of a row.
__device__ inline uint32_t row_of_tile(const PagedAttendArgs& a, const Lengths& n, uint32_t lane, uint32_t inner, uint32_t at, uint32_t& before, uint32_t& length) {
  before = 0u;
  for (uint32_t base = 0;; base += kWaveSize) {
    const uint32_t row = base + lane;
    uint32_t here = n.length, mine = n.tiles;
    if (base != 0u) {
      here = row < a.p.rows ? row_length(a, row) : 0u;
      mine = row < a.p.rows ? seen_tiles(seen_by_last(here, a.window, a.sinks)) : 0u;
    }
    mine *= inner;
    const uint32_t upto = before + wave_inclusive_scan(mine);
    const uint64_t over = __builtin_amdgcn_ballot_w64(upto > at);
    if (over != 0ull || base + kWaveSize >= a.p.rows) {
      const uint32_t who = over ? (uint32_t)__builtin_ctzll(over) : (a.p.rows - 1u) % kWaveSize;
      before = (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), (int)who);
      length = (uint32_t)__builtin_amdgcn_readlane((int)here, (int)who);
      return base + who;
    }
    before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
}

// RUN: tokens of a tile that surely lie in one page, one after the other: 32, or 1 where pages are smaller.
// The entry that lane l needs of a tile's pages: that of token l % 32, or where a page holds whole tiles the tile's.
template <uint32_t RUN>
__device__ inline uint32_t look_up(const PagedAttendArgs& a, uint32_t row, const TileRange& t, uint32_t lane) {
  const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
  if constexpr (RUN == 32u) return t.lo < t.hi ? (uint32_t)entries[t.first >> a.p.page_shift] : 0u;
  const uint32_t token = t.first + lane % kAttendTile;
  return token >= t.lo && token < t.hi ? (uint32_t)entries[token >> a.p.page_shift] : 0u;
}

// A tile whose entries have arrived: its tokens that count (a bit each), and the pages to read, which exist even where a token does not count.
struct Tile {
  uint32_t first, page, counted;
};
template <uint32_t RUN>
__device__ inline Tile settle(const PagedAttendArgs& a, const TileRange& t, uint32_t entry, uint32_t lane) {
  const uint32_t token = t.first + lane % kAttendTile;
  const bool inside = token >= t.lo && token < t.hi, known = entry < a.p.pages;
  Tile tile;
  tile.first = t.first;
  tile.counted = (uint32_t)__builtin_amdgcn_ballot_w64(inside && known);
  if ((uint32_t)__builtin_amdgcn_ballot_w64(inside && !known) != 0u && lane == 0u) flag(a.status, QKV_STATUS_BAD_PAGE);
  tile.page = known ? entry : 0u;
  return tile;
}
// Where the rows of a tile's tokens are read from, 16 bytes at a time: from a place that is the same for all lanes and 32 bits of a lane's own, or an address
// a lane.
template <uint32_t RUN>
struct RowSource {
  const uint8_t* base;
  __device__ inline RowSource(const PagedAttendArgs& a, const uint8_t* pool, const Tile& t) : base(pool) {
    if constexpr (RUN == 32u)
      base += (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)t.page) * a.p.page_stride +
              (uint64_t)(t.first & ((1u << a.p.page_shift) - 1u)) * a.p.token_stride;
  }
  __device__ inline const uint8_t* row(const PagedAttendArgs& a, const Tile& t, uint32_t of, uint32_t piece) const {
    if constexpr (RUN == 32u) return base + (of * (uint32_t)a.p.token_stride + piece);
    const uint32_t page = (uint32_t)__shfl((int)t.page, (int)of);
    return base + (uint64_t)page * a.p.page_stride + (uint64_t)((t.first + of) & ((1u << a.p.page_shift) - 1u)) * a.p.token_stride + piece;
  }
};

template <typename T, int D, uint32_t RUN>
__global__ __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) void attend_kernel(PagedAttendArgs a) {
  constexpr uint32_t kSteps = D / 32;                    // MFMAs along the head dimension
  constexpr uint32_t kSlabs = D / 16;                    // of 16 dimensions of the result
  constexpr uint32_t kLoads = kAttendTile * D / 8 / kWaveSize;         // 16-byte loads of V in a lane
  constexpr uint32_t kRowLanes = D / 8;                  // lanes that read one row of V
  constexpr uint32_t kRowsAtOnce = kWaveSize / kRowLanes;
  __shared__ __attribute__((aligned(256))) uint8_t lds[kAttendWaves][kAttendTile * D * 2];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 16u, g = lane / 16u;
  const uint32_t inner_count = a.p.kv_heads * a.blocks, q_heads = a.p.kv_heads * a.rep;
  const uint32_t share = blockIdx.x * kAttendWaves + wave;
  uint32_t row, inner, tile = 0u, length, at = 0u, end = 0xFFFFFFFFu, left = 0xFFFFFFFFu;       // left: items, where they are not cut
  if (a.cut) {
    const Lengths lengths = read_lengths(a, lane);
    const Shares shares = deal(lengths.total * inner_count, a.most);
    if (share >= shares.shares) return;
    at = share_begin(shares, share);
    end = share_begin(shares, share + 1u);
    uint32_t before;
    row = row_of_tile(a, lengths, lane, inner_count, at, before, length);
    const uint32_t tiles = seen_tiles(seen_by_last(length, a.window, a.sinks));
    // the item of the row, by counting those that end in front of `at`: a division took longer
    inner = 0u;
    for (uint32_t base = 0; base < inner_count; base += kWaveSize) {
      const uint64_t ended = __builtin_amdgcn_ballot_w64(base + lane < inner_count && before + (base + lane + 1u) * tiles <= at);
      inner += (uint32_t)__builtin_popcountll(ended);
      if (ended != ~0ull) break;
    }
    tile = at - before - inner * tiles;
  } else {
    const uint32_t items = a.p.rows * inner_count, each = items_each(items, a.most), item = share * each;
    if (item >= items) return;
    left = min(each, items - item);
    row = item / inner_count;
    inner = item % inner_count;
    length = row_length(a, row);
  }
  Seen seen = seen_by_last(length, a.window, a.sinks);
  uint32_t tiles = seen_tiles(seen);
  uint8_t* mine = lds[wave];

  for (;;) {
    // one item, or what of it falls into this share
    const uint32_t head = a.blocks == 1u ? inner : inner / a.blocks, block = a.blocks == 1u ? 0u : inner % a.blocks;
    const uint32_t heads = min(16u, a.rep - block * 16u);
    const uint32_t from = tile, upto = min(tiles, tile + (end - at));
    const uint32_t hq = head * a.rep + block * 16u + n;                // this lane's query head, if n < heads
    const uint8_t* keys = a.p.k + (uint64_t)head * a.p.head_stride;
    const uint8_t* values = a.p.v + (uint64_t)head * a.p.head_stride;
    u32x4 kx[2][kSteps], vx[kLoads];
    const auto load_keys = [&](const Tile& t) {
      const RowSource<RUN> from(a, keys, t);
#pragma unroll
      for (uint32_t h = 0; h < 2u; ++h) {
        const uint8_t* p = from.row(a, t, h * 16u + n, g * 16u);
#pragma unroll
        for (uint32_t k = 0; k < kSteps; ++k) kx[h][k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + k * 64u));
      }
    };
    const auto load_values = [&](const Tile& t) {
      const RowSource<RUN> from(a, values, t);
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) vx[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from.row(a, t, j * kRowsAtOnce + lane / kRowLanes, (lane % kRowLanes) * 16u)));
    };
    TileRange range = tile_range(seen, from);
    uint32_t entry = look_up<RUN>(a, row, range, lane);
    typename T::x8 q[kSteps];
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
      u32x4 x = (u32x4)(0u);
      if (n < heads) x = *reinterpret_cast<const u32x4*>(a.q + (uint64_t)row * a.q_token_stride + (uint64_t)hq * a.q_head_stride + (k * 32u + g * 8u) * 2u);
      q[k] = __builtin_bit_cast(typename T::x8, x);
    }
    Tile now = settle<RUN>(a, range, entry, lane);
    load_keys(now);
    load_values(now);
    if (from + 1u < upto) {
      range = tile_range(seen, from + 1u);
      entry = look_up<RUN>(a, row, range, lane);
    }
    f32x4 acc[kSlabs];
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d) acc[d] = (f32x4)(0.0f);
    float m = -INFINITY, l = 0.0f;

    for (uint32_t i = from; i < upto; ++i) {
      const uint32_t counted = now.counted;
      f32x4 s[2] = {(f32x4)(0.0f), (f32x4)(0.0f)};
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) {
        s[0] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[0][k]), q[k], s[0]);
        s[1] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[1][k]), q[k], s[1]);
      }
      // the registers of K are free: the next tile's keys are on their way while this one's weights are worked out
      if (i + 1u < upto) {
        now = settle<RUN>(a, range, entry, lane);
        load_keys(now);
        if (i + 2u < upto) {
          range = tile_range(seen, i + 2u);
          entry = look_up<RUN>(a, row, range, lane);
        }
      }
      if (counted != 0xFFFFFFFFu) {                                    // what does not count scores -inf, and its values, whatever they are, are 0
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j)
          s[j / 4u][j % 4u] = (counted >> (16u * (j / 4u) + 4u * g + j % 4u)) & 1u ? s[j / 4u][j % 4u] : a.nothing;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) vx[j] = (counted >> (j * kRowsAtOnce + lane / kRowLanes)) & 1u ? vx[j] : (u32x4)(0u);
      }
      float e[8];                                                      // the scores, then their weights
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) e[j] = s[j / 4u][j % 4u] * a.scale_log2;
      float top = e[0];
#pragma unroll
      for (uint32_t j = 1; j < 8u; ++j) top = fmaxf(top, e[j]);
      top = max32(max16(top));
      const float m_new = fmaxf(m, top);
      const float less = m_new == -INFINITY ? 0.0f : m_new - T::kLift; // what is taken off in the exponent
      if (__builtin_amdgcn_ballot_w64(m_new != m) != 0ull) {
        const float shrink = m == -INFINITY ? 0.0f : exp2f_(m - m_new);
        l *= shrink;
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) acc[d] *= shrink;
        m = m_new;
      }
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) e[j] = exp2f_(e[j] - less);    // rounded as the maximum is: none is above 2^16, however large the scores
      l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      typename T::x8 w[T::kParts];
      T::parts(e, w);

      __builtin_amdgcn_wave_barrier();                                 // the last tile's reads are issued in front of these writes
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        const uint32_t of = j * kRowsAtOnce + lane / kRowLanes, chunk = lane % kRowLanes;
        *reinterpret_cast<u32x4*>(mine + of * (D * 2u) + ((chunk >> 1) ^ value_turn<D>(of)) * 32u + (chunk & 1u) * 16u) = vx[j];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (i + 1u < upto) load_values(now);
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) {
        const uint32_t r = 4u * g + n / 4u;                            // token of the first half
        const u32x2 lo = read_turned(mine + r * (D * 2u) + (d ^ value_turn<D>(r)) * 32u + (n % 4u) * 8u);
        const u32x2 hi = read_turned(mine + (16u + r) * (D * 2u) + (d ^ value_turn<D>(16u + r)) * 32u + (n % 4u) * 8u);
        const typename T::x8 v = __builtin_bit_cast(typename T::x8, (u32x4){lo.x, lo.y, hi.x, hi.y});
#pragma unroll
        for (uint32_t part = 0; part < T::kParts; ++part) acc[d] = T::mfma16(v, w[part], acc[d]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    // No load is on its way any more, which the compiler cannot see: it would wait for them, and with them for this item's stores, where the next item begins.
    __builtin_amdgcn_s_waitcnt(0x0F70);                                // vmcnt(0)

    // Values that are infinite or no number.  Their products are whatever the parts of a weight make of them (0 times infinity is no number), so a dimension
    // that they have spoilt becomes their sum, whatever they weigh; what no such value has spoilt, a weight has, and stays.
    f32x4 zero = (f32x4)(0.0f);                                        // stays that only where all are numbers
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d) zero += acc[d] * 0.0f;
    const bool spoilt = n < heads && !(zero.x + zero.y + zero.z + zero.w == 0.0f);      // (places without a query head meet infinite keys with zeros)
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(spoilt) != 0ull, 0)) {
      f32x4 odd[kSlabs];
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) odd[d] = (f32x4)(0.0f);
      const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
      for (uint32_t i = from; i < upto; ++i) {
        const TileRange t = tile_range(seen, i);
        for (uint32_t token = t.lo; token < t.hi; ++token) {
          const uint32_t page = (uint32_t)entries[token >> a.p.page_shift];
          if (page >= a.p.pages) continue;
          const uint8_t* p = values + (uint64_t)page * a.p.page_stride + (uint64_t)(token & ((1u << a.p.page_shift) - 1u)) * a.p.token_stride + g * 8u;
#pragma unroll
          for (uint32_t d = 0; d < kSlabs; ++d) {
            const typename T::x4 v = *reinterpret_cast<const typename T::x4*>(p + d * 32u);
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j)
              if (!(__builtin_fabsf((float)v[j]) < INFINITY)) odd[d][j] += (float)v[j];
          }
        }
      }
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j)
          if (!(__builtin_fabsf(odd[d][j]) < INFINITY)) acc[d][j] = odd[d][j];
    }

    l = sum32(sum16(l));
    if (from == 0u && upto == tiles) {                                 // the whole item
      const uint64_t at_head = (uint64_t)row * q_heads + hq;
      float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
      float lse = m == -INFINITY ? -INFINITY : (m - T::kLift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
      float other = 0.0f;
      if (n < heads) {
        if (a.prior_out) join(lse, a.prior_lse[at_head], scale, other);
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) {
          f32x4 o = acc[d] * scale;
          const uint64_t where = at_head * D + d * 16u + g * 4u;
          if (a.prior_out && other != 0.0f) o += *reinterpret_cast<const f32x4*>(a.prior_out + where) * other;
          *reinterpret_cast<f32x4*>(a.out + where) = o;
        }
      }
      if (n < heads && a.lse && g == 0u) a.lse[at_head] = lse;
    } else if (n < heads) {
      const uint64_t slot = ((uint64_t)row * inner_count + inner + share) * min(16u, a.rep) + n;
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d)
        *reinterpret_cast<f32x4*>(a.part_o + slot * D + d * 16u + g * 4u) = acc[d];
      if (g == 0u) *reinterpret_cast<f32x2*>(a.part_ml + slot * 2u) = (f32x2){m, l};
    }

    at += upto - from;
    tile = 0u;
    if (--left == 0u || at >= end) return;
    if (++inner == inner_count) {
      inner = 0u;
      ++row;
      seen = seen_by_last((uint32_t)__builtin_amdgcn_readfirstlane((int)row_length(a, row)), a.window, a.sinks);
      tiles = seen_tiles(seen);
    }
  }
}

// Joins the parts of an item that was cut: a workgroup takes `together` query heads of one item, D / 4 lanes each, and goes through the
// parts in as many groups of those lanes as it has.
template <int D, uint32_t THREADS>
__global__ __launch_bounds__(THREADS) void attend_join_kernel(PagedAttendArgs a, uint32_t together, float lift) {
  constexpr uint32_t kLanes = D / 4, kAtOnce = 4;
  __shared__ f32x4 sums[THREADS];
  __shared__ f32x2 tops[THREADS / kLanes];
  const uint32_t lane = threadIdx.x % kWaveSize;
  const uint32_t heads = min(16u, a.rep), inner_count = a.p.kv_heads * a.blocks, q_heads = a.p.kv_heads * a.rep;
  const uint32_t item = blockIdx.x, row = item / inner_count, inner = item % inner_count, block = inner % a.blocks;
  uint32_t all = 0u, front = 0u, own = 0u;
  for (uint32_t r = lane; r < a.p.rows; r += kWaveSize) {
    const uint32_t x = seen_tiles(seen_by_last(row_length(a, r), a.window, a.sinks));
    all += x;
    front += r < row ? x : 0u;
    own += r == row ? x : 0u;
  }
  const uint32_t total = sum64(all) * inner_count, tiles = sum64(own), begin = sum64(front) * inner_count + inner * tiles;
  const Shares shares = deal(total, a.most);
  const uint32_t first = share_of(shares, begin), last = share_of(shares, begin + tiles - 1u);
  if (first == last) return;                                           // finished where it was
  const uint32_t groups = THREADS / kLanes / together;                 // at least one
  const uint32_t group = threadIdx.x / kLanes / together, at = threadIdx.x % kLanes, in_block = blockIdx.y * together + threadIdx.x / kLanes % together;
  const bool some = group < groups && in_block < heads && block * 16u + in_block < a.rep;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = (f32x4)(0.0f);
  for (uint32_t s = first + group; some && s <= last; s += kAtOnce * groups) {
    f32x2 ml[kAtOnce];
    f32x4 x[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t part = min(s + k * groups, last);                // past the last one: the last one, without weight
      const uint64_t slot = ((uint64_t)item + part) * heads + in_block;
      ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
      x[k] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
    }
    float top = m;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      if (s + k * groups > last) ml[k].x = -INFINITY;
      top = fmaxf(top, ml[k].x);
    }
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top);
    l *= keep;
    o *= keep;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      if (s + k * groups > last) continue;
      const float take = ml[k].x == -INFINITY ? 0.0f : exp2f_(ml[k].x - top);      // no weight, but what is infinite in it is seen
      l += ml[k].y * take;
      o += x[k] * take;
    }
    m = top;
  }
  sums[threadIdx.x] = o;
  if (at == 0u) tops[threadIdx.x / kLanes] = (f32x2){m, l};
  __syncthreads();
  if (group != 0u || !some) return;
  const uint32_t busy = min(groups, last - first + 1u);                // groups that have a part
#pragma unroll 4
  for (uint32_t k = 1; k < busy; ++k) {
    const f32x2 ml = tops[k * together + threadIdx.x / kLanes];
    const float top = fmaxf(m, ml.x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top), take = ml.x == -INFINITY ? 0.0f : exp2f_(ml.x - top);
    l = l * keep + ml.y * take;
    o = o * keep + sums[k * together * kLanes + threadIdx.x] * take;
    m = top;
  }
  const uint64_t at_head = (uint64_t)row * q_heads + (inner / a.blocks) * a.rep + block * 16u + in_block;
  float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
  float lse = m == -INFINITY ? -INFINITY : (m - lift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  float other = 0.0f;
  if (a.prior_out) join(lse, a.prior_lse[at_head], scale, other);
  o *= scale;
  if (a.prior_out && other != 0.0f) o += *reinterpret_cast<const f32x4*>(a.prior_out + at_head * D + at * 4u) * other;
  *reinterpret_cast<f32x4*>(a.out + at_head * D + at * 4u) = o;
  if (a.lse && at == 0u) a.lse[at_head] = lse;
}

template <typename T, int D>
hipError_t launch_attend_of(const PagedAttendArgs& a, bool may_split, hipStream_t stream) {
  const uint32_t items = a.p.rows * a.p.kv_heads * a.blocks;
  const uint32_t grid = (a.most + kAttendWaves - 1u) / kAttendWaves;
  // Pages that hold whole tiles: 64 rows of 1004 seen tokens 31.8 us, an address a lane 33.0; 131071 tokens 96.4, 97.1.  A third way, halves of a tile by page, was
  // no faster than an address a lane with pages of 16 (151.5 us each for 48 rows of up to 8K tokens).
  if (a.p.page_shift >= 5u) attend_kernel<T, D, 32u><<<grid, kAttendThreads, 0, stream>>>(a);
  else attend_kernel<T, D, 1u><<<grid, kAttendThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && may_split) {
    // The more parts an item has, the more threads a head: 1024, 256, or one workgroup for an item's heads.  131071 tokens, 256 parts: 96 us, with the small
    // workgroups 118; 1500 tokens, 47 parts: 11.2, with 1024 threads a head 12.5, with all heads in a workgroup 14; 16 rows of 1500, 16 parts: 19.7, 23.5,
    // 21.6; 64 rows with 4 parts: 31.6 together, 36.7 with 256 a head.
    const uint32_t heads = std::min(16u, a.rep), parts = a.most / items;
    if (parts >= 64u) {
      attend_join_kernel<D, 1024><<<dim3(items, heads), 1024, 0, stream>>>(a, 1u, T::kLift);
    } else {
      const uint32_t together = parts >= 8u ? 1u : std::min(heads, 256u / (D / 4u));
      attend_join_kernel<D, 256><<<dim3(items, (heads + together - 1u) / together), 256, 0, stream>>>(a, together, T::kLift);
    }
    e = hipGetLastError();
  }
  return e;
}

template <typename T>
hipError_t launch_attend_type(const PagedAttendArgs& a, uint32_t head_dim, bool may_split, hipStream_t stream) {
  if (head_dim == 64u) return launch_attend_of<T, 64>(a, may_split, stream);
  if (head_dim == 128u) return launch_attend_of<T, 128>(a, may_split, stream);
  return launch_attend_of<T, 256>(a, may_split, stream);
}

}  // namespace

hipError_t launch_paged_attend(const PagedAttendArgs& a, uint32_t head_dim, bool bf16, bool may_split, hipStream_t stream) {
  return bf16 ? launch_attend_type<BFloat>(a, head_dim, may_split, stream) : launch_attend_type<Half>(a, head_dim, may_split, stream);
}

}  // namespace qkv
