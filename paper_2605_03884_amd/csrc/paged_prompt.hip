// paged_prompt.hip — attention of many new tokens of every sequence over its pages: each sees what stands up to its own place, with a window
// the last `window` tokens and the first `sinks`.
//
// Work: a workgroup of 4 or 8 waves takes a tile of (query token, query head) pairs of one kv head, 32 a wave, so that a key is read once for all query
// heads that share it, and goes through the keys they see, 32 or 64 at a time, with a running maximum m, sum l and sum of p.V.  Where there are few query tiles
// the keys are split as well, and where their number would leave much of the chip idle at the end; a second kernel joins the parts.
//
// A tile of keys, one wave (lane = 32 h + n; n is the lane's pair):
//   staging  rows of K and V go from memory into registers and on into LDS, K three tiles ahead of its use and V two; entries are looked up a tile before that.
//   scores   S^T = K Q^T on v_mfma_f32_32x32x16, 32 keys at a time: a lane gets 16 scores of its own pair, the lane 32 further on the other 16.
//   softmax  in the lane, and with the lane 32 further on.  m follows the true maximum only when that has grown by 2^8: sums are
//            kept relative to m, and the weights have 2^7 of room below and 2^8 above before fp16 could overflow.
//   values   O^T = V^T P^T: the weights are where the product wants them; V^T comes out of LDS through the transposing read.
// The scores of the next 32 keys are worked out while the weights of these are (matrix and vector units side by side), their maximum while
// the product with the values is.
// The weights are rounded to the cache's type, as the result is: their errors average out over the keys and stay at the size of the result's own rounding.
//
// What bounds it: no one unit where everything is busy.  8192 tokens of 32 heads, 128 dimensions: 550 - 600 us, 920 - 1000 TFLOP/s, where a product of 8192^3 reaches
// 1256 alone; matrix units are busy 46 % of the cycles, vector instructions issue in 44 %, and the clock, cycles over time, is 1.8 - 2.0 GHz.  64 dimensions have
// half the matrix work for as many weights: a window of 1024 and four sinks over 8000 and 3711 tokens of 32 heads takes 164 - 173 us, vector instructions issuing in 55 % of the
// cycles (7 a weight), matrix units busy 26 %.  The same window without sinks, whose first keys not all pairs of a wave see, over 8000 and 7000 tokens: 64 dimensions 372 - 390 us for
// 64 heads, 128 dimensions 349 - 376 for 32.  61 tokens behind 32768: 64 - 67 us, of which 10 join 32 parts.  Scores beside weights brought the 8K prompt from 675 to 609 us, LDS rows that meet
// each bank once and reads six matrix instructions ahead of their use 593, masks as bits 584.
#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr float kLift = 7.0f, kSlack = 8.0f;
// From here on a maximum's rounding counts in an exponent that is not rounded: scores are multiplied with the scale by themselves, and m follows at once.
// A wave's pairs change over together.  Where one of them has a smaller maximum its scores were not rounded up to there and are afterwards, which may set
// equal ones apart by half a step: 2^-13 at most, a fraction of what rounding a weight to 16 bits does.
constexpr float kFar = 0x1p12f;
constexpr uint32_t kLost = 1u, kScaled = 2u;             // what a wave has met: an entry that names no page, a maximum beyond kFar
__device__ inline float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

// Rows of K and V in LDS are longer than they need to be, by 16 and 64 bytes: 16 lanes that read a piece of 16 bytes of as many rows of K, and 32 that
// read 64 bytes of four rows of V through the transposing read, then meet every bank once.

// Keys of a tile: as many as leave LDS for two workgroups of 4 waves a CU, or one of 8.  Workgroups of 8 waves go through 64 as two halves between two barriers.
constexpr uint32_t prompt_keys(uint32_t waves) { return waves == 8u ? 64u : 32u; }
// Waves a SIMD holds at once: what its 512 registers allow.
constexpr uint32_t prompt_waves_a_simd(int D) { return D == 256 ? 1u : D == 128 ? 2u : 3u; }

constexpr uint32_t key_row(int D) { return D * 2u + 16u; }
constexpr uint32_t value_row(int D) { return D * 2u + 64u; }

// Takes what is infinite or no number out of eight values; whether there was any.
template <typename T>
__device__ inline bool take_out(u32x4& x) {
  constexpr uint32_t e = T::kExponent;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t keep = 0xFFFFFFFFu;
    if ((x[i] & e) == e) keep = 0xFFFF0000u;
    if ((x[i] & (e << 16)) == (e << 16)) keep &= 0xFFFFu;
    any = any || keep != 0xFFFFFFFFu;
    x[i] &= keep;
  }
  return any;
}

template <typename T, int D, uint32_t RUN, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * kWaveSize, prompt_waves_a_simd(D)) void prompt_kernel(PagedPromptArgs a) {
  constexpr uint32_t kThreads = WAVES * kWaveSize;
  constexpr uint32_t kKeys = prompt_keys(WAVES), kHalves = kKeys / 32u;    // keys of a tile; scores are worked out 32 keys at a time
  constexpr uint32_t kPlaces = kHalves + 1u;                           // tiles of K in LDS
  constexpr uint32_t kChunks = D / 8;                                  // 16-byte pieces of a row
  constexpr uint32_t kLoads = kKeys * kChunks / kThreads;              // of them a thread loads, of K and of V
  constexpr uint32_t kRowsAtOnce = kThreads / kChunks;
  constexpr uint32_t kSteps = D / 16, kSlabs = D / 32;
  __shared__ __attribute__((aligned(256))) uint8_t k_place[kPlaces][kKeys * key_row(D)], v_place[2][kKeys * value_row(D)];
  __shared__ uint32_t taken_out;                                       // somebody took something out of the values
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 32u, h = lane / 32u;
  const uint32_t q_heads = a.p.kv_heads * a.rep;

  // the tile: sequence, queries, keys
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
  const int32_t window = (int32_t)a.window, sinks = (int32_t)min(a.sinks, 0x7FFFFFFFu);
  const int32_t reach = base + (int32_t)here;                          // keys below it are seen by somebody
  const KeyTiles key_tiles = key_tiles_of(base, here, window, sinks, kKeys);
  const int32_t win_lo = key_tiles.win_lo;
  const uint32_t sink_end = key_tiles.sink_end, head = key_tiles.head, body = key_tiles.body, tiles = key_tiles.tiles;
  const uint32_t splits = prompt_splits(tiles * kKeys, a.splits, a.least);
  if (blockIdx.y >= splits) return;
  const uint32_t first_tile = (uint32_t)((uint64_t)tiles * blockIdx.y / splits), last_tile = (uint32_t)((uint64_t)tiles * (blockIdx.y + 1u) / splits);
  const auto tile_at = [&](uint32_t i) -> int32_t { return (int32_t)((i < head ? i : body + (i - head)) * kKeys); };
  // Tiles [from, from + count) are seen whole by all queries at places [lo, hi]; those of the sinks are not counted among them.
  struct Range {
    uint32_t from, count;
  };
  const auto whole = [&](int32_t lo, int32_t hi) -> Range {
    const int32_t shift = (int32_t)head - (int32_t)body, win = hi - window + 1;
    const int32_t from = window != 0 && win > 0 ? max(shift + (win + (int32_t)kKeys - 1) / (int32_t)kKeys, (int32_t)head) : (int32_t)head;
    const int32_t upto = lo >= 0 ? shift + (lo + 1) / (int32_t)kKeys : 0;
    return Range{(uint32_t)from, upto > from ? (uint32_t)(upto - from) : 0u};
  };
  const auto holds = [](const Range& r, uint32_t i) { return i - r.from < r.count; };

  // the lane's pair
  const uint32_t pair = wave * 32u + n, token = pair / a.rep, hq = kv_head * a.rep + pair % a.rep;
  const bool live = token < here;
  const int32_t mine = live ? base + (int32_t)token : -1;
  const uint32_t wave_first = wave * 32u / a.rep, wave_last = min((wave * 32u + 31u) / a.rep, here - 1u);
  const Range whole_to_all = whole(base, reach - 1), whole_to_wave = whole(base + (int32_t)wave_first, base + (int32_t)wave_last);
  const uint64_t query = (uint64_t)(uint32_t)start + skip + token;
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
  const uint32_t in_page = (1u << a.p.page_shift) - 1u, my_row = threadIdx.x / kChunks, my_chunk = threadIdx.x % kChunks;
  u32x4 kx[kLoads], vx[kLoads];

  // A tile goes through four hands: its entries are looked up, its rows are loaded, stored to LDS, worked on.  Lane l has token t + l's entry.
  const auto seen_by_some = [&](int32_t key) { return key < reach && (key >= win_lo || key < (int32_t)sink_end); };
  const auto look_up = [&](uint32_t i) -> uint32_t {
    const uint32_t key = min((uint32_t)(tile_at(i) + (int32_t)(lane % kKeys)), (uint32_t)reach - 1u);
    return (uint32_t)entries[key >> a.p.page_shift];
  };
  // Where the thread's rows of a tile are, in head 0: with pages of at least RUN tokens a place for each load that is the same for the wave, to which `own` is
  // added, otherwise the thread's own.  Rows that nobody sees, and those without a page (`lost`, a bit a token), are read from page 0.
  constexpr uint32_t kSpots = RUN == 64u ? 1u : kLoads;
  struct Spots {
    uint64_t at[kSpots];
  };
  const uint32_t own = my_row % RUN * (RUN == 1u ? 0u : (uint32_t)a.p.token_stride) + my_chunk * 16u;
  uint64_t lost = 0ull;
  const auto settle = [&](uint32_t i, uint32_t entry) -> Spots {
    const int32_t t = tile_at(i);
    uint32_t page = entry;
    uint64_t there = ~0ull;
    if (!(holds(whole_to_all, i) && __builtin_amdgcn_ballot_w64(entry >= a.p.pages) == 0ull)) {
      const bool wanted = lane < kKeys && seen_by_some(t + (int32_t)lane), known = entry < a.p.pages;
      there = __builtin_amdgcn_ballot_w64(wanted && known);
      lost = __builtin_amdgcn_ballot_w64(wanted && !known);
      special = (uint32_t)__builtin_amdgcn_readfirstlane((int)(special | (lost != 0ull ? kLost : 0u)));
      page = wanted && known ? entry : 0u;
    }
    Spots to;
#pragma unroll
    for (uint32_t j = 0; j < kSpots; ++j) {
      const uint32_t of = j * kRowsAtOnce + my_row;                    // the row
      if constexpr (RUN == 1u) {
        to.at[j] = (uint64_t)(uint32_t)__shfl((int)page, (int)of) * a.p.page_stride + (uint64_t)(((uint32_t)t + of) & in_page) * a.p.token_stride;
      } else {
        // any token of the run that is there names the page; rows of a run lie one after the other
        const uint32_t first = RUN == 64u ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)(of / RUN * RUN));
        const uint64_t here = there >> first & (RUN == 64u ? ~0ull : (1ull << (RUN % 64u)) - 1ull);
        const uint32_t number = (uint32_t)__builtin_amdgcn_readlane((int)page, (int)(first + (here ? (uint32_t)__builtin_ctzll(here) : 0u)));
        to.at[j] = (uint64_t)number * a.p.page_stride + (((uint32_t)t + first) & in_page) * (uint32_t)a.p.token_stride +
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
  uint8_t* const k_rows = k_place[0] + my_row * key_row(D) + my_chunk * 16u;
  uint8_t* const v_rows = v_place[0] + my_row * value_row(D) + my_chunk * 16u;
  const auto store_keys = [&](uint32_t at, const u32x4 (&x)[kLoads]) {
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(k_rows + at + j * kRowsAtOnce * key_row(D)) = x[j];
  };
  const auto store_values = [&](uint32_t i, uint32_t at) {
    const bool any_lost = (special & kLost) != 0u;                     // in all waves or in none: they look at the same entries
    if (!holds(whole_to_all, i) || any_lost) {                         // only there can a value meet a weight that has to be nothing
      if (any_lost) {
        lost = 0ull;
        settle(i, look_up(i));
      }
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        const uint32_t of = j * kRowsAtOnce + my_row;
        if (!seen_by_some(tile_at(i) + (int32_t)of) || (any_lost && (lost >> of & 1ull))) vx[j] = (u32x4)(0u);
        if (take_out<T>(vx[j])) taken_out = 1u;
      }
      if (any_lost && threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_PAGE);
    }
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(v_rows + at + j * kRowsAtOnce * value_row(D)) = vx[j];
  };

  // The pieces of the work on 32 keys, written out in the order in which they are to be issued: the matrix instructions with what the vector
  // unit does meanwhile, and the reads of LDS kAhead matrix instructions in front of their use, from the keys on into the values and from the
  // values on into the next keys.
  constexpr uint32_t kProducts = 2u * kSlabs, kAhead = D == 64 ? 4u : 6u;
  static_assert(kAhead <= kSteps && kAhead <= kProducts && kProducts == kSteps);
  typename T::x8 k_piece[kSteps], v_piece[kProducts];
  const auto read_key = [&](const uint8_t* at, uint32_t k) { k_piece[k] = __builtin_bit_cast(typename T::x8, *reinterpret_cast<const u32x4*>(at + n * key_row(D) + (k * 2u + h) * 16u)); };
  const auto read_ahead = [&](const uint8_t* at) {
#pragma unroll
    for (uint32_t k = 0; k < kAhead; ++k) read_key(at, k);
  };
  const auto read_value = [&](const uint8_t* at, uint32_t k) {
    const uint8_t* p = at + (4u * h + (lane % 16u) / 4u) * value_row(D) + (lane / 16u % 2u) * 32u + (lane % 4u) * 8u;
    const u32x2 lo = read_turned(p + (k / kSlabs) * 16u * value_row(D) + (k % kSlabs) * 64u), hi = read_turned(p + ((k / kSlabs) * 16u + 8u) * value_row(D) + (k % kSlabs) * 64u);
    v_piece[k] = __builtin_bit_cast(typename T::x8, (u32x4){lo.x, lo.y, hi.x, hi.y});
  };
  constexpr uint32_t kEach = 16u / kSteps;                             // scores to a matrix instruction
  typename T::x8 w[2];
  const auto weigh = [&](const f32x16& s, uint32_t first, uint32_t count) {
    float e[16], sum = 0.0f;
#pragma unroll
    for (uint32_t j = first; j < first + count; ++j) e[j] = exp2f_(__builtin_fmaf(s[j], scale, -less));
#pragma unroll
    for (uint32_t j = first; j < first + count; ++j) {
      asm volatile("" : "+v"(e[j]));                                   // here, and not behind the next branch
      sum = j == first ? e[j] : sum + e[j];
      w[j / 8u][j % 8u] = (typename T::one)e[j];
    }
    l += sum;
  };
  float top = 0.0f;
  const auto largest = [&](const f32x16& s, uint32_t first, uint32_t count) {
#pragma unroll
    for (uint32_t j = first; j < first + count; ++j) top = j == 0u ? s[0] : fmaxf(top, s[j]);
  };
  // scores of 32 keys, whose first pieces have been read, beside the weights of the scores `now`
  const auto scores = [&](const uint8_t* k_at, const uint8_t* v_at, f32x16& next, const f32x16& now) {
    next = (f32x16)(0.0f);
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
      if (k + kAhead < kSteps) read_key(k_at, k + kAhead);
      else read_value(v_at, k + kAhead - kSteps);
      next = T::mfma32(k_piece[k], q[k], next);
      weigh(now, k * kEach, kEach);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // the product of 32 weights with their values, beside the largest of the scores `next`
  const auto product = [&](const uint8_t* v_at, const uint8_t* k_next, const f32x16& next) {          // k_next: read with two halves to a tile only
#pragma unroll
    for (uint32_t k = 0; k < kProducts; ++k) {
      if (k + kAhead < kProducts) read_value(v_at, k + kAhead);
      else if constexpr (kHalves == 2u) read_key(k_next, k + kAhead - kProducts);
      acc[k % kSlabs] = T::mfma32(v_piece[k], w[k / kSlabs], acc[k % kSlabs]);
      largest(next, k * kEach, kEach);
      asm volatile("" : "+v"(top));
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // what the lane's pair does not see of 32 keys scores -inf: a bit for each key
  const auto mask = [&](uint32_t i, uint32_t half, f32x16& s) {
    const int32_t t = tile_at(i) + (int32_t)(half * 32u);
    const auto below = [](int32_t n) { return (uint32_t)((1ull << (uint32_t)min(max(n, 0), 32)) - 1ull); };
    uint32_t seen = below(mine - t + 1);
    if (window != 0) seen &= ~below(mine - t - window + 1) | below(sinks - t);
    if (special != 0u) {
      if ((special & kLost) != 0u) {
        lost = 0ull;
        settle(i, look_up(i));
        seen &= ~(uint32_t)(lost >> (32u * half));
      }
      if ((special & kScaled) != 0u) s *= a.scale_log2;
    }
    seen >>= 4u * h;
#pragma unroll
    for (uint32_t j = 0; j < 16u; ++j) s[j] = seen >> (8u * (j / 4u) + j % 4u) & 1u ? s[j] : -INFINITY;
  };
  const auto masked = [&](uint32_t i) { return !holds(whole_to_wave, i) || special != 0u; };
  // m, which is -inf at first, to the largest of the scores s
  const auto follow = [&](f32x16& s) {
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

  if (threadIdx.x == 0u) taken_out = 0u;
  __syncthreads();
  if (first_tile < last_tile) {
    constexpr uint32_t kKeyPlace = kKeys * key_row(D), kValuePlace = kKeys * value_row(D);
    f32x16 s_one, s_two;
    uint32_t i = first_tile;
    const auto no_further = [&](uint32_t at) { return min(at, last_tile - 1u); };       // what is read ahead behind the last tile is the last tile
    uint32_t k_now = 0u, k_next = kKeyPlace, k_free = (kPlaces - 1u) * kKeyPlace, v_now = 0u;      // with two places of K k_free is not used
    const uint32_t entries_ahead[3] = {look_up(i), look_up(no_further(i + 1u)), look_up(no_further(i + 2u))};
    uint32_t entry = look_up(no_further(i + 3u));
    u32x4 second[kLoads];
    Spots spots = settle(i, entries_ahead[0]);
    load(keys, spots, kx);
    load(values, spots, vx);
    spots = settle(no_further(i + 1u), entries_ahead[1]);
    load(keys, spots, second);
    store_keys(0u, kx);
    store_values(i, 0u);
    store_keys(kKeyPlace, second);
    load(values, spots, vx);
    spots = settle(no_further(i + 2u), entries_ahead[2]);
    load(keys, spots, kx);
    __syncthreads();
    s_one = (f32x16)(0.0f);
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
      read_key(k_place[0], k);
      s_one = T::mfma32(k_piece[k], q[k], s_one);
    }
    if (masked(i)) mask(i, 0u, s_one);
    largest(s_one, 0u, 16u);
    follow(s_one);
    if constexpr (kHalves == 2u) read_ahead(k_place[0] + 32u * key_row(D));
    __syncthreads();
    // 32 keys: the weights of `now` and their product with the values, beside the scores of the next 32 and their largest.
    const auto half = [&](const uint8_t* k_at, const uint8_t* v_at, const uint8_t* k_next, const f32x16& now, f32x16& next, uint32_t next_tile, uint32_t next_half) {
      scores(k_at, v_at, next, now);
      if (masked(next_tile)) mask(next_tile, next_half, next);
      product(v_at, k_next, next);
      follow(next);
    };
    const auto last_half = [&](const uint8_t* v_at, const f32x16& now) {
      weigh(now, 0u, 16u);
#pragma unroll
      for (uint32_t k = 0; k < kProducts; ++k) {
        read_value(v_at, k);
        acc[k % kSlabs] = T::mfma32(v_piece[k], w[k / kSlabs], acc[k % kSlabs]);
      }
    };
    // tile i, whose first scores are `now`; afterwards `next` has the next tile's, or where a tile is two halves `now` again
    const auto step = [&](f32x16& now, f32x16& next) {
      // the keys of tile i + 2 and the values of i + 1 take places that nobody reads any more; those of i + 3 and i + 2 are asked for
      store_keys(kHalves == 2u ? k_free : k_now, kx);
      store_values(i + 1u, kValuePlace - v_now);
      load(values, spots, vx);
      spots = settle(no_further(i + 3u), entry);
      load(keys, spots, kx);
      entry = look_up(no_further(i + 4u));
      const uint8_t *const v_at = v_place[0] + v_now, *const k_at = k_place[0] + k_now, *const k_then = k_place[0] + k_next;
      if constexpr (kHalves == 2u) {
        half(k_at + 32u * key_row(D), v_at, k_then, now, next, i, 1u);
        half(k_then, v_at + 32u * value_row(D), k_then + 32u * key_row(D), next, now, i + 1u, 0u);
        const uint32_t old = k_now;
        k_now = k_next;
        k_next = k_free;
        k_free = old;
      } else {
        read_ahead(k_then);                                            // the tile after it takes its place meanwhile, behind the barrier
        half(k_then, v_at, k_then, now, next, i + 1u, 0u);
        k_now = k_next;
        k_next = kKeyPlace - k_next;
      }
      v_now = kValuePlace - v_now;
      ++i;
      __syncthreads();
    };
    if constexpr (kHalves == 2u) {
      while (i + 1u < last_tile) step(s_one, s_two);
      half(k_place[0] + k_now + 32u * key_row(D), v_place[0] + v_now, k_place[0] + k_now, s_one, s_two, i, 1u);
      last_half(v_place[0] + v_now + 32u * value_row(D), s_two);
    } else {
      while (i + 2u < last_tile) {
        step(s_one, s_two);
        step(s_two, s_one);
      }
      if (i + 1u < last_tile) {
        step(s_one, s_two);
        s_one = s_two;
      }
      last_half(v_place[0] + v_now, s_one);
    }
  }

  if (live) {
    if (taken_out != 0u) {
      // What was taken out counts for the pairs that see it, and for no other: their sums become infinite or no number, whatever the weight.
      for (uint32_t i = first_tile; i < last_tile; ++i) {
        const int32_t t = tile_at(i);
        for (int32_t key = t; key < t + (int32_t)kKeys; ++key) {
          if (key > mine || key >= reach || (window != 0 && key <= mine - window && key >= sinks)) continue;
          const uint32_t page = (uint32_t)entries[(uint32_t)key >> a.p.page_shift];
          if (page >= a.p.pages) continue;
          const uint8_t* from = values + (uint64_t)page * a.p.page_stride + (uint64_t)((uint32_t)key & in_page) * a.p.token_stride + h * 8u;
#pragma unroll
          for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) {
              const typename T::x4 v = *reinterpret_cast<const typename T::x4*>(from + (d * 4u + j) * 16u);
#pragma unroll
              for (uint32_t e = 0; e < 4u; ++e)
                if (!(__builtin_fabsf((float)v[e]) < INFINITY)) acc[d][4u * j + e] += (float)v[e];
            }
        }
      }
    }
    const uint64_t out_at = query * q_heads + hq;
    const float sum = sum32(l);
    if (splits != 1u) {
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
}

// Joins the parts of the query heads of one token, D / 4 lanes each: 32 parts of 61 tokens of 32 heads, 32 MB, 10.5 us (3 TB/s, two rounds of reads).
constexpr uint32_t kJoinThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void prompt_join_kernel(PagedPromptArgs a) {
  constexpr uint32_t kLanes = D / 4, kAtOnce = 8;
  const uint32_t lane = threadIdx.x % kWaveSize, q_heads = a.p.kv_heads * a.rep, token = blockIdx.x, keys = prompt_keys(a.waves);
  const uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return (uint32_t)a.starts[b] <= token; }));
  const int32_t start = a.starts[row], end = a.starts[row + 1u];
  if (start < 0 || (uint32_t)start > token || end <= (int32_t)token || (uint32_t)end > a.tokens) return;      // nobody's token has no parts
  const uint32_t count = (uint32_t)(end - start), skip = (token - (uint32_t)start) / a.per * a.per;
  const int32_t length = (int32_t)held(a.p.lens[row], a.p.row_pages, a.p.page_shift);
  const KeyTiles key_tiles = key_tiles_of(length - (int32_t)count + (int32_t)skip, min(a.per, count - skip), (int32_t)a.window, (int32_t)min(a.sinks, 0x7FFFFFFFu), keys);
  const uint32_t splits = prompt_splits(key_tiles.tiles * keys, a.splits, a.least);
  if (splits == 1u) return;                                            // finished where it was
  const uint32_t at = threadIdx.x % kLanes;
  const uint64_t all = (uint64_t)a.tokens * q_heads;
  for (uint32_t hq = blockIdx.y * (kJoinThreads / kLanes) + threadIdx.x / kLanes; hq < q_heads; hq += gridDim.y * (kJoinThreads / kLanes)) {
    const uint64_t pair = (uint64_t)token * q_heads + hq;
    float m = -INFINITY, l = 0.0f;
    f32x4 o = (f32x4)(0.0f);
    for (uint32_t s = 0; s < splits; s += kAtOnce) {
      f32x2 ml[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (uint32_t k = 0; k < kAtOnce; ++k) {
        const uint64_t slot = min(s + k, splits - 1u) * all + pair;      // past the last one: the last one, without weight
        ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
        x[k] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
      }
      float top = m;
#pragma unroll
      for (uint32_t k = 0; k < kAtOnce; ++k) {
        if (s + k >= splits) ml[k].x = -INFINITY;
        top = fmaxf(top, ml[k].x);
      }
      const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top);
      l *= keep;
      o *= keep;
#pragma unroll
      for (uint32_t k = 0; k < kAtOnce; ++k) {
        const float take = ml[k].x == -INFINITY ? 0.0f : exp2f_(ml[k].x - top);
        l += ml[k].y * take;
        o += x[k] * take;
      }
      m = top;
    }
    const float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
    typename T::x4 r;
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e) r[e] = (typename T::one)(o[e] * scale);
    *reinterpret_cast<typename T::x4*>(a.out + (pair * D + at * 4u) * 2u) = r;
    if (a.lse && at == 0u) a.lse[pair] = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

// Pages that hold a whole tile, pages that hold 16 rows, others: 8K prompt with pages of 64 tokens 571 us, 577 by runs of 16, 584 by an address a thread.
template <typename T, int D, uint32_t WAVES>
void launch_prompt_run(const PagedPromptArgs& a, hipStream_t stream) {
  const dim3 grid(places(a.tokens, a.p.rows, a.per) * a.p.kv_heads, a.splits);
  if (a.p.page_shift >= 6u) prompt_kernel<T, D, 64u, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
  else if (a.p.page_shift >= 4u) prompt_kernel<T, D, 16u, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
  else prompt_kernel<T, D, 1u, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
}

template <typename T, int D>
hipError_t launch_prompt_of(const PagedPromptArgs& a, hipStream_t stream) {
  if (D == 128 && a.waves == 8u) launch_prompt_run<T, 128, 8u>(a, stream);
  else launch_prompt_run<T, D, 4u>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1u) return e;
  // Long parts come with many tokens, and with none at all where sequences turn out to be short: a workgroup a token, which goes through its heads.
  const uint32_t groups = a.least > 512u ? 1u : (a.p.kv_heads * a.rep + kJoinThreads / (D / 4) - 1u) / (kJoinThreads / (D / 4));
  prompt_join_kernel<T, D><<<dim3(a.tokens, groups), kJoinThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_prompt_type(const PagedPromptArgs& a, uint32_t head_dim, hipStream_t stream) {
  if (head_dim == 64u) return launch_prompt_of<T, 64>(a, stream);
  if (head_dim == 128u) return launch_prompt_of<T, 128>(a, stream);
  return launch_prompt_of<T, 256>(a, stream);
}

}  // namespace

hipError_t launch_paged_prompt(const PagedPromptArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  return bf16 ? launch_prompt_type<BFloat>(a, head_dim, stream) : launch_prompt_type<Half>(a, head_dim, stream);
}

}  // namespace qkv
