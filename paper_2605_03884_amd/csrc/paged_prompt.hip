// paged_prompt.hip — attention of many new tokens of every sequence over its pages: each sees what stands up to its own place, with a window
// the last `window` tokens and the first `sinks`.
//
// Work: a workgroup takes a tile of (query token, query head) pairs of one kv head, 32 a wave, so that a key is read once for all query heads that
// share it, and goes through the keys they see 64 at a time, with a running maximum m, sum l and sum of p.V.  Where there are few query
// tiles the keys are split as well, and a second kernel joins the parts.
//
// A tile of 64 keys, one wave (lane = 32 h + n; n is the lane's pair):
//   staging  rows of K and V go from memory into registers and on into LDS, K two tiles ahead of its use and V one, each into one of two
//            places: K in 16-byte pieces exchanged by token, V in 64-byte pieces, so that no read below meets a bank twice.
//   scores   S^T = K Q^T on v_mfma_f32_32x32x16: a lane gets 32 scores of its own pair.
//   softmax  in the lane, and with the lane 32 further on.  m follows the true maximum only when that has grown by 2^8: sums are
//            kept relative to m, and the weights have 2^7 of room below and 2^8 above before fp16 could overflow.
//   values   O^T = V^T P^T: the weights are where the product wants them; V^T comes out of LDS through the transposing read.
// The scores of a tile are worked out while the weights of the tile before are (matrix and vector units side by side), its maximum
// while the product of the tile before is.
// The weights are rounded to the cache's type, as the result is: their errors average out over the keys and stay at the size of the result's own rounding.
#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr float kLift = 7.0f, kSlack = 8.0f;

// Waves a SIMD holds at once: what its 512 registers allow.
constexpr uint32_t prompt_waves_a_simd(int D, uint32_t waves) { return D == 256 ? 1u : waves == 8u ? 2u : D == 64 ? 2u : 1u; }

// Where the 16-byte piece `chunk` of token `token`'s row of K stands in LDS.
template <int D>
__device__ inline uint32_t key_at(uint32_t token, uint32_t chunk) {
  const uint32_t turn = D == 64 ? (token >> 1) & 7u : token & 15u;
  return token * (D * 2u) + (chunk ^ turn) * 16u;
}
// The same for V, by its piece of 64 bytes.
template <int D>
__device__ inline uint32_t value_at(uint32_t token, uint32_t piece) {
  const uint32_t turn = D == 64 ? (token >> 1) & 1u : token & 3u;
  return token * (D * 2u) + (piece ^ turn) * 64u;
}

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

template <typename T, int D, uint32_t RUN, bool SPLIT, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * kWaveSize, prompt_waves_a_simd(D, WAVES)) void prompt_kernel(PagedPromptArgs a) {
  constexpr uint32_t kThreads = WAVES * kWaveSize;
  constexpr uint32_t kKeys = kPromptKeys, kChunks = D / 8;             // 16-byte pieces of a row
  constexpr uint32_t kLoads = kKeys * kChunks / kThreads;              // of them a thread loads, of K and of V
  constexpr uint32_t kRowsAtOnce = kThreads / kChunks;
  constexpr uint32_t kSteps = D / 16, kSlabs = D / 32;
  __shared__ __attribute__((aligned(256))) uint8_t k_place[2][kKeys * D * 2], v_place[2][kKeys * D * 2];
  __shared__ uint32_t taken_out;                                       // somebody took something out of the values
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 32u, h = lane / 32u;
  const uint32_t q_heads = a.p.kv_heads * a.rep;

  // the tile: sequence, queries, keys
  const uint32_t kv_head = blockIdx.x % a.p.kv_heads;
  const uint32_t at = gridDim.x / a.p.kv_heads - 1u - blockIdx.x / a.p.kv_heads;      // tiles with many keys first
  const uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return first_place((uint32_t)a.starts[b], b, a.per) <= at; }));
  const int32_t start = a.starts[row], end = a.starts[row + 1u];
  if (start < 0 || end < start || (uint32_t)end > a.tokens) {
    if (threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_ROW);
    return;
  }
  const uint32_t count = (uint32_t)(end - start), skip = (at - first_place((uint32_t)start, row, a.per)) * a.per;
  if (at < first_place((uint32_t)start, row, a.per) || skip >= count) return;
  const uint32_t here = min(a.per, count - skip);                      // query tokens
  const int32_t length = (int32_t)held(a.p.lens[row], a.p.row_pages, a.p.page_shift);
  const int32_t base = length - (int32_t)count + (int32_t)skip;        // place of the tile's first query
  if (base < 0 && threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_ROW);
  const int32_t window = (int32_t)a.window, sinks = (int32_t)min(a.sinks, 0x7FFFFFFFu);
  const int32_t reach = base + (int32_t)here;                          // keys below it are seen by somebody
  const int32_t win_lo = window != 0 && base >= window ? base - window + 1 : 0;
  const uint32_t sink_end = (uint32_t)min(sinks, win_lo);
  const uint32_t head = (sink_end + kKeys - 1u) / kKeys;
  const uint32_t body = max((uint32_t)win_lo / kKeys, head), stop = reach > 0 ? ((uint32_t)reach + kKeys - 1u) / kKeys : 0u;
  const uint32_t tiles = head + (stop > body ? stop - body : 0u);
  const uint32_t first_tile = SPLIT ? (uint32_t)((uint64_t)tiles * blockIdx.y / a.splits) : 0u;
  const uint32_t last_tile = SPLIT ? (uint32_t)((uint64_t)tiles * (blockIdx.y + 1u) / a.splits) : tiles;
  const auto tile_at = [&](uint32_t i) -> int32_t { return (int32_t)((i < head ? i : body + (i - head)) * kKeys); };
  // whether every one of the queries at places [lo, hi] sees all of the tile's keys
  const auto whole = [&](int32_t t, int32_t lo, int32_t hi) { return t + (int32_t)kKeys - 1 <= lo && (window == 0 || t > hi - window || t + (int32_t)kKeys <= sinks); };
  // the lane's pair
  const uint32_t pair = wave * 32u + n, token = pair / a.rep, head_in = pair % a.rep;
  const bool live = token < here;
  const int32_t mine = live ? base + (int32_t)token : -1;
  const uint32_t wave_first = wave * 32u / a.rep, wave_last = min((wave * 32u + 31u) / a.rep, here - 1u);
  const int32_t wave_lo = base + (int32_t)wave_first, wave_hi = base + (int32_t)wave_last;
  const uint64_t query = (uint64_t)(uint32_t)start + skip + token;
  const uint32_t hq = kv_head * a.rep + head_in;
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
  float m = -INFINITY, l = 0.0f;

  const uint8_t* keys = a.p.k + (uint64_t)kv_head * a.p.head_stride;
  const uint8_t* values = a.p.v + (uint64_t)kv_head * a.p.head_stride;
  const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
  const uint32_t in_page = (1u << a.p.page_shift) - 1u, my_row = threadIdx.x / kChunks, my_chunk = threadIdx.x % kChunks;
  u32x4 kx[kLoads], vx[kLoads];

  // A tile goes through four hands: its entries are looked up, its rows are loaded, stored to LDS, worked on; each a tile ahead of the next.
  // Lane l has token t + l's entry.  Nobody sees the tokens of `hidden` (they may be anything); those of `lost` have no page.
  const auto seen_by_some = [&](int32_t key) { return key < reach && (key >= win_lo || key < (int32_t)sink_end); };
  const auto look_up = [&](uint32_t i) -> uint32_t {
    const int32_t key = tile_at(i) + (int32_t)lane;
    return seen_by_some(key) ? (uint32_t)entries[(uint32_t)key >> a.p.page_shift] : 0u;
  };
  struct Source {
    uint32_t page;                                                     // of token t + lane
    uint64_t hidden, lost;
  };
  const auto settle = [&](uint32_t i, uint32_t entry) -> Source {
    const bool wanted = seen_by_some(tile_at(i) + (int32_t)lane), known = entry < a.p.pages;
    return Source{wanted && known ? entry : 0u, ~__builtin_amdgcn_ballot_w64(wanted && known), __builtin_amdgcn_ballot_w64(wanted && !known)};
  };
  const auto load = [&](const uint8_t* pool, uint32_t i, const Source& from, u32x4 (&x)[kLoads]) {
    const int32_t t = tile_at(i);
    if constexpr (RUN == 1u) {
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        const uint32_t of = j * kRowsAtOnce + my_row;
        x[j] = *reinterpret_cast<const u32x4*>(pool + (uint64_t)(uint32_t)__shfl((int)from.page, (int)of) * a.p.page_stride +
                                               (uint64_t)(((uint32_t)t + of) & in_page) * a.p.token_stride + my_chunk * 16u);
      }
    } else {
      // rows of one run lie one after the other: a place that is the same for the wave and 32 bits of the lane's own
      const uint32_t own = my_row % RUN * (uint32_t)a.p.token_stride + my_chunk * 16u;
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        const uint32_t run = RUN == 64u ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)((j * kRowsAtOnce + my_row) / RUN));
        const uint64_t here = ~from.hidden >> (run * RUN % 64u) & (RUN == 64u ? ~0ull : (1ull << (RUN % 64u)) - 1ull);      // any of its tokens that is there names the page
        const uint32_t of = (uint32_t)__builtin_amdgcn_readlane((int)from.page, (int)(run * RUN + (here ? (uint32_t)__builtin_ctzll(here) : 0u)));
        const uint32_t in_run = kRowsAtOnce < RUN ? j * kRowsAtOnce % RUN : 0u;
        x[j] = *reinterpret_cast<const u32x4*>(pool + ((uint64_t)of * a.p.page_stride + (uint64_t)(((uint32_t)t + run * RUN) & in_page) * a.p.token_stride +
                                                       in_run * a.p.token_stride) + own);
      }
    }
  };
  const auto careful = [&](uint32_t i, uint64_t lost) { return !whole(tile_at(i), base, reach - 1) || lost != 0ull; };
  const auto store_keys = [&](uint32_t side) {
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) *reinterpret_cast<u32x4*>(k_place[side] + key_at<D>(j * kRowsAtOnce + my_row, my_chunk)) = kx[j];
  };
  const auto store_values = [&](uint32_t i, const Source& from, uint32_t side) {
    if (careful(i, from.lost)) {                                       // only there can a value meet a weight that has to be nothing
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        if (from.hidden >> (j * kRowsAtOnce + my_row) & 1ull) vx[j] = (u32x4)(0u);
        if (take_out<T>(vx[j])) taken_out = 1u;
      }
      if (from.lost != 0ull && threadIdx.x == 0u) flag(a.status, QKV_STATUS_BAD_PAGE);
    }
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j)
      *reinterpret_cast<u32x4*>(v_place[side] + value_at<D>(j * kRowsAtOnce + my_row, my_chunk / 4u) + (my_chunk % 4u) * 16u) = vx[j];
  };
  const auto scores = [&](uint32_t side, f32x16 (&s)[2]) {
    s[0] = s[1] = (f32x16)(0.0f);
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k)
#pragma unroll
      for (uint32_t u = 0; u < 2u; ++u) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(k_place[side] + key_at<D>(u * 32u + n, k * 2u + h));
        s[u] = T::mfma32(__builtin_bit_cast(typename T::x8, x), q[k], s[u]);
      }
  };
  const auto mask = [&](uint32_t i, uint64_t lost, f32x16 (&s)[2]) {
    const int32_t t = tile_at(i);
    const int32_t up = mine - t - 4 * (int32_t)h, low = window != 0 ? up - window : -1 - 4 * (int32_t)h - (int32_t)kKeys, sink = window != 0 ? sinks - t - 4 * (int32_t)h : 0;
#pragma unroll
    for (uint32_t u = 0; u < 2u; ++u)
#pragma unroll
      for (uint32_t j = 0; j < 16u; ++j) {
        const int32_t c = (int32_t)(u * 32u + 8u * (j / 4u) + j % 4u);
        bool seen = c <= up && (c > low || c < sink);
        if ((uint32_t)(lost >> (32u * u)) >> (8u * (j / 4u) + j % 4u + 4u * h) & 1u) seen = false;
        s[u][j] = seen ? s[u][j] : -INFINITY;
      }
  };
  const auto largest = [&](const f32x16 (&s)[2]) {
    float top = s[0][0];
#pragma unroll
    for (uint32_t j = 1; j < 32u; ++j) top = fmaxf(top, s[j / 16u][j % 16u]);
    return max32(top) * a.scale_log2;
  };
  const auto follow = [&](float top) {                                 // m, which is -inf at first, to the largest score there is
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0ull) {
      const float next = fmaxf(m, top);
      const float shrink = m == -INFINITY ? 0.0f : exp2f_(m - next);
      l *= shrink;
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) acc[d] *= shrink;
      m = next;
    }
  };
  const auto masked = [&](uint32_t i, uint64_t lost) { return !whole(tile_at(i), wave_lo, wave_hi) || lost != 0ull; };
  const auto weights = [&](const f32x16 (&s)[2], typename T::x8 (&w)[4]) {
    const float less = m == -INFINITY ? 0.0f : m - kLift;
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u) {
      float e[8];
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) {
        e[j] = exp2f_(__builtin_fmaf(s[u / 2u][8u * (u % 2u) + j], a.scale_log2, -less));
        w[u][j] = (typename T::one)e[j];
      }
      l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    }
  };
  const auto product = [&](uint32_t side, const typename T::x8 (&w)[4]) {
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u) {
      const uint32_t r = u * 16u + 4u * h + (lane % 16u) / 4u;         // token of the first four
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) {
        const uint32_t in_piece = (lane / 16u % 2u) * 32u + (lane % 4u) * 8u;
        const u32x2 lo = read_turned(v_place[side] + value_at<D>(r, d) + in_piece);
        const u32x2 hi = read_turned(v_place[side] + value_at<D>(r + 8u, d) + in_piece);
        acc[d] = T::mfma32(__builtin_bit_cast(typename T::x8, (u32x4){lo.x, lo.y, hi.x, hi.y}), w[u], acc[d]);
      }
    }
  };
  if (threadIdx.x == 0u) taken_out = 0u;
  __syncthreads();
  if (first_tile < last_tile) {
    f32x16 s_one[2], s_two[2];
    typename T::x8 w[4];
    Source first = {}, second = {}, third = {};                        // of the tiles i + 1, i + 2, i + 3
    uint32_t i = first_tile, entry = 0u;
    {
      const Source from = settle(i, look_up(i));
      load(keys, i, from, kx);
      load(values, i, from, vx);
      if (i + 1u < last_tile) first = settle(i + 1u, look_up(i + 1u));
      if (i + 2u < last_tile) second = settle(i + 2u, look_up(i + 2u));
      if (i + 3u < last_tile) entry = look_up(i + 3u);
      store_keys(0u);
      store_values(i, from, 0u);
      if (i + 1u < last_tile) {
        load(keys, i + 1u, first, kx);
        load(values, i + 1u, first, vx);
        store_keys(1u);
      }
      if (i + 2u < last_tile) load(keys, i + 2u, second, kx);
      __syncthreads();
      scores(0u, s_one);
      if (masked(i, from.lost)) mask(i, from.lost, s_one);
      follow(largest(s_one));
      __syncthreads();
    }
    // One tile: its weights and its product with the values, with the next tile's scores and their maximum.
    const auto step = [&](uint32_t side, const f32x16 (&now)[2], f32x16 (&next)[2]) {
      // keys of i + 2 take the place of those of i, values of i + 1 that of those of i - 1
      if (i + 2u < last_tile) store_keys(side);
      store_values(i + 1u, first, side ^ 1u);
      if (i + 3u < last_tile) {
        third = settle(i + 3u, entry);
        load(keys, i + 3u, third, kx);
      }
      if (i + 2u < last_tile) load(values, i + 2u, second, vx);
      if (i + 4u < last_tile) entry = look_up(i + 4u);
      scores(side ^ 1u, next);
      weights(now, w);
      if (masked(i + 1u, first.lost)) mask(i + 1u, first.lost, next);
      product(side, w);
      follow(largest(next));
      first = second;
      second = third;
      ++i;
      __syncthreads();
    };
    while (i + 2u < last_tile) {
      step(0u, s_one, s_two);
      step(1u, s_two, s_one);
    }
    if (i + 1u < last_tile) {
      step(0u, s_one, s_two);
      weights(s_two, w);
      product(1u, w);
    } else {
      weights(s_one, w);
      product(0u, w);
    }
  }

  if (taken_out != 0u && live) {
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
  if (!live) return;
  l = sum32(l);
  const uint64_t out = query * q_heads + hq;
  if constexpr (SPLIT) {
    const uint64_t slot = (uint64_t)blockIdx.y * a.tokens * q_heads + out;
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j)
        *reinterpret_cast<f32x4*>(a.part_o + slot * D + d * 32u + j * 8u + h * 4u) = (f32x4){acc[d][4 * j], acc[d][4 * j + 1], acc[d][4 * j + 2], acc[d][4 * j + 3]};
    if (h == 0u) *reinterpret_cast<f32x2*>(a.part_ml + slot * 2u) = (f32x2){m, l};
  } else {
    const float scale = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) {
        typename T::x4 o;
#pragma unroll
        for (uint32_t e = 0; e < 4u; ++e) o[e] = (typename T::one)(acc[d][4u * j + e] * scale);
        *reinterpret_cast<typename T::x4*>(a.out + (out * D + d * 32u + j * 8u + h * 4u) * 2u) = o;
      }
    if (a.lse && h == 0u) a.lse[out] = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_log2f(l)) * 0.6931471805599453f;
  }
}

// Joins the parts of every (query token, query head): D / 4 lanes each.
constexpr uint32_t kJoinThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void prompt_join_kernel(PagedPromptArgs a) {
  constexpr uint32_t kLanes = D / 4;
  const uint64_t all = (uint64_t)a.tokens * (a.p.kv_heads * a.rep);
  const uint64_t pair = (uint64_t)blockIdx.x * (kJoinThreads / kLanes) + threadIdx.x / kLanes;
  const uint32_t at = threadIdx.x % kLanes;
  const uint32_t used = (uint32_t)a.starts[a.p.rows];                  // tokens behind the last sequence have no parts
  if (pair >= all || pair / (a.p.kv_heads * a.rep) >= used || pair / (a.p.kv_heads * a.rep) < (uint32_t)a.starts[0]) return;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = (f32x4)(0.0f);
  for (uint32_t s = 0; s < a.splits; ++s) {
    const uint64_t slot = s * all + pair;
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
    const float top = fmaxf(m, ml.x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top), take = ml.x == -INFINITY ? 0.0f : exp2f_(ml.x - top);
    l = l * keep + ml.y * take;
    o = o * keep + x * take;
    m = top;
  }
  const float scale = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  typename T::x4 r;
#pragma unroll
  for (uint32_t e = 0; e < 4u; ++e) r[e] = (typename T::one)(o[e] * scale);
  *reinterpret_cast<typename T::x4*>(a.out + (pair * D + at * 4u) * 2u) = r;
  if (a.lse && at == 0u) a.lse[pair] = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_log2f(l)) * 0.6931471805599453f;
}

template <typename T, int D, bool SPLIT, uint32_t WAVES>
void launch_prompt_run(const PagedPromptArgs& a, hipStream_t stream) {
  const dim3 grid(places(a.tokens, a.p.rows, a.per) * a.p.kv_heads, a.splits);
  if (a.p.page_shift >= 6u) prompt_kernel<T, D, 64u, SPLIT, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
  else if (a.p.page_shift >= 4u) prompt_kernel<T, D, 16u, SPLIT, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
  else prompt_kernel<T, D, 1u, SPLIT, WAVES><<<grid, WAVES * kWaveSize, 0, stream>>>(a);
}

template <typename T, int D>
hipError_t launch_prompt_of(const PagedPromptArgs& a, hipStream_t stream) {
  if (a.splits == 1u) {
    if (D <= 128 && a.waves == 8u) launch_prompt_run<T, D <= 128 ? D : 64, false, 8u>(a, stream);
    else launch_prompt_run<T, D, false, 4u>(a, stream);
    return hipGetLastError();
  }
  launch_prompt_run<T, D, true, 4u>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint64_t pairs = (uint64_t)a.tokens * (a.p.kv_heads * a.rep);
  constexpr uint32_t kPairs = kJoinThreads / (D / 4);
  prompt_join_kernel<T, D><<<(uint32_t)((pairs + kPairs - 1u) / kPairs), kJoinThreads, 0, stream>>>(a);
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
