// paged_chosen.hip — attention of one new token of every sequence over the pages chosen for it, in one pass over their tokens.
//
//     s_t = scale * <q, K_t>,   out = sum_t softmax(s)_t V_t,   lse = log sum_t exp s_t,   t <= p in the pages whose bit is set, p = length - 1
//
// Work: an item is a (sequence, kv head, group of up to 16 query heads); one workgroup takes it, or where items are few several do, each a part.  The
// workgroup turns the item's bits into a list of page numbers in LDS - a word a thread, a prefix sum of the counts, a look at the table for all of them at
// once - so that small pages lie next to each other there and a tile of 32 tokens is full whatever pages it comes from.  The waves of all parts take the tiles in turn.
//
// A tile is what it is in attention over all pages (32 tokens a wave, keys from memory straight into the matrix instruction's operand, weights held to 22 bits,
// values through the transposing read of LDS; same layouts, same rounding, so results agree to the same bounds).  The waves' sums are joined in LDS, parts by a
// second kernel.
//
// What bounds it: memory where there is much to read, in pieces of a page's rows that lie anywhere.  48 rows with 64 pages of 16 of up to 8192 tokens, 8 kv heads of 128 dimensions: 40.5 us for
// 194 MB (4.8 TB/s, what a large copy reaches), and the same with keys and values through the caches, with items in the order of the dies, with two parts to an item.  Else
// the chain lengths - bits - entries - keys - values - two tiles: 131071 tokens of one row, 64 pages of 64: 11.8 us, 7.0 here and 4.2 - 5.3 to join 32 parts.  A row's
// entries read before the list is known, beside its bits, cost more than the trip to memory that they save (2000 entries of 4 rows: 9.9 us, so 9.5; of 48 rows 45.7, so 44.9).
#include <algorithm>

#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr uint32_t kChosenThreads = 256, kChosenWaves = kChosenThreads / kWaveSize;
constexpr uint32_t kChosenWords = kChosenThreads;        // words of a choice that are turned into a list at a time
constexpr uint32_t kChosenPages = kChosenWords * 32u;
constexpr uint32_t kNoPage = 0xFFFFFFFFu;

// RUN: tokens of a tile that surely lie in one page: 32, or 1 where pages are smaller.
template <typename T, int D, uint32_t RUN>
__global__ __launch_bounds__(kChosenThreads, D == 256 ? 1 : 2) void chosen_kernel(ChosenAttendArgs a) {
  constexpr uint32_t kSteps = D / 32, kSlabs = D / 16;
  constexpr uint32_t kLoads = kAttendTile * D / 8 / kWaveSize;         // 16-byte loads of V in a lane
  constexpr uint32_t kRowLanes = D / 8, kRowsAtOnce = kWaveSize / kRowLanes;
  __shared__ __attribute__((aligned(256))) uint8_t lds[kChosenWaves][kAttendTile * D * 2];      // values, then the waves' sums: 16 heads of D floats
  static_assert(kAttendTile * D * 2 == 16 * D * 4);
  __shared__ uint32_t list[kChosenPages];
  __shared__ f32x2 tops[kChosenWaves][16];
  __shared__ uint32_t counts[2][kChosenWaves];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 16u, g = lane / 16u;
  const uint32_t inner_count = a.p.kv_heads * a.blocks, q_heads = a.p.kv_heads * a.rep;
  const uint32_t item = blockIdx.x, row = item / inner_count, inner = item % inner_count, head = inner / a.blocks, block = inner % a.blocks;
  const uint32_t heads = min(16u, a.rep - block * 16u), hq = head * a.rep + block * 16u + n;      // this lane's query head, if n < heads
  const uint32_t length = held(a.p.lens[row], a.p.row_pages, a.p.page_shift);
  const uint32_t size = 1u << a.p.page_shift, all = length == 0u ? 0u : ((length - 1u) >> a.p.page_shift) + 1u;      // pages in sight
  const uint32_t in_last = length - (all == 0u ? 0u : (all - 1u) << a.p.page_shift);
  const uint32_t* bits = a.choice + ((uint64_t)row * a.p.kv_heads + head) * a.words;
  const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
  const uint8_t* keys = a.p.k + (uint64_t)head * a.p.head_stride;
  const uint8_t* values = a.p.v + (uint64_t)head * a.p.head_stride;
  uint8_t* mine = lds[wave];
  const auto in_sight = [&](uint32_t w, uint32_t x) -> uint32_t {      // of a word, the bits of pages that are in sight
    const uint32_t rest = all > w * 32u ? all - w * 32u : 0u;
    return rest < 32u ? x & ((1u << rest) - 1u) : x;
  };
  const auto word_at = [&](uint32_t w) -> uint32_t { return w * 32u < all ? in_sight(w, bits[w]) : 0u; };
  const uint32_t first_bits = threadIdx.x < a.words ? bits[threadIdx.x] : 0u;
  typename T::x8 q[kSteps];
#pragma unroll
  for (uint32_t k = 0; k < kSteps; ++k) {
    u32x4 x = (u32x4)(0u);
    if (n < heads) x = *reinterpret_cast<const u32x4*>(a.q + (uint64_t)row * a.q_token_stride + (uint64_t)hq * a.q_head_stride + (k * 32u + g * 8u) * 2u);
    q[k] = __builtin_bit_cast(typename T::x8, x);
  }
  f32x4 acc[kSlabs];
#pragma unroll
  for (uint32_t d = 0; d < kSlabs; ++d) acc[d] = (f32x4)(0.0f);
  float m = -INFINITY, l = 0.0f;

  uint32_t turn = 0u;
  for (uint32_t first_word = 0; first_word * 32u < all; first_word += kChosenWords) {
    // the list of this stretch's pages, in their order
    uint32_t word = first_word == 0u ? in_sight(threadIdx.x, first_bits) : word_at(first_word + threadIdx.x);
    const uint32_t upto = wave_inclusive_scan((uint32_t)__builtin_popcount(word));
    if (lane == kWaveSize - 1u) counts[turn][wave] = upto;
    __syncthreads();                                                   // nobody is at the last stretch's list any more
    uint32_t total = 0u, at = upto - (uint32_t)__builtin_popcount(word);
#pragma unroll
    for (uint32_t w = 0; w < kChosenWaves; ++w) {
      at += w < wave ? counts[turn][w] : 0u;
      total += counts[turn][w];
    }
    turn ^= 1u;
    total = (uint32_t)__builtin_amdgcn_readfirstlane((int)total);
    while (word != 0u) {
      list[at++] = (first_word + threadIdx.x) * 32u + (uint32_t)__builtin_ctz(word);
      word &= word - 1u;
    }
    __syncthreads();
    const bool own = total != 0u && list[total - 1u] == all - 1u;      // the page that need not be full is the last one
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < total; i += kChosenThreads) {
      const uint32_t page = (uint32_t)entries[list[i]];
      list[i] = page < a.p.pages ? page : kNoPage;
      if (page >= a.p.pages) flag(a.status, QKV_STATUS_BAD_PAGE);
    }
    __syncthreads();
    const uint64_t tokens = ((uint64_t)total << a.p.page_shift) - (own ? size - in_last : 0u);
    const uint32_t tiles = (uint32_t)((tokens + kAttendTile - 1u) / kAttendTile), step = a.parts * kChosenWaves;

    // A tile: its tokens that count (a bit each), and a lane's page (of token lane % 32, or of them all), which exists even where a token does not count.
    struct Tile {
      uint64_t first;
      uint32_t page, counted;
    };
    const auto tile_at = [&](uint32_t i) -> Tile {
      Tile t;
      t.first = (uint64_t)i * kAttendTile;
      const uint64_t token = t.first + lane % kAttendTile;
      const bool inside = token < tokens;
      const uint32_t page = inside ? list[(uint32_t)((RUN == 32u ? t.first : token) >> a.p.page_shift)] : kNoPage;
      t.counted = (uint32_t)__builtin_amdgcn_ballot_w64(page != kNoPage);
      t.page = page != kNoPage ? page : 0u;
      return t;
    };
    const auto row_at = [&](const uint8_t* pool, const Tile& t, uint32_t of, uint32_t piece) -> const uint8_t* {
      if constexpr (RUN == 32u)
        return pool + (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)t.page) * a.p.page_stride + ((uint32_t)t.first & (size - 1u)) * a.p.token_stride +
               (of * (uint32_t)a.p.token_stride + piece);
      const uint32_t page = (uint32_t)__shfl((int)t.page, (int)of);
      return pool + (uint64_t)page * a.p.page_stride + (uint64_t)(((uint32_t)t.first + of) & (size - 1u)) * a.p.token_stride + piece;
    };
    u32x4 kx[2][kSteps], vx[kLoads];
    const auto load_keys = [&](const Tile& t) {
#pragma unroll
      for (uint32_t h = 0; h < 2u; ++h) {
        const uint8_t* p = row_at(keys, t, h * 16u + n, g * 16u);
#pragma unroll
        for (uint32_t k = 0; k < kSteps; ++k) kx[h][k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + k * 64u));
      }
    };
    const auto load_values = [&](const Tile& t) {
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j)
        vx[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row_at(values, t, j * kRowsAtOnce + lane / kRowLanes, (lane % kRowLanes) * 16u)));
    };
    const uint32_t begin = blockIdx.y * kChosenWaves + wave;
    Tile now{};
    if (begin < tiles) {
      now = tile_at(begin);
      load_keys(now);
      load_values(now);
    }
    for (uint32_t i = begin; i < tiles; i += step) {
      const uint32_t counted = now.counted;
      f32x4 s[2] = {(f32x4)(0.0f), (f32x4)(0.0f)};
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) {
        s[0] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[0][k]), q[k], s[0]);
        s[1] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[1][k]), q[k], s[1]);
      }
      // the registers of K are free: the next tile's keys are on their way while this one's weights are worked out
      const bool more = i + step < tiles && i + step > i;
      if (more) {
        now = tile_at(i + step);
        load_keys(now);
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
      if (more) load_values(now);
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
      if (!more) break;
    }
  }

  // Values that are infinite or no number.  Their products are whatever the parts of a weight make of them (0 times infinity is no number), so a dimension
  // that they have spoilt becomes the sum of all such values that are seen, whatever they weigh: of the whole item, which adds up to the same.
  f32x4 zero = (f32x4)(0.0f);                                          // stays that only where all are numbers
#pragma unroll
  for (uint32_t d = 0; d < kSlabs; ++d) zero += acc[d] * 0.0f;
  const bool spoilt = n < heads && !(zero.x + zero.y + zero.z + zero.w == 0.0f);      // (places without a query head meet infinite keys with zeros)
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(spoilt) != 0ull, 0)) {
    f32x4 odd[kSlabs];
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d) odd[d] = (f32x4)(0.0f);
    for (uint32_t w = 0; w * 32u < all; ++w) {
      for (uint32_t word = word_at(w); word != 0u; word &= word - 1u) {
        const uint32_t j = w * 32u + (uint32_t)__builtin_ctz(word), page = (uint32_t)entries[j];
        if (page >= a.p.pages) continue;
        const uint32_t here = j == all - 1u ? in_last : size;
        for (uint32_t i = 0; i < here; ++i) {
          const uint8_t* p = values + (uint64_t)page * a.p.page_stride + (uint64_t)i * a.p.token_stride + g * 8u;
#pragma unroll
          for (uint32_t d = 0; d < kSlabs; ++d) {
            const typename T::x4 v = *reinterpret_cast<const typename T::x4*>(p + d * 32u);
#pragma unroll
            for (uint32_t k = 0; k < 4u; ++k)
              if (!(__builtin_fabsf((float)v[k]) < INFINITY)) odd[d][k] += (float)v[k];
          }
        }
      }
    }
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k)
        if (!(__builtin_fabsf(odd[d][k]) < INFINITY)) acc[d][k] = odd[d][k];
  }
  l = sum32(sum16(l));

  // the waves' sums, joined: a thread takes four dimensions of a head
  __builtin_amdgcn_wave_barrier();
  if (n < heads) {
#pragma unroll
    for (uint32_t d = 0; d < kSlabs; ++d) *reinterpret_cast<f32x4*>(mine + (n * D + d * 16u + g * 4u) * 4u) = acc[d];
    if (g == 0u) tops[wave][n] = (f32x2){m, l};
  }
  __syncthreads();
  for (uint32_t piece = threadIdx.x; piece < heads * (D / 4u); piece += kChosenThreads) {
    const uint32_t h = piece / (D / 4u), at = piece % (D / 4u);
    float top = -INFINITY, sum = 0.0f;
    f32x4 o = (f32x4)(0.0f);
#pragma unroll
    for (uint32_t w = 0; w < kChosenWaves; ++w) top = fmaxf(top, tops[w][h].x);
#pragma unroll
    for (uint32_t w = 0; w < kChosenWaves; ++w) {
      const f32x2 ml = tops[w][h];
      const float take = ml.x == -INFINITY ? 0.0f : exp2f_(ml.x - top);
      sum += ml.y * take;
      o += *reinterpret_cast<const f32x4*>(lds[w] + (h * D + at * 4u) * 4u) * take;
    }
    keep_odd(o, kChosenWaves, [&](uint32_t w) { return *reinterpret_cast<const f32x4*>(lds[w] + (h * D + at * 4u) * 4u); });
    if (a.parts != 1u) {
      const uint64_t slot = ((uint64_t)item * a.parts + blockIdx.y) * min(16u, a.rep) + h;
      *reinterpret_cast<f32x4*>(a.part_o + slot * D + at * 4u) = o;
      if (at == 0u) *reinterpret_cast<f32x2*>(a.part_ml + slot * 2u) = (f32x2){top, sum};
      continue;
    }
    const uint64_t at_head = (uint64_t)row * q_heads + head * a.rep + block * 16u + h;
    float scale = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum);
    float lse = top == -INFINITY ? -INFINITY : (top - T::kLift + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    float other = 0.0f;
    if (a.prior_out) join(lse, a.prior_lse[at_head], scale, other);
    o = weighed(o, scale);
    if (a.prior_out && other != 0.0f) o += *reinterpret_cast<const f32x4*>(a.prior_out + at_head * D + at * 4u) * other;
    *reinterpret_cast<f32x4*>(a.out + at_head * D + at * 4u) = o;
    if (a.lse && at == 0u) a.lse[at_head] = lse;
  }
}

// Joins the parts of a query head: D / 4 lanes each, as many heads of an item as fit a workgroup.
constexpr uint32_t kChosenJoin = 256;
template <int D>
__global__ __launch_bounds__(kChosenJoin) void chosen_join_kernel(ChosenAttendArgs a, float lift) {
  constexpr uint32_t kLanes = D / 4, kAtOnce = 8;
  const uint32_t heads = min(16u, a.rep), inner_count = a.p.kv_heads * a.blocks, item = blockIdx.x, row = item / inner_count, inner = item % inner_count;
  const uint32_t block = inner % a.blocks, h = blockIdx.y * (kChosenJoin / kLanes) + threadIdx.x / kLanes, at = threadIdx.x % kLanes;
  if (h >= heads || block * 16u + h >= a.rep) return;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = (f32x4)(0.0f);
  for (uint32_t s = 0; s < a.parts; s += kAtOnce) {
    f32x2 ml[kAtOnce];
    f32x4 x[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint64_t slot = ((uint64_t)item * a.parts + min(s + k, a.parts - 1u)) * heads + h;       // past the last one: the last one, without weight
      ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
      x[k] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
    }
    float top = m;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k)
      if (s + k < a.parts) top = fmaxf(top, ml[k].x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top);
    l *= keep;
    o *= keep;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      if (s + k >= a.parts) continue;
      const float take = ml[k].x == -INFINITY ? 0.0f : exp2f_(ml[k].x - top);
      l += ml[k].y * take;
      o += x[k] * take;
    }
    m = top;
  }
  keep_odd(o, a.parts, [&](uint32_t s) { return *reinterpret_cast<const f32x4*>(a.part_o + (((uint64_t)item * a.parts + s) * heads + h) * D + at * 4u); });
  const uint64_t at_head = (uint64_t)row * a.p.kv_heads * a.rep + (inner / a.blocks) * a.rep + block * 16u + h;
  float scale = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
  float lse = m == -INFINITY ? -INFINITY : (m - lift + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  float other = 0.0f;
  if (a.prior_out) join(lse, a.prior_lse[at_head], scale, other);
  o = weighed(o, scale);
  if (a.prior_out && other != 0.0f) o += *reinterpret_cast<const f32x4*>(a.prior_out + at_head * D + at * 4u) * other;
  *reinterpret_cast<f32x4*>(a.out + at_head * D + at * 4u) = o;
  if (a.lse && at == 0u) a.lse[at_head] = lse;
}

template <typename T, int D>
hipError_t launch_chosen_of(const ChosenAttendArgs& a, hipStream_t stream) {
  const uint32_t items = a.p.rows * a.p.kv_heads * a.blocks;
  const dim3 grid(items, a.parts);
  if (a.p.page_shift >= 5u) chosen_kernel<T, D, 32u><<<grid, kChosenThreads, 0, stream>>>(a);
  else chosen_kernel<T, D, 1u><<<grid, kChosenThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1u) return e;
  const uint32_t heads = std::min(16u, a.rep), together = kChosenJoin / (D / 4u);
  chosen_join_kernel<D><<<dim3(items, (heads + together - 1u) / together), kChosenJoin, 0, stream>>>(a, T::kLift);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_chosen_type(const ChosenAttendArgs& a, uint32_t head_dim, hipStream_t stream) {
  if (head_dim == 64u) return launch_chosen_of<T, 64>(a, stream);
  if (head_dim == 128u) return launch_chosen_of<T, 128>(a, stream);
  return launch_chosen_of<T, 256>(a, stream);
}

}  // namespace

hipError_t launch_paged_attend_chosen(const ChosenAttendArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  return bf16 ? launch_chosen_type<BFloat>(a, head_dim, stream) : launch_chosen_type<Half>(a, head_dim, stream);
}

}  // namespace qkv
