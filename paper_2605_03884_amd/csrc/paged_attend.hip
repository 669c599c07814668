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
// The weights are held to 22 bits (fp16: high part and remainder; bf16, 8 bits each, high part and two remainders), scaled by 2^10 so that
// what fp16 loses below 2^-14 counts for nothing; maxima, sums and results are in 32 bits.
#include <algorithm>

#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr uint32_t kAttendThreads = 256;
constexpr uint32_t kAttendWaves = kAttendThreads / kWaveSize;
constexpr float kLift = 10.0f;                           // weights are 2^kLift times what they are

// Where a share begins: item and tile in the item.  `total`: tiles of all items.
struct Cursor {
  uint32_t row, inner, tile, tiles;                      // inner: kv head * blocks + block; tiles: of the item
  Seen seen;
};

__device__ inline uint32_t sum64(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readlane((int)wave_inclusive_scan(x), 63);
}

__device__ inline Seen row_seen(const PagedAttendArgs& a, uint32_t row) {
  return seen_by_last(held(a.p.lens[row], a.p.row_pages, a.p.page_shift), a.window, a.sinks);
}

// Tiles of all items.
__device__ inline uint32_t all_tiles(const PagedAttendArgs& a, uint32_t lane) {
  uint32_t sum = 0u;
  for (uint32_t row = lane; row < a.p.rows; row += kWaveSize) sum += seen_tiles(row_seen(a, row));
  return sum64(sum) * (a.p.kv_heads * a.blocks);
}

// The row that tile `at` falls into, and the tiles in front of that row.
__device__ inline uint32_t row_of_tile(const PagedAttendArgs& a, uint32_t lane, uint32_t at, uint32_t& before) {
  const uint32_t inner = a.p.kv_heads * a.blocks;
  before = 0u;
  for (uint32_t base = 0;; base += kWaveSize) {
    const uint32_t row = base + lane;
    const uint32_t mine = row < a.p.rows ? seen_tiles(row_seen(a, row)) * inner : 0u;
    const uint32_t upto = before + wave_inclusive_scan(mine);
    const uint64_t over = __builtin_amdgcn_ballot_w64(upto > at);
    if (over != 0ull || base + kWaveSize >= a.p.rows) {
      const uint32_t who = over ? (uint32_t)__builtin_ctzll(over) : (a.p.rows - 1u) % kWaveSize;
      before = (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), (int)who);
      return base + who;
    }
    before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
}

// The pages of a tile's tokens: lane l holds that of token l % 32; `counted` has a bit for each token that is seen and has a page.
template <bool SMALL>
__device__ inline uint32_t look_up(const PagedAttendArgs& a, uint32_t row, const TileRange& t, uint32_t lane) {
  const int32_t* entries = a.p.table + (uint64_t)row * a.p.row_pages;
  if constexpr (SMALL) {
    const uint32_t token = t.first + lane % kAttendTile;
    return token >= t.lo && token < t.hi ? (uint32_t)entries[token >> a.p.page_shift] : 0u;
  } else {
    return t.lo < t.hi ? (uint32_t)entries[t.first >> a.p.page_shift] : 0u;
  }
}

template <typename T, int D, bool SMALL>
__global__ __launch_bounds__(kAttendThreads) void attend_kernel(PagedAttendArgs a) {
  constexpr uint32_t kSteps = D / 32;                    // MFMAs along the head dimension
  constexpr uint32_t kSlabs = D / 16;                    // of 16 dimensions of the result
  constexpr uint32_t kLoads = kAttendTile * D / 8 / kWaveSize;         // 16-byte loads of V in a lane
  constexpr uint32_t kRowLanes = D / 8;                  // lanes that read one row of V
  constexpr uint32_t kRowsAtOnce = kWaveSize / kRowLanes;
  __shared__ __attribute__((aligned(256))) uint8_t lds[kAttendWaves][kAttendTile * D * 2];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 16u, g = lane / 16u;
  const uint32_t share = blockIdx.x * kAttendWaves + wave;
  const uint32_t inner_count = a.p.kv_heads * a.blocks, q_heads = a.p.kv_heads * a.rep;
  const uint32_t total = (uint32_t)__builtin_amdgcn_readfirstlane((int)all_tiles(a, lane));
  const Shares shares = deal(total, a.most);
  if (share >= shares.shares) return;
  uint32_t at = share_begin(shares, share);
  const uint32_t end = share_begin(shares, share + 1u);
  uint32_t before;
  uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)row_of_tile(a, lane, at, before));
  Seen seen = row_seen(a, row);
  uint32_t tiles = seen_tiles(seen);
  uint32_t inner = (at - before) / tiles, tile = (at - before) % tiles;
  uint8_t* mine = lds[wave];

  while (at < end) {
    // one item, or what of it falls into this share
    const uint32_t head = inner / a.blocks, block = inner % a.blocks;
    const uint32_t heads = min(16u, a.rep - block * 16u);
    const uint32_t from = tile, upto = min(tiles, tile + (end - at));
    const uint32_t hq = head * a.rep + block * 16u + n;                // this lane's query head, if n < heads
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

    const uint8_t* keys = a.p.k + (uint64_t)head * a.p.head_stride;
    const uint8_t* values = a.p.v + (uint64_t)head * a.p.head_stride;
    TileRange t = tile_range(seen, from);
    uint32_t page = look_up<SMALL>(a, row, t, lane);
    for (uint32_t i = from; i < upto; ++i) {
      // tokens that count
      const uint32_t token = t.first + lane % kAttendTile;
      const bool inside = token >= t.lo && token < t.hi, known = page < a.p.pages;
      const uint32_t counted = (uint32_t)__builtin_amdgcn_ballot_w64(inside && known);
      if ((uint32_t)__builtin_amdgcn_ballot_w64(inside && !known) != 0u && lane == 0u) flag(a.status, QKV_STATUS_BAD_PAGE);
      if (!(inside && known) && SMALL) page = 0u;
      if (!SMALL) page = (uint32_t)__builtin_amdgcn_readfirstlane((int)(known ? page : 0u));
      const uint32_t in_page = (1u << a.p.page_shift) - 1u;
      const auto row_at = [&](uint32_t of) -> uint64_t {               // byte offset of the tile's token `of`
        if constexpr (SMALL) {
          const uint32_t p = (uint32_t)__shfl((int)page, (int)of);
          return (uint64_t)p * a.p.page_stride + ((t.first + of) & in_page) * a.p.token_stride;
        } else {
          return (uint64_t)page * a.p.page_stride + ((t.first + of) & in_page) * a.p.token_stride;
        }
      };
      u32x4 kx[2][kSteps], vx[kLoads];
#pragma unroll
      for (uint32_t h = 0; h < 2u; ++h) {
        const uint8_t* p = keys + row_at(h * 16u + n) + g * 16u;
#pragma unroll
        for (uint32_t k = 0; k < kSteps; ++k) kx[h][k] = *reinterpret_cast<const u32x4*>(p + k * 64u);
      }
#pragma unroll
      for (uint32_t j = 0; j < kLoads; ++j) {
        const uint8_t* p = values + row_at(j * kRowsAtOnce + lane / kRowLanes) + (lane % kRowLanes) * 16u;
        vx[j] = *reinterpret_cast<const u32x4*>(p);
      }
      if (i + 1u < upto) {
        t = tile_range(seen, i + 1u);
        page = look_up<SMALL>(a, row, t, lane);
      }

      f32x4 s[2] = {(f32x4)(0.0f), (f32x4)(0.0f)};
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) {
        s[0] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[0][k]), q[k], s[0]);
        s[1] = T::mfma16(__builtin_bit_cast(typename T::x8, kx[1][k]), q[k], s[1]);
      }
      float e[8];
      float top = -INFINITY;
      if (counted == 0xFFFFFFFFu) {
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j) {
          e[j] = s[j / 4u][j % 4u];
          top = fmaxf(top, e[j] * a.scale_log2);
        }
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j) {
          e[j] = s[j / 4u][j % 4u];
          const float x = (counted >> (16u * (j / 4u) + 4u * g + j % 4u)) & 1u ? e[j] * a.scale_log2 : -INFINITY;
          top = fmaxf(top, x);
        }
      }
      top = max32(max16(top));
      const float m_new = fmaxf(m, top);
      const float less = m_new == -INFINITY ? 0.0f : m_new - kLift;    // what is taken off in the exponent
      if (__builtin_amdgcn_ballot_w64(m_new != m) != 0ull) {
        const float shrink = m == -INFINITY ? 0.0f : exp2f_(m - m_new);
        l *= shrink;
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) acc[d] *= shrink;
        m = m_new;
      }
      if (counted == 0xFFFFFFFFu) {
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j) e[j] = exp2f_(__builtin_fmaf(e[j], a.scale_log2, -less));
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j)
          e[j] = (counted >> (16u * (j / 4u) + 4u * g + j % 4u)) & 1u ? exp2f_(__builtin_fmaf(e[j], a.scale_log2, -less)) : 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; ++j) {                        // whatever stands in rows that do not count
          const bool counts = (counted >> (j * kRowsAtOnce + lane / kRowLanes)) & 1u;
          vx[j] = counts ? vx[j] : (u32x4)(0u);
        }
      }
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) l += e[j];
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

    l = sum32(sum16(l));
    if (from == 0u && upto == tiles) {                                 // the whole item
      const uint64_t at_head = (uint64_t)row * q_heads + hq;
      float scale = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
      float lse = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_log2f(l)) * 0.6931471805599453f;
      float other = 0.0f;
      if (a.prior_out && n < heads) join(lse, a.prior_lse[at_head], scale, other);
      if (n < heads) {
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) {
          f32x4 o = acc[d] * scale;
          const uint64_t where = at_head * D + d * 16u + g * 4u;
          if (a.prior_out && other != 0.0f) o += *reinterpret_cast<const f32x4*>(a.prior_out + where) * other;
          *reinterpret_cast<f32x4*>(a.out + where) = o;
        }
        if (a.lse && g == 0u) a.lse[at_head] = lse;
      }
    } else if (n < heads) {
      const uint64_t slot = ((uint64_t)row * inner_count + inner + share) * min(16u, a.rep) + n;
#pragma unroll
      for (uint32_t d = 0; d < kSlabs; ++d) *reinterpret_cast<f32x4*>(a.part_o + slot * D + d * 16u + g * 4u) = acc[d];
      if (g == 0u) *reinterpret_cast<f32x2*>(a.part_ml + slot * 2u) = (f32x2){m, l};
    }

    at += upto - from;
    tile = 0u;
    if (++inner == inner_count && at < end) {
      inner = 0u;
      ++row;
      seen = row_seen(a, row);
      tiles = seen_tiles(seen);
    }
  }
}

// Joins the parts of an item that was cut: a workgroup takes one query head of one item.
constexpr uint32_t kJoinThreads = 256;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(PagedAttendArgs a) {
  constexpr uint32_t kLanes = D / 4, kGroups = kJoinThreads / kLanes;  // a group of lanes goes through every kGroups-th part
  __shared__ f32x4 sums[kGroups][kLanes];
  __shared__ f32x2 tops[kGroups];
  const uint32_t lane = threadIdx.x % kWaveSize;
  const uint32_t heads = min(16u, a.rep), inner_count = a.p.kv_heads * a.blocks, q_heads = a.p.kv_heads * a.rep;
  const uint32_t item = blockIdx.x, row = item / inner_count, inner = item % inner_count;
  const uint32_t in_block = blockIdx.y, block = inner % a.blocks;
  if (block * 16u + in_block >= a.rep) return;
  uint32_t all = 0u, front = 0u;
  for (uint32_t r = lane; r < a.p.rows; r += kWaveSize) {
    const uint32_t x = seen_tiles(row_seen(a, r));
    all += x;
    front += r < row ? x : 0u;
  }
  const uint32_t total = sum64(all) * inner_count;
  const uint32_t tiles = seen_tiles(row_seen(a, row));
  const uint32_t begin = sum64(front) * inner_count + inner * tiles;
  const Shares shares = deal(total, a.most);
  const uint32_t first = share_of(shares, begin), last = share_of(shares, begin + tiles - 1u);
  if (first == last) return;                                           // finished where it was
  const uint32_t group = threadIdx.x / kLanes, at = threadIdx.x % kLanes;
  float m = -INFINITY, l = 0.0f;
  f32x4 o = (f32x4)(0.0f);
  for (uint32_t s = first + group; s <= last; s += kGroups) {
    const uint64_t slot = ((uint64_t)item + s) * heads + in_block;
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2u);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at * 4u);
    const float top = fmaxf(m, ml.x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top), take = ml.x == -INFINITY ? 0.0f : exp2f_(ml.x - top);
    l = l * keep + ml.y * take;
    o = o * keep + x * take;
    m = top;
  }
  sums[group][at] = o;
  if (at == 0u) tops[group] = (f32x2){m, l};
  __syncthreads();
  if (group != 0u) return;
#pragma unroll
  for (uint32_t k = 1; k < kGroups; ++k) {
    const f32x2 ml = tops[k];
    const float top = fmaxf(m, ml.x);
    const float keep = m == -INFINITY ? 0.0f : exp2f_(m - top), take = ml.x == -INFINITY ? 0.0f : exp2f_(ml.x - top);
    l = l * keep + ml.y * take;
    o = o * keep + sums[k][at] * take;
    m = top;
  }
  const uint64_t at_head = (uint64_t)row * q_heads + (inner / a.blocks) * a.rep + block * 16u + in_block;
  float scale = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  float lse = m == -INFINITY ? -INFINITY : (m - kLift + __builtin_log2f(l)) * 0.6931471805599453f;
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
  if ((1u << a.p.page_shift) < kAttendTile) attend_kernel<T, D, true><<<grid, kAttendThreads, 0, stream>>>(a);
  else attend_kernel<T, D, false><<<grid, kAttendThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && may_split) {
    attend_join_kernel<D><<<dim3(items, std::min(16u, a.rep)), kJoinThreads, 0, stream>>>(a);
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
