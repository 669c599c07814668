// paged_prompt.hip — attention of many new tokens of every sequence over its pages: each sees what stands up to its own place, with a window
// the last `window` tokens and the first `sinks`.
//
// Work: a workgroup takes a tile of up to 128 (query token, query head) pairs of one kv head, so that a key is read once for all query
// heads that share it, and goes through the keys they see 64 at a time, with a running maximum m, sum l and sum of p.V.  Four waves
// of 32 pairs; where there are few query tiles the keys are split as well, and a second kernel joins the parts.
//
// A tile of 64 keys, one wave (lane = 32 h + n; n is the lane's pair):
//   staging  rows of K and V are loaded into registers while the tile before is worked on, and stored into one of two places in LDS: K in
//            16-byte pieces exchanged by token, V in 64-byte pieces, so that no read below meets a bank twice.
//   scores   S^T = K Q^T on v_mfma_f32_32x32x16: a lane gets 32 scores of its own pair.
//   softmax  in the lane, and with the lane 32 further on.  m follows the true maximum only when that has grown by 2^8: sums are
//            kept relative to m, and the weights have 2^7 of room below and 2^8 above before fp16 could overflow.
//   values   O^T = V^T P^T: the weights are where the product wants them; V^T comes out of LDS through the transposing read.
// The weights are rounded to the cache's type, as the result is: their errors average out over the keys and stay at the size of the result's own rounding.
#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

constexpr uint32_t kThreads = 256;
constexpr float kLift = 7.0f, kSlack = 8.0f;

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

// Whether one of eight values is infinite or no number.
template <typename T>
__device__ inline bool not_finite(u32x4 x) {
  constexpr uint32_t e = T::kExponent;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad = bad || (x[i] & e) == e || (x[i] & (e << 16)) == (e << 16);
  return bad;
}

template <typename T, int D, bool SMALL, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void prompt_kernel(PagedPromptArgs a) {
  constexpr uint32_t kKeys = kPromptKeys, kChunks = D / 8;             // 16-byte pieces of a row
  constexpr uint32_t kLoads = kKeys * kChunks / kThreads;              // of them a thread loads, of K and of V
  constexpr uint32_t kRowsAtOnce = kThreads / kChunks;
  constexpr uint32_t kSteps = D / 16, kSlabs = D / 32;
  struct Place {
    uint8_t k[kKeys * D * 2], v[kKeys * D * 2];
  };
  __shared__ __attribute__((aligned(256))) Place place[2];
  __shared__ __attribute__((aligned(16))) uint32_t marks[2][4];        // tokens without a page; tokens with infinities or NaN among their values
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
  // whether every one of the queries at places [lo, hi] sees all of the tile's keys, or none of them sees any
  const auto whole = [&](int32_t t, int32_t lo, int32_t hi) { return t + (int32_t)kKeys - 1 <= lo && (window == 0 || t > hi - window || t + (int32_t)kKeys <= sinks); };
  const auto nothing = [&](int32_t t, int32_t lo, int32_t hi) {
    return t > hi || (window != 0 && t + (int32_t)kKeys - 1 <= lo - window && t >= sinks);
  };

  // the lane's pair
  const uint32_t pair = wave * 32u + n, token = pair / a.rep, head_in = pair % a.rep;
  const bool live = token < here;
  const int32_t mine = live ? base + (int32_t)token : -1;
  const uint32_t wave_first = wave * 32u / a.rep, wave_last = min((wave * 32u + 31u) / a.rep, here - 1u);
  const bool wave_live = wave_first < here;
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
  uint32_t absent = 0u;                                                // bit j: nobody sees the thread's j-th row, or (16 + j too) it has no page

  const auto load = [&](uint32_t i) {
    const int32_t t = tile_at(i);
    absent = 0u;
    uint32_t page_of_tile = 0u;
    if constexpr (!SMALL) page_of_tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)entries[(uint32_t)t >> a.p.page_shift]);
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) {
      const int32_t key = t + (int32_t)(j * kRowsAtOnce + my_row);
      const bool wanted = key < reach && (key >= win_lo || key < (int32_t)sink_end);       // somebody sees it
      uint32_t page = page_of_tile;
      if constexpr (SMALL) page = wanted ? (uint32_t)entries[(uint32_t)key >> a.p.page_shift] : 0u;
      const bool there = wanted && page < a.p.pages;
      if (!there) absent |= (wanted ? 0x10001u : 1u) << j;
      const uint64_t where = (uint64_t)(there ? page : 0u) * a.p.page_stride + (uint64_t)((uint32_t)key & in_page) * a.p.token_stride + my_chunk * 16u;
      kx[j] = *reinterpret_cast<const u32x4*>(keys + where);
      vx[j] = *reinterpret_cast<const u32x4*>(values + where);
    }
  };
  const auto store = [&](uint32_t i, uint32_t side) {
    const int32_t t = tile_at(i);
    const bool careful = !whole(t, base, reach - 1);                   // only there can a value meet a weight that has to be nothing
#pragma unroll
    for (uint32_t j = 0; j < kLoads; ++j) {
      const uint32_t of = j * kRowsAtOnce + my_row;
      if (absent != 0u && (absent >> j & 1u)) {
        vx[j] = (u32x4)(0u);
        if ((absent >> (16u + j) & 1u) && my_chunk == 0u) {
          atomicOr(&marks[side][of / 32u], 1u << (of % 32u));
          flag(a.status, QKV_STATUS_BAD_PAGE);
        }
      }
      if (careful && not_finite<T>(vx[j])) {
        vx[j] = (u32x4)(0u);
        atomicOr(&marks[side][2u + of / 32u], 1u << (of % 32u));
      }
      *reinterpret_cast<u32x4*>(place[side].k + key_at<D>(of, my_chunk)) = kx[j];
      *reinterpret_cast<u32x4*>(place[side].v + value_at<D>(of, my_chunk / 4u) + (my_chunk % 4u) * 16u) = vx[j];
    }
  };

  if (threadIdx.x < 8u) marks[threadIdx.x / 4u][threadIdx.x % 4u] = 0u;
  __syncthreads();
  if (first_tile < last_tile) {
    load(first_tile);
    store(first_tile, 0u);
    if (first_tile + 1u < last_tile) load(first_tile + 1u);
  }
  __syncthreads();
  for (uint32_t i = first_tile; i < last_tile; ++i) {
    const uint32_t side = (i - first_tile) & 1u;
    const int32_t t = tile_at(i);
    const u32x4 marked = *reinterpret_cast<const u32x4*>(marks[side]);
    if (wave_live && !nothing(t, wave_lo, wave_hi)) {
      const uint8_t* const ks = place[side].k;
      const uint8_t* const vs = place[side].v;
      f32x16 s[2] = {(f32x16)(0.0f), (f32x16)(0.0f)};
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) {
#pragma unroll
        for (uint32_t u = 0; u < 2u; ++u) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(ks + key_at<D>(u * 32u + n, k * 2u + h));
          s[u] = T::mfma32(__builtin_bit_cast(typename T::x8, x), q[k], s[u]);
        }
      }
      const bool all = whole(t, wave_lo, wave_hi) && (marked.x | marked.y) == 0u;
      if (!all) {
        const int32_t up = mine - t - 4 * (int32_t)h, low = window != 0 ? up - window : -1 - 4 * (int32_t)h - (int32_t)kKeys, sink = window != 0 ? sinks - t - 4 * (int32_t)h : 0;
#pragma unroll
        for (uint32_t u = 0; u < 2u; ++u)
#pragma unroll
          for (uint32_t j = 0; j < 16u; ++j) {
            const int32_t c = (int32_t)(u * 32u + 8u * (j / 4u) + j % 4u);
            bool seen = c <= up && (c > low || c < sink);
            if (marked[u] >> (8u * (j / 4u) + j % 4u + 4u * h) & 1u) seen = false;
            s[u][j] = seen ? s[u][j] : -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (uint32_t j = 1; j < 32u; ++j) top = fmaxf(top, s[j / 16u][j % 16u]);
      top = max32(top) * a.scale_log2;
      if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0ull) {     // m is -inf at first
        const float next = fmaxf(m, top);
        const float shrink = m == -INFINITY ? 0.0f : exp2f_(m - next);
        l *= shrink;
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) acc[d] *= shrink;
        m = next;
      }
      const float less = m == -INFINITY ? 0.0f : m - kLift;
      typename T::x8 w[4];
#pragma unroll
      for (uint32_t u = 0; u < 4u; ++u) {
        float e[8];
#pragma unroll
        for (uint32_t j = 0; j < 8u; ++j) {
          e[j] = exp2f_(__builtin_fmaf(s[u / 2u][8u * (u % 2u) + j], a.scale_log2, -less));
          l += e[j];
          w[u][j] = (typename T::one)e[j];
        }
        if (__builtin_expect((marked.z | marked.w) != 0u, 0)) {
#pragma unroll
          for (uint32_t j = 0; j < 8u; ++j) s[u / 2u][8u * (u % 2u) + j] = e[j];
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < 4u; ++u) {
        const uint32_t r = u * 16u + 4u * h + (lane % 16u) / 4u;       // token of the first four
#pragma unroll
        for (uint32_t d = 0; d < kSlabs; ++d) {
          const uint32_t in_piece = (lane / 16u % 2u) * 32u + (lane % 4u) * 8u;
          const u32x2 lo = read_turned(vs + value_at<D>(r, d) + in_piece);
          const u32x2 hi = read_turned(vs + value_at<D>(r + 8u, d) + in_piece);
          acc[d] = T::mfma32(__builtin_bit_cast(typename T::x8, (u32x4){lo.x, lo.y, hi.x, hi.y}), w[u], acc[d]);
        }
      }
      if (__builtin_expect((marked.z | marked.w) != 0u, 0)) {
        // Values that are infinite or no number were left out above (with the seven beside them): they count for the pairs that give
        // them a weight, and for no other.
        for (uint32_t word = 0; word < 2u; ++word) {
          uint32_t left = word ? marked.w : marked.z;
          while (left != 0u) {
            const uint32_t bit = (uint32_t)__builtin_ctz(left), key = (uint32_t)t + word * 32u + bit;
            left &= left - 1u;
            float weight = 0.0f;
#pragma unroll
            for (uint32_t j = 0; j < 16u; ++j) {
              const float x = word ? s[1][j] : s[0][j];
              if (8u * (j / 4u) + j % 4u + 4u * h == bit) weight = x;
            }
            weight = sum32(weight);                                    // one of the two lanes has it
            if (key >= (uint32_t)length) continue;
            const uint32_t page = (uint32_t)entries[key >> a.p.page_shift];
            if (page >= a.p.pages) continue;
            const uint8_t* from = values + (uint64_t)page * a.p.page_stride + (uint64_t)(key & in_page) * a.p.token_stride;
#pragma unroll
            for (uint32_t d = 0; d < kSlabs; ++d)
#pragma unroll
              for (uint32_t j = 0; j < 4u; ++j) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(from + (d * 4u + j) * 16u);
                if (not_finite<T>(x) && weight != 0.0f) {
                  const typename T::x8 v = __builtin_bit_cast(typename T::x8, x);
#pragma unroll
                  for (uint32_t e = 0; e < 4u; ++e) acc[d][4u * j + e] += weight * (float)(h ? v[4u + e] : v[e]);
                }
              }
          }
        }
      }
    }
    if (i + 1u < last_tile) {
      store(i + 1u, side ^ 1u);
      if (i + 2u < last_tile) load(i + 2u);
    }
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane((int)(marked.x | marked.y | marked.z | marked.w)) != 0) {       // the same for all
      if (threadIdx.x < 4u) marks[side][threadIdx.x] = 0u;
      __syncthreads();
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
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void prompt_join_kernel(PagedPromptArgs a) {
  constexpr uint32_t kLanes = D / 4;
  const uint64_t all = (uint64_t)a.tokens * (a.p.kv_heads * a.rep);
  const uint64_t pair = (uint64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
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

template <typename T, int D>
hipError_t launch_prompt_of(const PagedPromptArgs& a, hipStream_t stream) {
  const bool small = (1u << a.p.page_shift) < kPromptKeys;
  const dim3 grid(places(a.tokens, a.p.rows, a.per) * a.p.kv_heads, a.splits);
  if (a.splits == 1u) {
    if (small) prompt_kernel<T, D, true, false><<<grid, kThreads, 0, stream>>>(a);
    else prompt_kernel<T, D, false, false><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  if (small) prompt_kernel<T, D, true, true><<<grid, kThreads, 0, stream>>>(a);
  else prompt_kernel<T, D, false, true><<<grid, kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint64_t pairs = (uint64_t)a.tokens * (a.p.kv_heads * a.rep);
  prompt_join_kernel<T, D><<<(uint32_t)((pairs + kThreads / (D / 4) - 1u) / (kThreads / (D / 4))), kThreads, 0, stream>>>(a);
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
