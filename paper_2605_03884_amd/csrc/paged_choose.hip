// paged_choose.hip — which pages a query reads: scores of all pages in whole numbers, and the highest of them.
//
//     P_d = sum_r max(q_rd, 0),  N_d = sum_r min(q_rd, 0),  x = max_d (floor log2 max(P_d, -N_d) + e_d)
//     p_d = min(127, rne(P_d 2^(e_d - x + 6))),  n_d likewise;   score_j = sum_d p_d hi_jd + n_d lo_jd
//
// A score is a product of two rows of 2 D codes, so the scores of 16 pages with 16 tokens are one chain of v_mfma_i32_16x16x64_i8, which reads the digests as they lie
// in memory.  It is below 2^23 (127 * 128 * 2 * 256) and exact.
//
// First kernel: a workgroup takes a tile of query tokens of one kv head and a stretch of pages, works the tokens' codes out into LDS and goes through the pages, 16 a
// wave.  Second kernel: a token and kv head is a wave's or a workgroup's; its scores stay in registers while bisection finds the score of the last page
// that is chosen, and a ballot writes 64 bits of the choice at once.
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
  t.row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return first_place((uint32_t)a.starts[b], b, a.per) <= at; }));
  const int32_t start = a.starts[t.row], end = a.starts[t.row + 1u];
  if (start < 0 || end < start || (uint32_t)end > a.tokens) {
    if (tell) flag(a.status, QKV_STATUS_BAD_ROW);
    return t;
  }
  const uint32_t count = (uint32_t)(end - start), first = first_place((uint32_t)start, t.row, a.per), skip = (at - first) * a.per;
  if (at < first || skip >= count) return t;
  t.here = min(a.per, count - skip);
  t.query = (uint32_t)start + skip;
  t.base = (int32_t)held(a.p.lens[t.row], a.p.row_pages, a.p.page_shift) - (int32_t)count + (int32_t)skip;
  if (t.base < 0 && tell) flag(a.status, QKV_STATUS_BAD_ROW);
  return t;
}

__device__ inline int32_t wave_max(int32_t x) {
#pragma unroll
  for (uint32_t across = 1; across < kWaveSize; across *= 2u) x = max(x, __shfl_xor(x, (int)across));
  return x;
}
__device__ inline int32_t wave_min(int32_t x) {
#pragma unroll
  for (uint32_t across = 1; across < kWaveSize; across *= 2u) x = min(x, __shfl_xor(x, (int)across));
  return x;
}

// Codes of one token's queries to LDS, a wave: lane l has the channels l D / 64 and on.
template <typename T, int D>
__device__ inline void query_codes(const ChooseArgs& a, uint32_t token, uint32_t head, uint32_t lane, int8_t* to) {
  constexpr int kEach = D / 64;
  float above[kEach], below[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) above[i] = below[i] = 0.0f;
  const uint8_t* q = a.q + (uint64_t)token * a.q_token_stride + (uint64_t)head * a.rep * a.q_head_stride + lane * kEach * 2u;
  struct Values {
    typename T::one v[kEach];
  };
  for (uint32_t r = 0; r < a.rep; ++r) {
    const Values x = *reinterpret_cast<const Values*>(q + (uint64_t)r * a.q_head_stride);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      above[i] += fmaxf((float)x.v[i], 0.0f);            // no number: 0
      below[i] += fminf((float)x.v[i], 0.0f);
    }
  }
  int32_t e[kEach], height = INT32_MIN;
  const int8_t* exponents = a.exponents + (uint64_t)head * D + lane * kEach;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    above[i] = fminf(above[i], 3.40282347e38f);
    below[i] = fmaxf(below[i], -3.40282347e38f);
    e[i] = exponents[i];
    const float most = fmaxf(above[i], -below[i]);
    if (most > 0.0f) height = max(height, __builtin_amdgcn_frexp_expf(most) - 1 + e[i]);
  }
  height = wave_max(height);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int32_t by = height == INT32_MIN ? 0 : e[i] - height + 6;
    to[lane * kEach + i] = (int8_t)fminf(__builtin_rintf(__builtin_amdgcn_ldexpf(above[i], by)), 127.0f);
    to[D + lane * kEach + i] = (int8_t)fmaxf(__builtin_rintf(__builtin_amdgcn_ldexpf(below[i], by)), -127.0f);
  }
}

// GROUPS: 16 tokens each.  Pages [blockIdx.y * chunk, + chunk) of the row.
template <typename T, int D, uint32_t GROUPS>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ChooseArgs a, uint32_t chunk) {
  constexpr uint32_t kSteps = 2u * D / 64u, kRow = 2u * D + 16u;       // 16 bytes between the tokens: 16 lanes that read one piece of theirs meet every bank once
  __shared__ __attribute__((aligned(16))) int8_t codes[GROUPS * 16u][kRow];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t n = lane % 16u, g = lane / 16u;
  const uint32_t tile = blockIdx.x / a.p.kv_heads, head = blockIdx.x % a.p.kv_heads;
  const QueryTile t = query_tile(a, a.first_tile + tile, lane, false);
  const int32_t last_place = t.base + (int32_t)t.here - 1;
  if (t.here == 0u || last_place < 0) return;
  const uint32_t all = ((uint32_t)last_place >> a.p.page_shift) + 1u;  // pages in sight
  const uint32_t begin = max(blockIdx.y * chunk, a.first & ~15u), end = min((blockIdx.y + 1u) * chunk, all > a.last ? all - a.last : 0u);
  if (begin >= end) return;                                            // what has no score is chosen anyway
  for (uint32_t token = wave; token < GROUPS * 16u; token += kScoreWaves) {
    if (token >= t.here) break;
    query_codes<T, D>(a, t.query + token, head, lane, codes[token]);
  }
  __syncthreads();
  i32x4 q[GROUPS][kSteps];
#pragma unroll
  for (uint32_t c = 0; c < GROUPS; ++c)
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
      q[c][k] = (i32x4)(0);
      if (c * 16u + n < t.here) q[c][k] = *reinterpret_cast<const i32x4*>(codes[c * 16u + n] + k * 64u + g * 16u);
    }
  const int32_t* entries = a.p.table + (uint64_t)t.row * a.p.row_pages;
  int32_t* scores = a.scores + (((uint64_t)tile * a.per) * a.p.kv_heads + head) * a.stride;
  const uint64_t next_token = (uint64_t)a.p.kv_heads * a.stride;
  for (uint32_t at = begin + wave * 16u; at < end; at += kScoreWaves * 16u) {
    const uint32_t j = at + n;
    const uint32_t page = j < end ? (uint32_t)entries[j] : 0xFFFFFFFFu;
    const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(page < a.p.pages) & 0xFFFFu;
    const int8_t* row = a.digest + ((uint64_t)(page < a.p.pages ? page : 0u) * a.p.kv_heads + head) * (2u * D) + g * 16u;
    i32x4 x[kSteps], s[GROUPS];
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) x[k] = *reinterpret_cast<const i32x4*>(row + k * 64u);
#pragma unroll
    for (uint32_t c = 0; c < GROUPS; ++c) {
      s[c] = (i32x4)(0);
#pragma unroll
      for (uint32_t k = 0; k < kSteps; ++k) s[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[k], q[c][k], s[c], 0, 0, 0);
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i) s[c][i] = there >> (4u * g + i) & 1u ? s[c][i] : kAbsent;
      if (c * 16u + n < t.here) *reinterpret_cast<i32x4*>(scores + (c * 16u + n) * next_token + at + 4u * g) = s[c];
    }
  }
}

// WAVES share a (token, kv head); with KEEP blocks of 64 scores a wave keeps them in registers, where they are no more than that, else they are read again.
template <uint32_t WAVES, uint32_t KEEP>
__global__ __launch_bounds__(WAVES == 1u ? 256u : WAVES * kWaveSize) void choose_kernel(ChooseArgs a) {
  constexpr uint32_t kUnits = WAVES == 1u ? 4u : 1u;                   // of a workgroup
  __shared__ int32_t shared[2][16];
  const uint32_t lane = threadIdx.x % kWaveSize, wave_of = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t wave = WAVES == 1u ? 0u : wave_of;
  const uint64_t unit = (uint64_t)blockIdx.x * kUnits + (WAVES == 1u ? wave_of : 0u);
  const uint32_t pairs = a.per * a.p.kv_heads, tile = (uint32_t)(unit / pairs), in_tile = (uint32_t)(unit % pairs);
  if (tile >= a.tiles) return;
  const uint32_t token = in_tile / a.p.kv_heads, head = in_tile % a.p.kv_heads;
  const QueryTile t = query_tile(a, a.first_tile + tile, lane, in_tile == 0u && wave == 0u && lane == 0u);
  if (token >= t.here) return;
  const int32_t place = t.base + (int32_t)token;
  const uint32_t all = place < 0 ? 0u : ((uint32_t)place >> a.p.page_shift) + 1u;
  const uint32_t scored = all > a.last ? all - a.last : 0u;            // pages from here on are chosen, as those in front of `first` are
  const int32_t* entries = a.p.table + (uint64_t)t.row * a.p.row_pages;
  const int32_t* scores = a.scores + (((uint64_t)tile * a.per + token) * a.p.kv_heads + head) * a.stride;
  uint32_t* choice = a.choice + ((uint64_t)(t.query + token) * a.p.kv_heads + head) * a.words;
  const uint32_t blocks = (all + 63u) / 64u, each = (blocks + WAVES - 1u) / WAVES, from = min(wave * each, blocks), upto = min(from + each, blocks);
  const bool kept = each <= KEEP;
  int32_t keep[KEEP];
  const auto read = [&](uint32_t block) -> int32_t {
    const uint32_t j = block * 64u + lane;
    if (j >= all) return kAbsent;
    if (j >= a.first && j < scored) return scores[j];
    return (uint32_t)entries[j] < a.p.pages ? kAlways : kAbsent;
  };
  int32_t low = kAlways, high = kAbsent;
  uint32_t present = 0u;
  const auto look = [&](int32_t x) {
    present += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(x != kAbsent));
    if (x != kAbsent && x != kAlways) {
      low = min(low, x);
      high = max(high, x);
    }
  };
  if (kept) {
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i) keep[i] = from + i < upto ? read(from + i) : kAbsent;
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i) look(keep[i]);
  } else {
    for (uint32_t i = from; i < upto; ++i) look(read(i));
  }
  // sums and extremes over the waves that share; the same in all lanes
  uint32_t turn = 0u;
  const auto together = [&](int32_t x, auto join) -> int32_t {
    if constexpr (WAVES == 1u) return x;
    if (lane == 0u) shared[turn][wave] = x;
    __syncthreads();
    int32_t got = shared[turn][0];
    for (uint32_t w = 1; w < WAVES; ++w) got = join(got, shared[turn][w]);
    turn ^= 1u;
    return got;
  };
  const auto add = [](int32_t x, int32_t y) { return x + y; };
  low = together(wave_min(low), [](int32_t x, int32_t y) { return min(x, y); });
  high = together(wave_max(high), [](int32_t x, int32_t y) { return max(x, y); });
  present = (uint32_t)together((int32_t)present, add);
  low = __builtin_amdgcn_readfirstlane(low);
  high = __builtin_amdgcn_readfirstlane(high);
  present = (uint32_t)__builtin_amdgcn_readfirstlane((int)present);
  const auto count = [&](int32_t least) -> uint32_t {
    uint32_t sum = 0u;
    if (kept) {
#pragma unroll
      for (uint32_t i = 0; i < KEEP; ++i) sum += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(keep[i] >= least));
    } else {
      for (uint32_t i = from; i < upto; ++i) sum += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(read(i) >= least));
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)together((int32_t)sum, add));
  };
  // The largest value that at least `most` keys reach: all that are there, if they are no more; otherwise above some score, or the score itself.
  int32_t least = kAbsent + 1;
  uint32_t equal = 0xFFFFFFFFu;                                        // how many of those with the value itself are chosen
  if (present > a.most) {
    // count(low) > most; high + 1 is reached by the pages that are always chosen only, which are no more than `most`
    int32_t lo = low, hi = high + 1;
    bool exact = false;
    while (lo < hi) {
      const int32_t middle = lo + (hi - lo + 1) / 2;
      const uint32_t c = count(middle);
      if (c == a.most) {
        lo = middle;
        exact = true;
        break;
      }
      if (c > a.most) lo = middle;
      else hi = middle - 1;
    }
    least = lo;
    if (!exact) equal = a.most - count(least + 1);
  }
  // equal ones are taken from the front
  uint32_t taken = 0u;
  if (equal != 0xFFFFFFFFu && WAVES != 1u) {
    uint32_t mine = 0u;
    for (uint32_t i = from; i < upto; ++i) mine += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(read(i) == least));
    if (lane == 0u) shared[turn][wave] = (int32_t)mine;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) taken += (uint32_t)shared[turn][w];
  }
  const auto bits_of = [&](int32_t x) -> uint64_t {
    uint64_t over = __builtin_amdgcn_ballot_w64(equal == 0xFFFFFFFFu ? x >= least : x > least);
    if (equal != 0xFFFFFFFFu) {
      const uint64_t same = __builtin_amdgcn_ballot_w64(x == least);
      const uint32_t in_front = taken + (uint32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
      over |= __builtin_amdgcn_ballot_w64(x == least && in_front < equal);
      taken += (uint32_t)__builtin_popcountll(same);
    }
    return over;
  };
  const auto write = [&](uint32_t block, uint64_t bits) {
    const uint32_t word = 2u * block + lane;
    if (lane < 2u && word < a.words) choice[word] = (uint32_t)(bits >> (32u * lane));
  };
  if (kept) {
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i)
      if (from + i < upto) write(from + i, bits_of(keep[i]));
  } else {
    for (uint32_t i = from; i < upto; ++i) write(i, bits_of(read(i)));
  }
  for (uint32_t word = 2u * blocks + wave * kWaveSize + lane; word < a.words; word += WAVES * kWaveSize) choice[word] = 0u;
}

template <typename T, int D>
hipError_t launch_choose_of(const ChooseArgs& given, hipStream_t stream) {
  ChooseArgs a = given;
  const uint32_t all = a.starts ? places(a.tokens, a.p.rows, a.per) : a.p.rows, at_once = a.tiles;
  for (a.first_tile = 0u; a.first_tile < all; a.first_tile += at_once) {
    a.tiles = std::min(at_once, all - a.first_tile);
    // Few tiles: their pages in stretches, until there are two workgroups to a CU, of 64 pages at least.
    const uint32_t groups = a.tiles * a.p.kv_heads, pages = (a.p.row_pages + 63u) / 64u;
    const uint32_t cuts = std::min(pages, groups >= 512u ? 1u : (511u + groups) / groups), chunk = (pages + cuts - 1u) / cuts * 64u;
    const dim3 grid(groups, (a.p.row_pages + chunk - 1u) / chunk);
    if (!a.starts || a.per == 16u) score_kernel<T, D, 1u><<<grid, kScoreThreads, 0, stream>>>(a, chunk);
    else score_kernel<T, D, 4u><<<grid, kScoreThreads, 0, stream>>>(a, chunk);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t units = a.tiles * a.per * a.p.kv_heads;
    if (a.p.row_pages <= 1024u) choose_kernel<1u, 16u><<<(units + 3u) / 4u, 256, 0, stream>>>(a);
    else choose_kernel<16u, 16u><<<units, 1024, 0, stream>>>(a);
    e = hipGetLastError();
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
