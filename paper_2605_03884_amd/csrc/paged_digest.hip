// paged_digest.hip — bounds of the keys of a page in 8 bits, and the maps of a ragged batch.
#include "paged.h"
#include "paged_values.h"
#include "qkv_common.h"

namespace qkv {
namespace {

typedef short i16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- digests
//
//     hi = sat8(ceil(max_t K_t 2^-e)),   lo = sat8(floor(min_t K_t 2^-e))      per page, kv head and channel
//
// Rounding up and scaling by a power of two keep the order, so the extremes are found first, among the 16-bit patterns: with the lower bits of negative ones
// turned they are ordered as whole numbers (no number at either end, behind infinity), two to an instruction for both types.  The codes are worked out once a
// channel, in 64 bits, where every product with a power of two is exact.
//
// What bounds it: memory, and for a step the chain lengths - entry - keys - codes.  4100 tokens of 32 layers, 8 kv heads of 128 dimensions, pages of 32: 49.7 us for 277 MB (5.6 TB/s); with two
// loads at a time the same, with eight 55, through the caches 60, layers side by side 51.5.  64 sequences' new tokens, of which some fill a page of 16: 5.2 us a call, 4.6 here.
// Pages of more than 64 tokens are shared by the workgroup's waves: 8 layers of 4100 tokens in pages of 128 14.1 us, a wave each 16.2, a step's pages of 128 6.6 and 10.4; of 64 the same either way; of
// 32 21.3 if they were shared, 15.2 a wave each.
constexpr uint32_t kDigestThreads = 256;
constexpr uint32_t kDigestWaves = kDigestThreads / kWaveSize;
constexpr uint32_t kDigestSplit = 64;                    // tokens of a page from which on the waves of a workgroup share one

__device__ inline i16x8 ordered(i16x8 x) { return x ^ ((x >> 15) & (short)0x7FFF); }      // its own inverse

__device__ inline i16x8 from_lane(i16x8 x, uint32_t across) {
  u32x4 y = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (uint32_t)__shfl_xor((int)y[i], (int)across);
  return __builtin_bit_cast(i16x8, y);
}

// The rows' pages: which one `at` of a ragged batch's places names, if any.
struct FilledPage {
  uint32_t row, entry;
  bool there;
};
__device__ inline FilledPage filled_page(const DigestArgs& a, uint32_t at, uint32_t lane, bool tell) {
  FilledPage f{at, 0u, false};
  const uint32_t size = 1u << a.p.page_shift;
  if (!a.starts) {                                       // one token a row: the last page, if it has just been filled
    const uint32_t length = held(a.p.lens[at], a.p.row_pages, a.p.page_shift);
    f.entry = (length >> a.p.page_shift) - 1u;
    f.there = length != 0u && (length & (size - 1u)) == 0u;
    return f;
  }
  f.row = (uint32_t)__builtin_amdgcn_readfirstlane((int)find_row(a.p.rows, lane, [&](uint32_t b) { return first_place((uint32_t)a.starts[b], b, size) <= at; }));
  const int32_t start = a.starts[f.row], end = a.starts[f.row + 1u];
  const uint32_t length = held(a.p.lens[f.row], a.p.row_pages, a.p.page_shift);
  if (start < 0 || end < start || (uint32_t)end > a.tokens || (uint32_t)(end - start) > length) {
    if (tell) flag(a.status, QKV_STATUS_BAD_ROW);
    return f;
  }
  const uint32_t place = first_place((uint32_t)start, f.row, size);
  if (at < place) return f;
  f.entry = ((length - (uint32_t)(end - start)) >> a.p.page_shift) + (at - place);
  f.there = f.entry < length >> a.p.page_shift;
  return f;
}

// A wave takes a (page, kv head), or all waves of a workgroup do: D / 8 lanes read a row, 64 / (D / 8) rows at once.
template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(kDigestThreads) void digest_kernel(DigestArgs a) {
  constexpr uint32_t kRowLanes = D / 8, kRowsAtOnce = kWaveSize / kRowLanes, kAtOnce = 4;
  constexpr short kInfinity = (short)T::kExponent;
  __shared__ i16x8 parts[SPLIT ? kDigestWaves : 1u][2][kRowLanes];
  const uint32_t lane = threadIdx.x % kWaveSize, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWaveSize));
  const uint32_t unit = SPLIT ? blockIdx.x : blockIdx.x * kDigestWaves + wave, layer = blockIdx.y;
  const uint32_t at = unit / a.p.kv_heads, head = unit % a.p.kv_heads;
  if (at >= (a.starts ? places(a.tokens, a.p.rows, 1u << a.p.page_shift) : a.p.rows)) return;
  const bool first = head == 0u && layer == 0u && lane == 0u;
  const FilledPage f = filled_page(a, at, lane, first);
  if (!f.there) return;                                  // the same for the workgroup where its waves share a page
  const uint32_t page = (uint32_t)a.p.table[(uint64_t)f.row * a.p.row_pages + f.entry];
  if (page >= a.p.pages) {
    if (first) flag(a.status, QKV_STATUS_BAD_PAGE);
    return;
  }
  const uint32_t size = 1u << a.p.page_shift, chunk = lane % kRowLanes;
  const uint8_t* keys = a.k[layer] + (uint64_t)page * a.p.page_stride + (uint64_t)head * a.p.head_stride + chunk * 16u;
  i16x8 hi = (i16x8)((short)-32768), lo = (i16x8)((short)32767);
  constexpr uint32_t kStep = kRowsAtOnce * kAtOnce;
  for (uint32_t t = lane / kRowLanes + (SPLIT ? wave * kStep : 0u); t < size; t += kStep * (SPLIT ? kDigestWaves : 1u)) {
    i16x8 x[kAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j)               // behind the page's end its first row of the loop again
      x[j] = __builtin_bit_cast(i16x8, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(keys + (uint64_t)(t + j * kRowsAtOnce < size ? t + j * kRowsAtOnce : t) * a.p.token_stride)));
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      const i16x8 y = ordered(x[j]);
      hi = __builtin_elementwise_max(hi, y);
      lo = __builtin_elementwise_min(lo, y);
    }
  }
#pragma unroll
  for (uint32_t across = kRowLanes; across < kWaveSize; across *= 2u) {
    hi = __builtin_elementwise_max(hi, from_lane(hi, across));
    lo = __builtin_elementwise_min(lo, from_lane(lo, across));
  }
  if constexpr (SPLIT) {
    if (lane < kRowLanes) {
      parts[wave][0][lane] = hi;
      parts[wave][1][lane] = lo;
    }
    __syncthreads();
    if (wave != 0u) return;
#pragma unroll
    for (uint32_t w = 1; w < kDigestWaves; ++w) {
      hi = __builtin_elementwise_max(hi, parts[w][0][chunk]);
      lo = __builtin_elementwise_min(lo, parts[w][1][chunk]);
    }
  }
  if (lane >= kRowLanes) return;
  const u32x2 e = *reinterpret_cast<const u32x2*>(a.exponents + ((uint64_t)layer * a.p.kv_heads + head) * D + chunk * 8u);
  u32x2 top = (u32x2)(0u), low = (u32x2)(0u);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int down = -(int)(int8_t)(e[i / 4] >> (8 * (i % 4)));
    const bool numbers = hi[i] <= kInfinity && lo[i] >= (short)~kInfinity;      // ~: the order's place of minus infinity
    const double x = (double)(float)__builtin_bit_cast(typename T::x8, ordered(hi))[i], y = (double)(float)__builtin_bit_cast(typename T::x8, ordered(lo))[i];
    const double above = numbers ? fmin(fmax(__builtin_ceil(__builtin_ldexp(x, down)), -128.0), 127.0) : 127.0;
    const double below = numbers ? fmin(fmax(__builtin_floor(__builtin_ldexp(y, down)), -128.0), 127.0) : -128.0;
    top[i / 4] |= ((uint32_t)(int)above & 0xFFu) << (8 * (i % 4));
    low[i / 4] |= ((uint32_t)(int)below & 0xFFu) << (8 * (i % 4));
  }
  int8_t* to = a.digest[layer] + ((uint64_t)page * a.p.kv_heads + head) * (2u * D) + chunk * 8u;
  *reinterpret_cast<u32x2*>(to) = top;
  *reinterpret_cast<u32x2*>(to + D) = low;
}

template <typename T, int D>
hipError_t launch_digest_of(const DigestArgs& a, hipStream_t stream) {
  const uint64_t units = (uint64_t)(a.starts ? places(a.tokens, a.p.rows, 1u << a.p.page_shift) : a.p.rows) * a.p.kv_heads;
  if (1u << a.p.page_shift > kDigestSplit) digest_kernel<T, D, true><<<dim3((uint32_t)units, a.layers), kDigestThreads, 0, stream>>>(a);
  else digest_kernel<T, D, false><<<dim3((uint32_t)((units + kDigestWaves - 1u) / kDigestWaves), a.layers), kDigestThreads, 0, stream>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------- maps of a ragged batch
//
// Starts are prefix sums of the rows' numbers; a token finds its row by bisection.  Up to kSlotRows rows (what LDS is set aside for) every workgroup works out all starts by itself, in LDS, and
// one launch does; otherwise one workgroup writes them first.  Launches are what it costs: 64 tokens of as many rows 2.2 us here, 34993 places of 300 rows (572 KB) 4.1, of
// which reading lengths and numbers, summing and looking up are one chain.  In a graph 64 rows 3.1 us, two kernels 5.1; 2000 rows 6.6 and 8.3; 4096 rows of a token 10.2 and 10.6, of 20 11.7 and 11.0.
// The border is by rows alone, though every workgroup of 256 tokens sums all rows again: 1000 rows of up to 1000 tokens 8.4 and 8.4, but 4000 of up to 40 11.5 and 10.8, and of up to 1000 (2 million tokens) 55 and 25.
constexpr uint32_t kSlotThreads = 256;
constexpr uint32_t kSlotRows = 4096;

// New tokens of a row as they count; `bad`: what was given is not what may be.
__device__ inline uint32_t counted(const SlotsArgs& a, uint32_t row, bool& bad) {
  const uint32_t length = held(a.p.lens[row], a.p.row_pages, a.p.page_shift);
  if (!a.more) return length != 0u ? 1u : 0u;
  const int32_t n = a.more[row];
  if (n >= 0 && (uint32_t)n <= length) return (uint32_t)n;
  bad = true;
  return 0u;
}

// Prefix sums of numbers below 2^31 over a wave, in 64 bits, as two scans of 16 and 15 bits that cannot overflow.
__device__ inline uint64_t scan64(uint32_t x) { return (uint64_t)wave_inclusive_scan(x & 0xFFFFu) + ((uint64_t)wave_inclusive_scan(x >> 16) << 16); }

// Starts of all rows to `to` [rows + 1] (all threads of the workgroup).  Whether something was not what it may be, in this thread's rows.
struct StartSums {
  uint64_t wave[16];
  uint32_t fit;                                          // the largest sum that is not more than there is room for
};
template <uint32_t THREADS>
__device__ inline bool work_out_starts(const SlotsArgs& a, int32_t* to, StartSums& sums) {
  const uint32_t lane = threadIdx.x % kWaveSize, wave = threadIdx.x / kWaveSize;
  bool bad = false;
  uint64_t before = 0u;                                  // tokens of the rows before this round's, whether they fit or not
  if (threadIdx.x == 0u) {
    to[0] = 0;
    sums.fit = 0u;
  }
  for (uint32_t base = 0; base < a.p.rows; base += THREADS) {
    const uint32_t row = base + threadIdx.x;
    const uint64_t upto = scan64(row < a.p.rows ? counted(a, row, bad) : 0u);
    __syncthreads();
    if (lane == kWaveSize - 1u) sums.wave[wave] = upto;
    __syncthreads();
    uint64_t mine = before + upto;
    const uint64_t front = before;
#pragma unroll
    for (uint32_t w = 0; w < THREADS / kWaveSize; ++w) {
      mine += w < wave ? sums.wave[w] : 0u;
      before += sums.wave[w];
    }
    if (before <= a.tokens) {                            // the usual round: all of them fit
      if (row < a.p.rows) to[row + 1u] = (int32_t)mine;
      continue;
    }
    if (mine <= a.tokens) atomicMax(&sums.fit, (uint32_t)mine);
    if (threadIdx.x == 0u && front <= a.tokens) atomicMax(&sums.fit, (uint32_t)front);
    __syncthreads();
    if (row < a.p.rows) to[row + 1u] = (int32_t)(mine <= a.tokens ? (uint32_t)mine : sums.fit);
    bad = bad || mine > a.tokens;
  }
  __syncthreads();
  return bad;
}

// One token: its row is the last one that starts at or before it.  Rows without tokens start where the next one does, so that one has it.
__device__ inline void map_token(const SlotsArgs& a, const int32_t* starts, uint32_t token) {
  int32_t row = -1, place = -1;
  int64_t slot = -1;
  if ((int32_t)token < starts[a.p.rows]) {
    uint32_t lo = 0u, hi = a.p.rows;                     // starts[lo] <= token < starts[hi]
    while (hi - lo > 1u) {
      const uint32_t middle = (lo + hi) / 2u;
      if ((uint32_t)starts[middle] <= token) lo = middle;
      else hi = middle;
    }
    row = (int32_t)lo;
    place = (int32_t)held(a.p.lens[lo], a.p.row_pages, a.p.page_shift) - starts[lo + 1u] + (int32_t)token;
    if (a.slot) {
      const uint32_t page = (uint32_t)a.p.table[(uint64_t)lo * a.p.row_pages + ((uint32_t)place >> a.p.page_shift)];
      if (page < a.p.pages) slot = ((int64_t)page << a.p.page_shift) + (place & ((1 << a.p.page_shift) - 1));
      else flag(a.status, QKV_STATUS_BAD_PAGE);
    }
  }
  if (a.row) a.row[token] = row;
  if (a.place) a.place[token] = place;
  if (a.slot) a.slot[token] = slot;
}

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(SlotsArgs a) {
  __shared__ int32_t starts[kSlotRows + 1u];
  __shared__ StartSums sums;
  const bool bad = work_out_starts<kSlotThreads>(a, starts, sums);
  if (blockIdx.x == 0u) {
    if (bad) flag(a.status, QKV_STATUS_BAD_ROW);
    for (uint32_t i = threadIdx.x; i <= a.p.rows; i += kSlotThreads) a.starts[i] = starts[i];
  }
  const uint32_t token = blockIdx.x * kSlotThreads + threadIdx.x;
  if (token < a.tokens) map_token(a, starts, token);
}

__global__ __launch_bounds__(1024) void starts_kernel(SlotsArgs a) {
  __shared__ StartSums sums;
  if (work_out_starts<1024u>(a, a.starts, sums)) flag(a.status, QKV_STATUS_BAD_ROW);
}

__global__ __launch_bounds__(kSlotThreads) void map_kernel(SlotsArgs a) {
  const uint32_t token = blockIdx.x * kSlotThreads + threadIdx.x;
  if (token < a.tokens) map_token(a, a.starts, token);
}

}  // namespace

hipError_t launch_pages_digest(const DigestArgs& a, uint32_t head_dim, bool bf16, hipStream_t stream) {
  if (head_dim == 64u) return bf16 ? launch_digest_of<BFloat, 64>(a, stream) : launch_digest_of<Half, 64>(a, stream);
  if (head_dim == 128u) return bf16 ? launch_digest_of<BFloat, 128>(a, stream) : launch_digest_of<Half, 128>(a, stream);
  return bf16 ? launch_digest_of<BFloat, 256>(a, stream) : launch_digest_of<Half, 256>(a, stream);
}

hipError_t launch_pages_slots(const SlotsArgs& a, hipStream_t stream) {
  const uint32_t grid = (a.tokens + kSlotThreads - 1u) / kSlotThreads;
  if (a.p.rows <= kSlotRows) {
    slots_kernel<<<grid, kSlotThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  starts_kernel<<<1, 1024, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  map_kernel<<<grid, kSlotThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace qkv
