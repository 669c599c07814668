// paged_api.hip — the C ABI of the cache in pages: argument checks and launch planning.
#include <algorithm>
#include <cmath>
#include <limits>

#include "paged.h"

using namespace qkv;

namespace {

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

int check_pages(const qkv_pages_t* p, bool counted) {
  if (!p || !p->k_layers || !p->v_layers || !p->table_dev || !p->lens_dev || (counted && !p->refs_dev)) return QKV_ERR_NULL;
  if (p->layers < 1 || p->layers > QKV_INJECT_MAX_LAYERS || p->kv_heads < 1 || p->kv_heads > (1 << 16)) return QKV_ERR_SHAPE;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return QKV_ERR_SHAPE;
  if (p->page_tokens < 1 || p->page_tokens > (1 << 20) || (p->page_tokens & (p->page_tokens - 1)) != 0) return QKV_ERR_SHAPE;
  if (p->value_type != QKV_VALUE_FP16 && p->value_type != QKV_VALUE_BF16) return QKV_ERR_SHAPE;
  if (p->pages < 1 || p->rows < 1 || p->rows > (int32_t)kMaxRows || p->row_pages < 1) return QKV_ERR_SHAPE;
  if ((int64_t)p->row_pages * p->page_tokens >= (1ll << 31) - p->page_tokens || (int64_t)p->rows * p->row_pages >= (1ll << 31)) return QKV_ERR_SHAPE;
  const int64_t strides[3] = {p->page_stride, p->head_stride, p->token_stride};
  for (int i = 0; i < 3; ++i)
    if (strides[i] < 0 || strides[i] % 8 != 0 || strides[i] >= (1ll << 31)) return QKV_ERR_SHAPE;
  if (p->token_stride < p->head_dim || (int64_t)p->page_tokens * p->token_stride > (1ll << 30)) return QKV_ERR_SHAPE;
  if ((int64_t)p->page_tokens * p->kv_heads * p->head_dim >= (1ll << 31)) return QKV_ERR_SHAPE;     // a page's own size counts in 32 bits
  if (misaligned(p->table_dev, 4) || misaligned(p->lens_dev, 4) || misaligned(p->refs_dev, 4)) return QKV_ERR_ALIGN;
  for (int i = 0; i < p->layers; ++i) {
    if (!p->k_layers[i] || !p->v_layers[i]) return QKV_ERR_NULL;
    if (misaligned(p->k_layers[i], 16) || misaligned(p->v_layers[i], 16)) return QKV_ERR_ALIGN;
  }
  return QKV_OK;
}

uint32_t log2_of(int32_t power) { return (uint32_t)__builtin_ctz((unsigned)power); }

PageCache cache_of(const qkv_pages_t* p) {
  PageCache c = {};
  for (int i = 0; i < p->layers; ++i) {
    c.k[i] = static_cast<uint8_t*>(p->k_layers[i]);
    c.v[i] = static_cast<uint8_t*>(p->v_layers[i]);
  }
  c.page_stride = (uint64_t)p->page_stride * 2u;
  c.head_stride = (uint64_t)p->head_stride * 2u;
  c.token_stride = (uint64_t)p->token_stride * 2u;
  c.table = p->table_dev;
  c.lens = p->lens_dev;
  c.refs = p->refs_dev;
  c.layers = (uint32_t)p->layers;
  c.kv_heads = (uint32_t)p->kv_heads;
  c.head_dim = (uint32_t)p->head_dim;
  c.page_shift = log2_of(p->page_tokens);
  c.pages = (uint32_t)p->pages;
  c.rows = (uint32_t)p->rows;
  c.row_pages = (uint32_t)p->row_pages;
  return c;
}

PageLayer layer_of(const qkv_pages_t* p, int32_t layer) {
  PageLayer l;
  l.k = static_cast<const uint8_t*>(p->k_layers[layer]);
  l.v = static_cast<const uint8_t*>(p->v_layers[layer]);
  l.page_stride = (uint64_t)p->page_stride * 2u;
  l.head_stride = (uint64_t)p->head_stride * 2u;
  l.token_stride = (uint64_t)p->token_stride * 2u;
  l.table = p->table_dev;
  l.lens = p->lens_dev;
  l.rows = (uint32_t)p->rows;
  l.row_pages = (uint32_t)p->row_pages;
  l.pages = (uint32_t)p->pages;
  l.page_shift = log2_of(p->page_tokens);
  l.kv_heads = (uint32_t)p->kv_heads;
  return l;
}

int check_heads(const qkv_pages_t* p, int32_t q_heads) {
  if (q_heads < p->kv_heads || q_heads % p->kv_heads != 0 || q_heads / p->kv_heads > QKV_PAGED_MAX_REP) return QKV_ERR_SHAPE;
  return QKV_OK;
}

int check_where(const qkv_pages_t* p, const qkv_paged_query_t* a) {
  if (!a->q_dev || !a->out_dev) return QKV_ERR_NULL;
  if (a->layer < 0 || a->layer >= p->layers) return QKV_ERR_SHAPE;
  const int rc = check_heads(p, a->q_heads);
  if (rc) return rc;
  if (a->q_token_stride < 0 || a->q_token_stride % 8 != 0 || a->q_token_stride >= (1ll << 40) || a->q_head_stride < 0 || a->q_head_stride % 8 != 0 ||
      a->q_head_stride >= (1ll << 31))
    return QKV_ERR_SHAPE;
  if (a->window < 0 || a->sinks < 0 || (a->window == 0 && a->sinks != 0) || !std::isfinite(a->softmax_scale)) return QKV_ERR_SHAPE;
  if (misaligned(a->q_dev, 16) || misaligned(a->out_dev, 16) || misaligned(a->lse_dev, 4) || misaligned(a->status_dev, 4)) return QKV_ERR_ALIGN;
  return QKV_OK;
}

// Tiles of 32 tokens that the longest sequence the table has room for can have, sinks and the window's edge included.
uint64_t most_tiles(const qkv_pages_t* p) { return ((uint64_t)p->row_pages * (uint64_t)p->page_tokens + 31u) / 32u + 2u; }

// A window that holds any sequence the table has room for is none.
uint32_t window_of(const qkv_pages_t* p, int32_t window) { return (int64_t)window >= (int64_t)p->row_pages * p->page_tokens ? 0u : (uint32_t)window; }

// The scale for powers of two.  One of 0 is as good as none, but infinity times it has to stay infinite, as 0 times the largest has to stay 0.
float scale_of(float scale) {
  const double most = std::numeric_limits<float>::max();
  const float x = (float)std::min(std::max((double)scale * 1.4426950408889634, -most), most);
  return std::fabs(x) >= 1e-37f ? x : x < 0.0f ? -1e-37f : 1e-37f;
}

struct AttendPlan {
  uint32_t rep, blocks, heads;      // query heads per kv head, groups of 16, heads of a group
  uint64_t items;
  uint32_t most;                    // shares
  bool split;
  uint64_t floats;
};
int plan_attend(const qkv_pages_t* p, int32_t q_heads, AttendPlan& a) {
  a.rep = (uint32_t)(q_heads / p->kv_heads);
  a.blocks = (a.rep + 15u) / 16u;
  a.heads = a.rep < 16u ? a.rep : 16u;
  a.items = (uint64_t)p->rows * (uint64_t)p->kv_heads * a.blocks;
  if (a.items * most_tiles(p) >= (1ull << 31) || a.items >= (1ull << 22)) return QKV_ERR_SHAPE;
  a.split = most_tiles(p) - 2u > kAttendWhole;
  // Waves: as many as the chip holds at once at 128 dimensions' registers, two a SIMD, or at 256 one, or as many as there may be tiles.  128 dimensions with one a
  // SIMD: 48 rows of up to 8K tokens 150.5 us (with two 152), 200 of them 550 (545), 131071 tokens of one row 93 (96); 64 dimensions, 48 rows 97.5 (80.4); with
  // three a SIMD 64 rows of 1004 seen tokens 32.8 (31.8).
  const uint64_t shares = a.items * most_tiles(p), fit = p->head_dim == 256 ? 1024u : 2048u;
  a.most = (uint32_t)(shares < fit ? shares : fit);
  a.floats = a.split ? (a.items + a.most) * a.heads * ((uint64_t)p->head_dim + 2u) : 0u;
  return QKV_OK;
}

constexpr int64_t kLargePrompt = 256 * 256;      // (token, query head) pairs
constexpr uint64_t kMostCut = 4u * 768u;         // query tiles from which on keys are never cut

struct PromptPlan {
  uint32_t rep, per, waves, splits, least;
  uint64_t floats;
};
int plan_prompt(const qkv_pages_t* p, int32_t q_heads, int64_t tokens, PromptPlan& a) {
  if (tokens < 1 || tokens >= (1ll << 31) / q_heads) return QKV_ERR_SHAPE;
  a.rep = (uint32_t)(q_heads / p->kv_heads);
  // 128 dimensions: tiles of 256 pairs (8 waves) where there is one for every CU (an 8K prompt 571 us, with tiles of 128 619; six short prompts 21.4, 17.4).
  // 64 dimensions do better with three workgroups of 4 waves a CU (170 us, 198), 256 have no registers for two waves a SIMD.
  a.waves = p->head_dim == 128 && tokens * q_heads >= kLargePrompt ? 8u : 4u;
  a.per = 32u * a.waves / a.rep;
  const uint64_t tiles = (uint64_t)(tokens / a.per + p->rows) * (uint64_t)p->kv_heads;
  if (tiles * a.waves * 64u >= (1ull << 32)) return QKV_ERR_SHAPE;       // threads of a grid's dimension
  // Few query tiles: the keys are split until there are two workgroups to a CU, where sequences turn out to have that many (61 tokens of 32 heads behind
  // 32768: 16 parts 75 us, 32 65, 64 87 while their join still took a fifth longer).  Tiles of 256 pairs are never so few.
  const uint64_t room = (uint64_t)p->row_pages * (uint64_t)p->page_tokens + 128u, groups = (uint64_t)((tokens + a.per - 1) / a.per) * (uint64_t)p->kv_heads;
  a.least = 512u;
  a.splits = a.waves == 8u || groups > 256u ? 1u : prompt_splits((uint32_t)room, groups > 8u ? (uint32_t)(512u / groups) : 64u);
  // Workgroups that leave much of the chip idle at the end (264 where 256 run at once): up to four long parts, until they fill 82 % of its turns, from where on the
  // power is what counts; each part costs a few percent to write and to join.  32 heads of 128 dimensions behind 32768 tokens: 1100 tokens 1004 us -> 787, 2100
  // 1900 -> 1370, 4500 3280 -> 2845; behind 16000 503 -> 404, 934 -> 690, 1625 -> 1493, with parts of at least 8192 keys 504, 773, 1499; with parts of
  // 2048, 4500 tokens with nothing in front 201 -> 242.  Where sequences turn out to be short, the join's look at them is 1 - 2 us.
  const uint64_t at_once = p->head_dim == 64 ? 768u : p->head_dim == 128 && a.waves == 4u ? 512u : 256u;      // kMostCut / 4 at most
  if (a.splits == 1u && groups > 256u && groups < 4u * at_once) {
    a.least = 4096u;
    double best = 0.0;
    for (uint64_t n = 1; n <= 4u && (n == 1u || n * a.least <= room); ++n) {
      const double turns = (double)(groups * n) / (double)at_once, worth = std::fmin(turns / std::ceil(turns), 0.82) - 0.025 * (double)(n - 1u);
      if (worth > best) {
        best = worth;
        a.splits = (uint32_t)n;
      }
    }
  }
  a.floats = a.splits == 1u ? 0u : a.splits * (uint64_t)tokens * (uint64_t)q_heads * ((uint64_t)p->head_dim + 2u);
  return QKV_OK;
}

// The most that any batch of up to `tokens` tokens needs.  It is not the largest one that needs it: parts get fewer as query tiles get more.  With a number of
// query tiles given the batch that fills them needs most; behind kMostCut of them none has parts.
int most_prompt_floats(const qkv_pages_t* p, int32_t q_heads, int64_t tokens, uint64_t& floats) {
  PromptPlan plan;
  const int rc = plan_prompt(p, q_heads, tokens, plan);
  if (rc) return rc;
  floats = plan.floats;
  const int64_t large = p->head_dim == 128 ? (kLargePrompt + q_heads - 1) / q_heads : INT64_MAX;      // batches from here on have tiles of 8 waves
  for (uint32_t waves = 4u; waves <= plan.waves; waves += 4u) {
    const int64_t last = waves == 4u ? std::min(tokens, large - 1) : tokens, per = 32u * waves / plan.rep;
    for (int64_t n = per; n - per < last && (uint64_t)(n / per) * (uint64_t)p->kv_heads < kMostCut; n += per) {
      PromptPlan smaller;
      if (plan_prompt(p, q_heads, std::min(n, last), smaller) == QKV_OK) floats = std::max(floats, smaller.floats);
    }
  }
  return QKV_OK;
}

int check_digests(const qkv_pages_t* p, const qkv_digests_t* d) {
  if (!d || !d->layers || !d->exponents_dev) return QKV_ERR_NULL;
  if (misaligned(d->exponents_dev, 16)) return QKV_ERR_ALIGN;
  for (int i = 0; i < p->layers; ++i) {
    if (!d->layers[i]) return QKV_ERR_NULL;
    if (misaligned(d->layers[i], 16)) return QKV_ERR_ALIGN;
  }
  return QKV_OK;
}

uint32_t words_of(const qkv_pages_t* p) { return ((uint32_t)p->row_pages + 31u) / 32u; }

// Scores stay in LDS where they fit and there are enough tiles or few pages to each; otherwise they go through the workspace, those of as many tiles of query tokens at a
// time as fit in kScoreBytes, or of one.  In us, 8 kv heads of 128 dimensions:
//   one token of a row       1 row of 300 pages 7.4 in LDS, 8.2 through the workspace; of 1000 pages 12.3, 8.6; 16 rows of 1000 pages 12.3, 12.0; 32 rows 13.9, 16.4; 64 rows of 2040 pages 33, 37
//   16 tokens a tile in LDS  with more than 768 pages a workgroup fills a CU: 600 tokens of 1000 pages 17.2, 28.2; of 1500 22.9, 33.8; 3000 tokens of 1000 pages 80, 63
//   32 tokens a tile in LDS  3000 tokens of 180 pages 25, in tiles of 16 34; 1200 tokens 12.9, 12.9; 600 tokens 13.1, 11.3
//   64 through the workspace 512 tokens of 2 heads and 12000 pages 53.7, in tiles of 16 59.7; of 20000 pages 119, 129
constexpr uint64_t kScoreBytes = 128ull << 20;
struct ChoosePlan {
  uint32_t per, stride, all, tiles;         // query tokens of a tile; scores of a (token, kv head); tiles in all and at a time
  uint64_t bytes;
};
int plan_choose(const qkv_pages_t* p, int64_t tokens, bool single, ChoosePlan& a) {
  a.stride = ((uint32_t)p->row_pages + 63u) / 64u * 64u;
  const uint64_t items = (uint64_t)p->rows * (uint64_t)p->kv_heads;
  const bool enough = tokens >= 32ll * p->rows;
  const uint64_t tiles_of_16 = ((uint64_t)tokens / 16u + (uint64_t)p->rows) * (uint64_t)p->kv_heads;
  const bool within = single ? a.stride <= 512u || (a.stride <= 2048u && items >= 256u) : a.stride <= 768u || (a.stride <= 1536u && tiles_of_16 <= 768u);
  a.per = single ? 1u : !within ? (enough && 64u * (uint64_t)p->kv_heads * a.stride * 4u <= kScoreBytes ? 64u : 16u) : enough && a.stride <= 384u && (uint64_t)tokens * (uint64_t)p->kv_heads >= 8192u ? 32u : 16u;
  a.all = single ? (uint32_t)p->rows : (uint32_t)(tokens / a.per) + (uint32_t)p->rows;
  if ((uint64_t)a.all * (uint64_t)p->kv_heads >= (1ull << 23)) return QKV_ERR_SHAPE;     // 512 threads each, of a grid's 2^32
  a.tiles = a.all;
  a.bytes = 0u;
  if (within) return QKV_OK;
  const uint64_t tile = (uint64_t)a.per * (uint64_t)p->kv_heads * a.stride * 4u;
  // also few enough for a workgroup to each (token, kv head), of 1024 threads
  const uint64_t fit = std::max<uint64_t>(1u, std::min<uint64_t>(kScoreBytes / tile, (1ull << 21) / ((uint64_t)a.per * (uint64_t)p->kv_heads)));
  a.tiles = (uint32_t)std::min<uint64_t>(a.all, fit);
  a.bytes = a.tiles * tile;
  return QKV_OK;
}
// What is enough for every batch of up to `tokens`: tiles get larger with their number, and the largest that are cut off at kScoreBytes need not be those of most tokens.
// As many tokens as there are rows may be one of each where prompts of as many have no room in a launch: then the most that prompts may have counts.
int most_choose_bytes(const qkv_pages_t* p, int64_t tokens, uint64_t& bytes) {
  bytes = 0u;
  const int64_t border = 32ll * p->rows - 1, most = 16ll * (((1ll << 23) - 1) / p->kv_heads - p->rows) + 15;
  for (int64_t n : {tokens, std::min(tokens, border)}) {
    ChoosePlan plan;
    int rc = plan_choose(p, n, false, plan);
    if (rc && tokens != p->rows) return rc;
    if (rc && most < 1) continue;
    if (rc) rc = plan_choose(p, std::min(n, most), false, plan);
    if (rc) return rc;
    bytes = std::max(bytes, plan.bytes);
  }
  if (tokens >= p->rows) {
    ChoosePlan plan;
    const int rc = plan_choose(p, p->rows, true, plan);
    if (rc) return rc;
    bytes = std::max(bytes, plan.bytes);
  }
  return QKV_OK;
}
int check_choose(const qkv_pages_t* p, int64_t tokens) {
  if (tokens < 1 || tokens >= (1ll << 31) / 64 / p->kv_heads || p->row_pages >= (1 << 20)) return QKV_ERR_SHAPE;
  return QKV_OK;
}

struct ChosenPlan {
  uint32_t rep, blocks, parts;
  uint64_t floats, rows;                    // rows: of dimensions in the workspace
};
int plan_chosen(const qkv_pages_t* p, int32_t q_heads, int32_t most, ChosenPlan& a) {
  if (most < 0) return QKV_ERR_SHAPE;
  a.rep = (uint32_t)(q_heads / p->kv_heads);
  a.blocks = (a.rep + 15u) / 16u;
  const uint64_t items = (uint64_t)p->rows * (uint64_t)p->kv_heads * a.blocks;
  if (items >= (1ull << 22)) return QKV_ERR_SHAPE;
  // Few items: parts, until there are two workgroups to a CU.  16 rows of 8 kv heads, 64 pages of 16: 19.9 us, with one to a CU 20.3, with four 23.7; 8 rows, 256 pages: 29.2, 30.6, 33.3.
  const uint64_t pages = most == 0 || most > p->row_pages ? (uint64_t)p->row_pages : (uint64_t)most;
  const uint64_t turns = (pages * (uint64_t)p->page_tokens + kAttendTile * 4u - 1u) / (kAttendTile * 4u);      // of a workgroup's four waves
  a.parts = (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>(items >= 512u ? 1u : 512u / items, turns));
  a.rows = a.parts == 1u ? 0u : items * a.parts * std::min(16u, a.rep);
  a.floats = a.rows * ((uint64_t)p->head_dim + 2u);
  return QKV_OK;
}

// As for all pages, but that a workgroup's pairs share a list, and no part's length is known beforehand: parts are cut by what there is room for.
int plan_prompt_chosen(const qkv_pages_t* p, int32_t q_heads, int64_t tokens, PromptPlan& a) {
  if (tokens < 1 || tokens >= (1ll << 31) / q_heads) return QKV_ERR_SHAPE;
  a.rep = (uint32_t)(q_heads / p->kv_heads);
  a.waves = 4u;
  a.per = 128u / a.rep;
  const uint64_t tiles = (uint64_t)(tokens / a.per + p->rows) * (uint64_t)p->kv_heads;
  if (tiles * 256u >= (1ull << 32)) return QKV_ERR_SHAPE;
  const uint64_t room = (uint64_t)p->row_pages * (uint64_t)p->page_tokens, groups = (uint64_t)((tokens + a.per - 1) / a.per) * (uint64_t)p->kv_heads;
  a.least = 0u;
  a.splits = groups > 256u ? 1u : prompt_splits((uint32_t)std::min<uint64_t>(room, 1u << 30), groups > 8u ? (uint32_t)(512u / groups) : 64u);
  // Workgroups that leave much of the chip idle at the end: up to four parts, until they fill 82 % of its turns; each part costs a few percent to write and to join.
  // 1000 tokens of 64 heads of 64 dimensions behind 32768, 504 workgroups where 768 run at once: 176 us, in 2 parts 168, in 3 152, in 4 162.
  const uint64_t at_once = p->head_dim == 64 ? 768u : p->head_dim == 128 ? 512u : 256u;
  if (groups > 256u && groups < 4u * at_once) {
    double best = 0.0;
    for (uint64_t n = 1; n <= 4u && (n == 1u || n * 4096u <= room); ++n) {
      const double turns = (double)(groups * n) / (double)at_once, worth = std::fmin(turns / std::ceil(turns), 0.82) - 0.025 * (double)(n - 1u);
      if (worth > best) {
        best = worth;
        a.splits = (uint32_t)n;
      }
    }
  }
  a.floats = a.splits == 1u ? 0u : a.splits * (uint64_t)tokens * (uint64_t)q_heads * ((uint64_t)p->head_dim + 2u);
  return QKV_OK;
}
int most_prompt_chosen_floats(const qkv_pages_t* p, int32_t q_heads, int64_t tokens, uint64_t& floats) {
  PromptPlan plan;
  const int rc = plan_prompt_chosen(p, q_heads, tokens, plan);
  if (rc) return rc;
  floats = plan.floats;
  // parts get fewer as query tiles get more: of the batches with as many tiles the one that fills them needs most, and behind kMostCut of them none has parts
  const int64_t per = 128 / (int64_t)plan.rep;
  for (int64_t n = per; n - per < tokens && (uint64_t)(n / per - 1) * (uint64_t)p->kv_heads < kMostCut; n += per) {
    PromptPlan smaller;
    if (plan_prompt_chosen(p, q_heads, std::min(n, tokens), smaller) == QKV_OK) floats = std::max(floats, smaller.floats);
  }
  return QKV_OK;
}

void set_prompt(const qkv_pages_t* pages, const qkv_paged_query_t* query, const PromptPlan& plan, PagedPromptArgs& a) {
  a.p = layer_of(pages, query->layer);
  a.q = static_cast<const uint8_t*>(query->q_dev);
  a.q_token_stride = (uint64_t)query->q_token_stride * 2u;
  a.q_head_stride = (uint64_t)query->q_head_stride * 2u;
  a.starts = query->starts_dev;
  a.tokens = (uint32_t)query->tokens;
  a.rep = plan.rep;
  a.per = plan.per;
  a.waves = plan.waves;
  a.window = window_of(pages, query->window);
  a.sinks = a.window ? (uint32_t)query->sinks : 0u;
  a.scale_log2 = std::fabs(scale_of(query->softmax_scale));
  a.flip = query->softmax_scale < 0.0f ? 1u : 0u;
  a.out = static_cast<uint8_t*>(query->out_dev);
  a.lse = query->lse_dev;
  a.part_o = static_cast<float*>(query->workspace_dev);
  a.part_ml = plan.floats ? a.part_o + plan.splits * (uint64_t)query->tokens * (uint64_t)query->q_heads * (uint64_t)pages->head_dim : nullptr;
  a.splits = plan.splits;
  a.least = plan.least;
  a.status = query->status_dev;
  a.choice = nullptr;
  a.words = 0u;
}

}  // namespace

extern "C" {

int qkv_pages_append(const qkv_pages_t* pages, const qkv_rows_t* rows, uint32_t* status_dev, void* stream) {
  const int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!rows || !rows->k_dev || !rows->v_dev) return QKV_ERR_NULL;
  if (rows->layer_begin < 0 || rows->layer_count < 1 || rows->layer_begin > pages->layers - rows->layer_count) return QKV_ERR_SHAPE;
  if (rows->tokens < 0 || rows->tokens >= (1ll << 27) || (!rows->starts_dev && rows->tokens != pages->rows)) return QKV_ERR_SHAPE;
  const int64_t strides[3] = {rows->layer_stride, rows->head_stride, rows->token_stride};
  for (int i = 0; i < 3; ++i)
    if (strides[i] < 0 || strides[i] % 8 != 0 || strides[i] >= (1ll << 40)) return QKV_ERR_SHAPE;
  if (misaligned(rows->k_dev, 16) || misaligned(rows->v_dev, 16) || misaligned(rows->starts_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  AppendArgs a;
  a.k = static_cast<const uint8_t*>(rows->k_dev);
  a.v = static_cast<const uint8_t*>(rows->v_dev);
  a.layer_stride = (uint64_t)rows->layer_stride * 2u;
  a.head_stride = (uint64_t)rows->head_stride * 2u;
  a.token_stride = (uint64_t)rows->token_stride * 2u;
  a.starts = rows->starts_dev;
  a.tokens = (uint32_t)rows->tokens;
  a.layer_begin = (uint32_t)rows->layer_begin;
  a.layer_count = (uint32_t)rows->layer_count;
  a.first = 0u;
  a.status = status_dev;
  return launch_pages_append(cache_of(pages), a, static_cast<hipStream_t>(stream)) == hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_reserve(const qkv_pages_t* pages, const int32_t* more_dev, uint32_t* status_dev, void* stream) {
  const int rc = check_pages(pages, true);
  if (rc) return rc;
  if (!status_dev) return QKV_ERR_NULL;
  if (misaligned(more_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  return launch_pages_reserve(cache_of(pages), more_dev, status_dev, static_cast<hipStream_t>(stream)) == hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_fork(const qkv_pages_t* pages, const int32_t* source_dev, const int32_t* target_dev, int32_t count, uint32_t* status_dev,
                   void* stream) {
  const int rc = check_pages(pages, true);
  if (rc) return rc;
  if (!source_dev || !target_dev || !status_dev) return QKV_ERR_NULL;
  if (count < 1 || count > pages->rows) return QKV_ERR_SHAPE;
  if (misaligned(source_dev, 4) || misaligned(target_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  return launch_pages_fork(cache_of(pages), source_dev, target_dev, (uint32_t)count, status_dev, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_free(const qkv_pages_t* pages, const int32_t* rows_dev, int32_t count, int32_t window, int32_t sinks, uint32_t* status_dev,
                   void* stream) {
  const int rc = check_pages(pages, true);
  if (rc) return rc;
  if (count < 1 || count > pages->rows || (!rows_dev && count != pages->rows)) return QKV_ERR_SHAPE;
  if (window < 0 || sinks < 0 || (window == 0 && sinks != 0)) return QKV_ERR_SHAPE;
  if (misaligned(rows_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  return launch_pages_free(cache_of(pages), rows_dev, (uint32_t)count, (uint32_t)window, (uint32_t)sinks, status_dev,
                           static_cast<hipStream_t>(stream)) == hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_compact_workspace(const qkv_pages_t* pages, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  const int rc = check_pages(pages, false);
  if (rc) return rc;
  *bytes_out = 16u + 12u * (uint64_t)pages->pages;
  return QKV_OK;
}

int qkv_pages_compact(const qkv_pages_t* pages, int32_t* live_dev, void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev,
                      void* stream) {
  const int rc = check_pages(pages, true);
  if (rc) return rc;
  if (!workspace_dev || !status_dev) return QKV_ERR_NULL;
  uint64_t bytes = 0;
  qkv_pages_compact_workspace(pages, &bytes);
  if (workspace_bytes < bytes) return QKV_ERR_CAPACITY;
  if (misaligned(workspace_dev, 16) || misaligned(live_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  return launch_pages_compact(cache_of(pages), live_dev, static_cast<int32_t*>(workspace_dev), status_dev, static_cast<hipStream_t>(stream)) ==
                 hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

int qkv_paged_attend_workspace(const qkv_pages_t* pages, int32_t q_heads, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_heads(pages, q_heads);
  if (rc) return rc;
  AttendPlan plan;
  rc = plan_attend(pages, q_heads, plan);
  if (rc) return rc;
  *bytes_out = plan.floats * sizeof(float);
  return QKV_OK;
}

int qkv_paged_attend(const qkv_pages_t* pages, const qkv_paged_query_t* query, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!query) return QKV_ERR_NULL;
  rc = check_where(pages, query);
  if (rc) return rc;
  if (query->tokens != pages->rows || query->starts_dev) return QKV_ERR_SHAPE;
  if ((query->prior_out_dev == nullptr) != (query->prior_lse_dev == nullptr)) return QKV_ERR_NULL;
  AttendPlan plan;
  rc = plan_attend(pages, query->q_heads, plan);
  if (rc) return rc;
  if (plan.floats != 0u && !query->workspace_dev) return QKV_ERR_NULL;
  if (query->workspace_bytes < plan.floats * sizeof(float)) return QKV_ERR_CAPACITY;
  if (misaligned(query->workspace_dev, 16) || misaligned(query->prior_out_dev, 16) || misaligned(query->prior_lse_dev, 4)) return QKV_ERR_ALIGN;
  PagedAttendArgs a;
  a.p = layer_of(pages, query->layer);
  a.q = static_cast<const uint8_t*>(query->q_dev);
  a.q_token_stride = (uint64_t)query->q_token_stride * 2u;
  a.q_head_stride = (uint64_t)query->q_head_stride * 2u;
  a.rep = plan.rep;
  a.blocks = plan.blocks;
  a.window = window_of(pages, query->window);
  a.sinks = a.window ? (uint32_t)query->sinks : 0u;
  a.scale_log2 = scale_of(query->softmax_scale);
  a.nothing = a.scale_log2 < 0.0f ? INFINITY : -INFINITY;
  a.prior_out = query->prior_out_dev;
  a.prior_lse = query->prior_lse_dev;
  a.out = static_cast<float*>(query->out_dev);
  a.lse = query->lse_dev;
  a.part_o = static_cast<float*>(query->workspace_dev);
  a.part_ml = plan.floats ? a.part_o + (plan.items + plan.most) * plan.heads * (uint64_t)pages->head_dim : nullptr;
  a.most = plan.most;
  a.cut = plan.split ? 1u : 0u;
  a.status = query->status_dev;
  return launch_paged_attend(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, plan.split, static_cast<hipStream_t>(stream)) ==
                 hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

int qkv_paged_prompt_workspace(const qkv_pages_t* pages, int32_t q_heads, int64_t tokens, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_heads(pages, q_heads);
  if (rc) return rc;
  uint64_t floats = 0;
  rc = most_prompt_floats(pages, q_heads, tokens, floats);
  if (rc) return rc;
  *bytes_out = floats * sizeof(float);
  return QKV_OK;
}

int qkv_paged_prompt(const qkv_pages_t* pages, const qkv_paged_query_t* query, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!query || !query->starts_dev) return QKV_ERR_NULL;
  rc = check_where(pages, query);
  if (rc) return rc;
  if (query->prior_out_dev || query->prior_lse_dev) return QKV_ERR_SHAPE;
  PromptPlan plan;
  rc = plan_prompt(pages, query->q_heads, query->tokens, plan);
  if (rc) return rc;
  if (plan.floats != 0u && !query->workspace_dev) return QKV_ERR_NULL;
  if (query->workspace_bytes < plan.floats * sizeof(float)) return QKV_ERR_CAPACITY;
  if (misaligned(query->workspace_dev, 16) || misaligned(query->starts_dev, 4)) return QKV_ERR_ALIGN;
  PagedPromptArgs a;
  set_prompt(pages, query, plan, a);
  return launch_paged_prompt(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_digest(const qkv_pages_t* pages, const qkv_digests_t* digests, const int32_t* starts_dev, int64_t tokens, int32_t layer_begin,
                     int32_t layer_count, uint32_t* status_dev, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_digests(pages, digests);
  if (rc) return rc;
  if (layer_begin < 0 || layer_count < 1 || layer_begin > pages->layers - layer_count) return QKV_ERR_SHAPE;
  if (tokens < 0 || tokens >= (1ll << 27) || (!starts_dev && tokens != pages->rows)) return QKV_ERR_SHAPE;
  if ((uint64_t)(tokens / pages->page_tokens + pages->rows) * (uint64_t)pages->kv_heads >= (1ull << 24)) return QKV_ERR_SHAPE;      // 256 threads each, of a grid's 2^32
  if (misaligned(starts_dev, 4) || misaligned(status_dev, 4)) return QKV_ERR_ALIGN;
  DigestArgs a = {};
  for (int i = 0; i < layer_count; ++i) {
    a.k[i] = static_cast<const uint8_t*>(pages->k_layers[layer_begin + i]);
    a.digest[i] = static_cast<int8_t*>(digests->layers[layer_begin + i]);
  }
  a.p = layer_of(pages, layer_begin);
  a.exponents = digests->exponents_dev + (int64_t)layer_begin * pages->kv_heads * pages->head_dim;
  a.starts = starts_dev;
  a.tokens = (uint32_t)tokens;
  a.layers = (uint32_t)layer_count;
  a.status = status_dev;
  return launch_pages_digest(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_paged_choose_workspace(const qkv_pages_t* pages, int64_t tokens, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_choose(pages, tokens);
  if (rc) return rc;
  return most_choose_bytes(pages, tokens, *bytes_out);
}

int qkv_paged_choose(const qkv_pages_t* pages, const qkv_digests_t* digests, const qkv_choose_t* choose, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_digests(pages, digests);
  if (rc) return rc;
  if (!choose || !choose->q_dev || !choose->choice_dev) return QKV_ERR_NULL;
  if (choose->layer < 0 || choose->layer >= pages->layers) return QKV_ERR_SHAPE;
  rc = check_heads(pages, choose->q_heads);
  if (rc) return rc;
  if (choose->q_token_stride < 0 || choose->q_token_stride % 8 != 0 || choose->q_token_stride >= (1ll << 40) || choose->q_head_stride < 0 ||
      choose->q_head_stride % 8 != 0 || choose->q_head_stride >= (1ll << 31))
    return QKV_ERR_SHAPE;
  if (choose->first < 0 || choose->last < 1 || (int64_t)choose->most < (int64_t)choose->first + choose->last) return QKV_ERR_SHAPE;
  rc = check_choose(pages, choose->tokens);
  if (rc) return rc;
  if (!choose->starts_dev && choose->tokens != pages->rows) return QKV_ERR_SHAPE;
  ChoosePlan plan;
  rc = plan_choose(pages, choose->tokens, !choose->starts_dev, plan);
  if (rc) return rc;
  if (misaligned(choose->q_dev, 16) || misaligned(choose->choice_dev, 4) || misaligned(choose->starts_dev, 4) || misaligned(choose->status_dev, 4) ||
      misaligned(choose->workspace_dev, 16))
    return QKV_ERR_ALIGN;
  if (plan.bytes != 0u && !choose->workspace_dev) return QKV_ERR_NULL;
  if (choose->workspace_bytes < plan.bytes) return QKV_ERR_CAPACITY;
  ChooseArgs a;
  a.p = layer_of(pages, choose->layer);
  a.q = static_cast<const uint8_t*>(choose->q_dev);
  a.q_token_stride = (uint64_t)choose->q_token_stride * 2u;
  a.q_head_stride = (uint64_t)choose->q_head_stride * 2u;
  a.digest = static_cast<const int8_t*>(digests->layers[choose->layer]);
  a.exponents = digests->exponents_dev + (int64_t)choose->layer * pages->kv_heads * pages->head_dim;
  a.starts = choose->starts_dev;
  a.tokens = (uint32_t)choose->tokens;
  a.rep = (uint32_t)(choose->q_heads / pages->kv_heads);
  a.per = plan.per;
  a.first_tile = 0u;
  a.tiles = plan.tiles;
  a.most = (uint32_t)choose->most;
  a.first = (uint32_t)choose->first;
  a.last = (uint32_t)choose->last;
  a.words = words_of(pages);
  a.stride = plan.stride;
  a.choice = choose->choice_dev;
  a.status = choose->status_dev;
  a.scores = plan.bytes ? static_cast<int32_t*>(choose->workspace_dev) : nullptr;
  return launch_paged_choose(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_paged_attend_chosen_workspace(const qkv_pages_t* pages, int32_t q_heads, int32_t most, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_heads(pages, q_heads);
  if (rc) return rc;
  ChosenPlan plan;
  rc = plan_chosen(pages, q_heads, most, plan);
  if (rc) return rc;
  *bytes_out = plan.floats * sizeof(float);
  return QKV_OK;
}

int qkv_paged_attend_chosen(const qkv_pages_t* pages, const qkv_paged_query_t* query, const uint32_t* choice_dev, int32_t most, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!query || !choice_dev) return QKV_ERR_NULL;
  rc = check_where(pages, query);
  if (rc) return rc;
  if (query->tokens != pages->rows || query->starts_dev || query->window != 0) return QKV_ERR_SHAPE;
  if ((query->prior_out_dev == nullptr) != (query->prior_lse_dev == nullptr)) return QKV_ERR_NULL;
  ChosenPlan plan;
  rc = plan_chosen(pages, query->q_heads, most, plan);
  if (rc) return rc;
  if (plan.floats != 0u && !query->workspace_dev) return QKV_ERR_NULL;
  if (query->workspace_bytes < plan.floats * sizeof(float)) return QKV_ERR_CAPACITY;
  if (misaligned(query->workspace_dev, 16) || misaligned(query->prior_out_dev, 16) || misaligned(query->prior_lse_dev, 4) || misaligned(choice_dev, 4))
    return QKV_ERR_ALIGN;
  ChosenAttendArgs a;
  a.p = layer_of(pages, query->layer);
  a.q = static_cast<const uint8_t*>(query->q_dev);
  a.q_token_stride = (uint64_t)query->q_token_stride * 2u;
  a.q_head_stride = (uint64_t)query->q_head_stride * 2u;
  a.choice = choice_dev;
  a.words = words_of(pages);
  a.rep = plan.rep;
  a.blocks = plan.blocks;
  a.parts = plan.parts;
  a.scale_log2 = scale_of(query->softmax_scale);
  a.nothing = a.scale_log2 < 0.0f ? INFINITY : -INFINITY;
  a.prior_out = query->prior_out_dev;
  a.prior_lse = query->prior_lse_dev;
  a.out = static_cast<float*>(query->out_dev);
  a.lse = query->lse_dev;
  a.part_o = static_cast<float*>(query->workspace_dev);
  a.part_ml = plan.floats ? a.part_o + plan.rows * (uint64_t)pages->head_dim : nullptr;
  a.status = query->status_dev;
  return launch_paged_attend_chosen(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_paged_prompt_chosen_workspace(const qkv_pages_t* pages, int32_t q_heads, int64_t tokens, uint64_t* bytes_out) {
  if (!bytes_out) return QKV_ERR_NULL;
  int rc = check_pages(pages, false);
  if (rc) return rc;
  rc = check_heads(pages, q_heads);
  if (rc) return rc;
  uint64_t floats = 0;
  rc = most_prompt_chosen_floats(pages, q_heads, tokens, floats);
  if (rc) return rc;
  *bytes_out = floats * sizeof(float);
  return QKV_OK;
}

int qkv_paged_prompt_chosen(const qkv_pages_t* pages, const qkv_paged_query_t* query, const uint32_t* choice_dev, void* stream) {
  int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!query || !query->starts_dev || !choice_dev) return QKV_ERR_NULL;
  rc = check_where(pages, query);
  if (rc) return rc;
  if (query->prior_out_dev || query->prior_lse_dev || query->window != 0) return QKV_ERR_SHAPE;
  PromptPlan plan;
  rc = plan_prompt_chosen(pages, query->q_heads, query->tokens, plan);
  if (rc) return rc;
  if (plan.floats != 0u && !query->workspace_dev) return QKV_ERR_NULL;
  if (query->workspace_bytes < plan.floats * sizeof(float)) return QKV_ERR_CAPACITY;
  if (misaligned(query->workspace_dev, 16) || misaligned(query->starts_dev, 4) || misaligned(choice_dev, 4)) return QKV_ERR_ALIGN;
  PagedPromptArgs a;
  set_prompt(pages, query, plan, a);
  a.choice = choice_dev;
  a.words = words_of(pages);
  return launch_paged_prompt_chosen(a, (uint32_t)pages->head_dim, pages->value_type == QKV_VALUE_BF16, static_cast<hipStream_t>(stream)) == hipSuccess
             ? QKV_OK : QKV_ERR_HIP;
}

int qkv_pages_slots(const qkv_pages_t* pages, const qkv_slots_t* slots, uint32_t* status_dev, void* stream) {
  const int rc = check_pages(pages, false);
  if (rc) return rc;
  if (!slots || !slots->starts_dev) return QKV_ERR_NULL;
  if (slots->tokens < 1 || slots->tokens >= (1ll << 27)) return QKV_ERR_SHAPE;
  if (misaligned(slots->more_dev, 4) || misaligned(slots->starts_dev, 4) || misaligned(slots->row_dev, 4) || misaligned(slots->place_dev, 4) ||
      misaligned(slots->slot_dev, 8) || misaligned(status_dev, 4))
    return QKV_ERR_ALIGN;
  SlotsArgs a;
  a.p = layer_of(pages, 0);
  a.more = slots->more_dev;
  a.tokens = (uint32_t)slots->tokens;
  a.starts = slots->starts_dev;
  a.row = slots->row_dev;
  a.place = slots->place_dev;
  a.slot = slots->slot_dev;
  a.status = status_dev;
  return launch_pages_slots(a, static_cast<hipStream_t>(stream)) == hipSuccess ? QKV_OK : QKV_ERR_HIP;
}

}  // extern "C"
