/*
 * qkvcard.h — C ABI of the CacheCard library for MI355X (gfx950).
 *
 * A CacheCard is the artifact one agent hands to the next (paper Sec. 4.2.1):
 * the sender's K/V cache as quantized groups, the token-level bit-width vector,
 * sequence length, model / sender identifiers, a position-offset placeholder and
 * the achieved average bit width.  The receiver rebuilds a dense fp16 K/V cache
 * from it before its next forward pass (paper Sec. 4.2.2).
 *
 * The paper fixes what a card carries, not its bytes; this header fixes the
 * bytes ("card layout v1").  All multi-byte fields are little-endian.
 *
 * Tensors.  K and V are fp16, contiguous [layers][kv_heads][tokens][head_dim]
 * (paper Sec. 3.1: K^(l,h), V^(l,h) in R^{n x d}).  A "plane" is one (kv, l, h)
 * matrix; planes are numbered p = kv*L*H + l*H + h with kv = 0 for K, 1 for V,
 * P = 2*L*H planes in all.  A "row" is the head_dim values of one token in one
 * plane.
 *
 * Bit widths.  Every token t has one width b(t) in {2, 4, 8, 16} shared by all
 * planes (paper Sec. 3.3); 16 means the fp16 row is carried unchanged.  Classes
 * are numbered 0..3 for widths 2, 4, 8, 16.
 *
 * Quantizer (per row, per group of G consecutive head_dim values, b < 16):
 *   mn, mx   = min / max of the group under the fp16 total order (-0 < +0)
 *   scale_h  = fp16_rne( (f32(mx) - f32(mn)) / (2^b - 1) )     fp32, IEEE division
 *   zero_h   = mn
 *   inv      = scale_h > 0 ? 1.0f / f32(scale_h) : 0           fp32, IEEE division
 *   code_i   = min(2^b - 1, rne_int( (f32(x_i) - f32(mn)) * inv ))
 *              (difference rounded to fp32, product exact, rounded once)
 *   decode   = fp16_rne( fma(f32(code_i), f32(scale_h), f32(zero_h)) )   fp32 fma
 * Code i of a row sits in bits [(i*b) mod 8, +b) of row byte floor(i*b/8).
 *
 * Card layout v1.  al(x) = x rounded up to a multiple of 256.  Sections, in order,
 * each starting 256-byte aligned, pad bytes zero:
 *   header            256 bytes, see qkv_card_header_t
 *   bits              u8 [T]           al(T)      the token-level bit-width vector
 *   slot              u32[T]           al(4T)     rank of t among tokens of its width
 *   order             u32[T]           al(4T)     tokens sorted by (class, t)
 *   codes_2, meta_2   [P][n2][D*2/8] bytes, then [P][n2][D/G]{fp16 scale, fp16 zero}
 *   codes_4, meta_4   likewise for the 4-bit tokens
 *   codes_8, meta_8   likewise for the 8-bit tokens
 *   fp16              [P][n16][D] raw fp16
 * Row j of a segment belongs to token order[base_c + j], base_c = number of tokens
 * in lower classes.  The card holds byte offsets only, so it can be copied, saved
 * and reloaded freely.
 *
 * Conventions for every entry point.
 *   - Return value: QKV_OK (0) or a negative QKV_ERR_* code.  Nothing is thrown or
 *     aborted across this boundary.  When an error is returned no output buffer has
 *     been written and no GPU work has been enqueued.
 *   - "device" pointers are HIP device memory of the current device; "host"
 *     pointers are ordinary process memory.  The caller owns every buffer; the
 *     library keeps no pointer to caller memory after a call returns and reads no
 *     environment variable.  Its only state between calls is the fixed scratch
 *     array of qkv_card_attend_static (one per GPU, its address looked up once).
 *   - No call allocates device memory except qkv_count_bits (32 bytes, freed before
 *     it returns).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  GPU
 *     work is enqueued there and the call returns without waiting, except where
 *     a function says it synchronises.
 *   - Supported shapes: head_dim in {64, 128, 256}; group_size in {32, 64, 128},
 *     group_size <= head_dim; layers, kv_heads, tokens >= 1; P * tokens < 2^32.
 */
#ifndef QKVCARD_H
#define QKVCARD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define QKV_OK             0
#define QKV_ERR_NULL      -1  /* a required pointer is NULL                                  */
#define QKV_ERR_SHAPE     -2  /* layers / kv_heads / tokens / head_dim outside the supported set */
#define QKV_ERR_GROUP     -3  /* group_size unsupported or not dividing head_dim              */
#define QKV_ERR_BUDGET    -4  /* average-bit budget outside [2, 16] or not finite             */
#define QKV_ERR_CAPACITY  -5  /* card buffer smaller than the card                            */
#define QKV_ERR_ALIGN     -6  /* a device pointer is not aligned as required                  */
#define QKV_ERR_COUNTS    -7  /* class counts negative or not summing to tokens               */
#define QKV_ERR_HIP       -8  /* a HIP runtime call failed                                    */
#define QKV_ERR_FORMAT    -9  /* card header is not a valid layout-v1 header (peek, flags)    */
#define QKV_ERR_OVERLAP   -10 /* an output buffer overlaps an input that is read meanwhile    */

#define QKV_CARD_VERSION        1u
#define QKV_CARD_HEADER_BYTES   256u
#define QKV_CARD_ALIGN          256u

/* bits in the status words written by the kernels */
/* Header flags. */
#define QKV_FLAG_KEYS_PER_CHANNEL 1u   /* uniform card whose key groups run along the tokens of a channel */

#define QKV_STATUS_BAD_BITS     0x1u  /* a bits[] value was not 2, 4, 8 or 16 (treated as 2)   */
#define QKV_STATUS_BAD_COUNTS   0x2u  /* counts[] passed by the host differ from the histogram */
#define QKV_STATUS_BAD_HEADER   0x4u  /* unpack: magic / version / shape / sizes do not match  */
#define QKV_STATUS_BAD_ORDER    0x8u  /* an order[] entry was >= tokens (row skipped / zeros)  */
#define QKV_STATUS_BAD_PAGE     0x10u /* a table entry that was needed names no page (its tokens are not seen / written) */
#define QKV_STATUS_BAD_ROW      0x20u /* a row number, a length or a row's place in a batch is not what it may be        */
#define QKV_STATUS_NO_PAGES     0x40u /* fewer free pages than the call needs (nothing was changed)                      */

/* Problem description, host memory, caller-owned (paper Sec. 3.1 shape, Sec. 4.2.1 metadata). */
typedef struct qkv_desc {
  int32_t  layers;          /* L                                                   */
  int32_t  kv_heads;        /* H: heads the cache stores (8 for Llama-3.1-8B)      */
  int32_t  head_dim;        /* D                                                   */
  int32_t  group_size;      /* G: consecutive head_dim values sharing scale / zero */
  int64_t  tokens;          /* T: sequence length                                  */
  uint64_t model_id;        /* opaque, copied into the header                      */
  uint64_t sender_id;       /* opaque, copied into the header                      */
  int64_t  position_offset; /* placeholder, stored, not interpreted                */
} qkv_desc_t;

/* The first 256 bytes of a card (paper Sec. 4.2.1: metadata and average-bit statistics). */
typedef struct qkv_card_header {
  uint8_t  magic[8];        /*   0  "QKVCARD\0"                                 */
  uint32_t version;         /*   8  QKV_CARD_VERSION                            */
  uint32_t header_bytes;    /*  12  256                                         */
  uint32_t layers;          /*  16                                              */
  uint32_t kv_heads;        /*  20                                              */
  uint32_t head_dim;        /*  24                                              */
  uint32_t group_size;      /*  28                                              */
  uint64_t tokens;          /*  32                                              */
  uint64_t count[4];        /*  40  tokens of width 2, 4, 8, 16                 */
  uint64_t total_bytes;     /*  72  size of the whole card                      */
  uint64_t off_bits;        /*  80  byte offsets of the sections from card start */
  uint64_t off_slot;        /*  88                                              */
  uint64_t off_order;       /*  96                                              */
  uint64_t off_codes[3];    /* 104  widths 2, 4, 8                              */
  uint64_t off_meta[3];     /* 128  widths 2, 4, 8                              */
  uint64_t off_fp16;        /* 152                                              */
  uint64_t model_id;        /* 160                                              */
  uint64_t sender_id;       /* 168                                              */
  int64_t  position_offset; /* 176                                              */
  float    avg_bits;        /* 184  (float)((double)sum of b(t) / (double)T)    */
  uint32_t flags;           /* 188  0, or QKV_FLAG_KEYS_PER_CHANNEL             */
  uint32_t status;          /* 192  QKV_STATUS_* bits set by the packing kernels */
  uint8_t  reserved[60];    /* 196  zero                                        */
} qkv_card_header_t;

/* Library version as major*10000 + minor*100 + patch.  Host only.  (A utility of the boundary; no passage of the
 * paper stands behind it.  The same holds for qkv_error_string.) */
int qkv_version(void);

/* Static, NUL-terminated text for a return code.  Host only; never NULL. */
const char* qkv_error_string(int code);

/*
 * Exact size in bytes of the card for `desc` and class counts {n2, n4, n8, n16}
 * (closed form of the layout above; the paper's size model, Sec. 3.1, is its
 * leading term).  Pure host integer arithmetic, no GPU call.
 *   desc, counts, bytes_out: host.  counts must be >= 0 and sum to desc->tokens.
 */
int qkv_card_bytes(const qkv_desc_t* desc, const int64_t counts[4], uint64_t* bytes_out);

/*
 * Class counts {n2, n4, n8, n16} that an average code-bit budget buys for T tokens
 * (paper Sec. 3.3: sum of b(t) stays within the budget).  Piecewise-linear between
 * three anchor mixes: all 2-bit at 2.0; 30 % / 40 % / 25 % / 5 % (2/4/8/16 bit) at
 * 5.0; all fp16 at 16.0.  Integer arithmetic on round(budget*1000), floors, so
 * sum b(t) <= budget*T.  Pure host arithmetic, no GPU call.
 */
int qkv_budget_counts(int64_t tokens, double avg_bits_budget, int64_t counts_out[4]);

/*
 * Bit-width assignment from per-token scores and a budget (paper Sec. 3.3: S(t)
 * decides b(t) under a memory budget).  Tokens are ranked by (score descending,
 * index ascending), scores compared in the IEEE total order (-0 < +0; NaN is a
 * precondition violation); the first n16 get 16, the next n8 get 8, the next n4
 * get 4, the rest 2, with the counts of qkv_budget_counts.
 *   scores_dev: device, float[T].   bits_dev: device, uint8_t[T], written.  Beyond 32768 tokens it
 *   holds intermediate counts until the call's last kernel: its bytes are widths only once all of the call's
 *   work has run.
 *   counts_out: host, int64_t[4], filled before return without a device sync.
 * Asynchronous on `stream`.
 */
int qkv_assign_bits(const float* scores_dev, int64_t tokens, double avg_bits_budget,
                    uint8_t* bits_dev, int64_t counts_out[4], void* stream);

/*
 * Histogram of a caller-made bits vector (uniform cards as in the paper's latency experiment, Sec. 5.3, or any
 * explicit mix): a utility that yields the class counts the card-building calls need; it restates no formula of
 * the paper.
 *   bits_dev: device, uint8_t[T].  counts_out: host, int64_t[4] for widths 2,4,8,16.
 * Values other than 2/4/8/16 are not counted (the sum then falls short of T).
 * Allocates and frees a small device scratch buffer and SYNCHRONISES `stream`.
 */
int qkv_count_bits(const uint8_t* bits_dev, int64_t tokens, int64_t counts_out[4], void* stream);

/*
 * Parameters of the extended controller's network (paper Sec. 4.1.2): a 2-layer MLP with 512
 * parameters over the 6 per-token features [frequency, quality, attention variance, entropy,
 * downstream demand, segment type].  The paper fixes neither hidden width, activation nor
 * output; here: 64 hidden units with ReLU and one linear output without bias
 * (6*64 + 64 + 64 = 512), the output being the combined score S(t) of Sec. 3.3.
 */
typedef struct qkv_controller {
  float w1[64][6];   /* hidden unit j, feature i */
  float b1[64];
  float w2[64];
} qkv_controller_t;

/*
 * Scores of the controller network for every token (paper Sec. 4.1.2).
 *   features_dev: device, float[T][6], row-major, 8-byte aligned.  Caller-owned, read only.
 *   params:       host; copied into the launch, may be freed on return.
 *   scores_dev:   device, float[T], written.
 * fp32 in a fixed order: hidden unit j = relu(fma chain over the features in order, starting
 * from b1[j]); score = fma chain over the hidden units in order, starting from +0.  A hidden
 * pre-activation that is NaN counts as 0.  Asynchronous on `stream`.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE (T < 1 or T >= 2^31), QKV_ERR_ALIGN, QKV_ERR_HIP.
 */
int qkv_controller_scores(const float* features_dev, int64_t tokens, const qkv_controller_t* params,
                          float* scores_dev, void* stream);

/*
 * Bit widths that follow the budgeted objective of paper Sec. 3.3 literally: minimise
 * sum_t eps(b(t)) * S(t) under sum_t b(t) <= avg_bits_budget * T, with the error model
 * eps(b) = 1 / (2^b - 1).  Every token starts at 2 bits; the upgrades 2->4, 4->8, 8->16 cost
 * 2, 4, 8 bits and gain max(S, 0) * {2/15, 4/255, 32/65535} per bit (one fp32 product with the
 * constant rounded to fp32; NaN scores count as 0).  All upgrades are ranked by (gain per bit
 * descending, level ascending, token index ascending) and the longest prefix whose cost fits
 * floor(budget * T) - 2T bits is taken; the budget is read as in qkv_assign_bits (rounded to
 * 1/1000 bit).  The class counts depend on the scores, so they are produced on the device:
 *   scores_dev: device, float[T], 4-byte aligned.   bits_dev: device, uint8_t[T], written (beyond
 *   32768 tokens intermediate counts first, as in qkv_assign_bits).
 *   counts_dev: device, uint64_t[4] for widths 2,4,8,16, 8-byte aligned, written; may be NULL.
 * Asynchronous on `stream`; allocates nothing.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE (T < 1 or T >= 2^28), QKV_ERR_BUDGET, QKV_ERR_ALIGN, QKV_ERR_HIP.
 */
int qkv_assign_bits_greedy(const float* scores_dev, int64_t tokens, double avg_bits_budget,
                           uint8_t* bits_dev, uint64_t* counts_dev, void* stream);

/*
 * CacheCard creation (paper Sec. 4.2.1): classify tokens by width and compact them
 * stably into per-width segments (slot, order), quantize and bit-pack K and V rows
 * at their token's width, copy 16-bit rows unchanged, write header and metadata.
 *   desc:     host.
 *   k_dev, v_dev: device, fp16 [L][H][T][D], 16-byte aligned, read only.  Values of
 *             tokens with b < 16 must be finite; 16-bit tokens may hold anything.
 *   bits_dev: device, uint8_t[T], values in {2,4,8,16}.
 *   counts:   host, {n2,n4,n8,n16}, must equal the histogram of bits_dev (it fixes
 *             the segment sizes before the device has looked at bits_dev).
 *   card_dev: device, 256-byte aligned, card_capacity >= qkv_card_bytes(desc, counts).
 *             Exactly qkv_card_bytes bytes are written, none beyond.
 * Faults only the device can see set header.status: QKV_STATUS_BAD_BITS,
 * QKV_STATUS_BAD_COUNTS.  The card is then unusable but every access stayed in bounds.
 * Asynchronous on `stream`.
 */
int qkv_quantize_pack(const qkv_desc_t* desc, const void* k_dev, const void* v_dev,
                      const uint8_t* bits_dev, const int64_t counts[4],
                      void* card_dev, uint64_t card_capacity, void* stream);

/*
 * The two halves of qkv_quantize_pack, for a sender that knows the widths before its K/V
 * are final (paper Sec. 4.2.1: the card's metadata - bit-width vector, sequence length,
 * identifiers, average-bit statistic - does not depend on the cache contents):
 *   qkv_card_plan  writes the header, the bits / slot / order tables and the section pads;
 *   qkv_card_fill  quantizes, packs and copies the K/V rows into a card planned with the
 *                  same desc and counts (it reads the card's order table, not bits_dev).
 * Arguments, alignment rules, error codes and status bits are those of qkv_quantize_pack;
 * plan followed by fill on one stream produces the same bytes.  Both are asynchronous.
 * qkv_card_fill trusts nothing it reads from the card: an order[] entry that names no token
 * (a card that was never planned, or was overwritten since) yields a row of zeros and sets
 * QKV_STATUS_BAD_ORDER in the status word at byte 192 of the card; no access leaves K, V or
 * the first qkv_card_bytes bytes of the card.
 */
int qkv_card_plan(const qkv_desc_t* desc, const uint8_t* bits_dev, const int64_t counts[4],
                  void* card_dev, uint64_t card_capacity, void* stream);
int qkv_card_fill(const qkv_desc_t* desc, const void* k_dev, const void* v_dev, const int64_t counts[4],
                  void* card_dev, uint64_t card_capacity, void* stream);

/*
 * Scores to a planned card in one step (paper Sec. 3.3: the score decides the width under the
 * budget; Sec. 4.2.1: the card's bit-width vector, sequence length, identifiers and average-bit
 * statistic).  Does what qkv_assign_bits followed by qkv_card_plan does - same widths, same
 * header, tables and pads, byte for byte - but without a second pass over the widths: whoever ranks
 * the scores already holds every token's width, so slots, order[] and the header follow at once
 * (one kernel up to 16384 tokens, a chain of five small ones beyond).
 *   desc:       host.  tokens < 2^31.
 *   scores_dev: device, float[T], 4-byte aligned (NaN is a precondition violation).
 *   bits_dev:   device, uint8_t[T], written; may be NULL (the widths are in the card anyway).
 *   counts_out: host, int64_t[4]: the budget's class counts (= qkv_budget_counts), filled before
 *               return without a device sync; pass them on to qkv_card_fill.
 *   card_dev:   device, 256-byte aligned, card_capacity >= qkv_card_bytes(desc, counts_out).  Beyond
 *               16384 tokens its slot and order tables hold intermediate counts until the call's last kernel.
 * qkv_card_fill on the same stream completes the card.  qkv_assign_quantize_pack is the two in
 * one call: scores, budget and K/V in, widths and the whole card out (k_dev, v_dev as for
 * qkv_quantize_pack).  Asynchronous on `stream`; allocate nothing.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE, QKV_ERR_GROUP, QKV_ERR_BUDGET, QKV_ERR_ALIGN,
 * QKV_ERR_CAPACITY, QKV_ERR_HIP.
 */
int qkv_assign_plan(const qkv_desc_t* desc, const float* scores_dev, double avg_bits_budget,
                    uint8_t* bits_dev, int64_t counts_out[4], void* card_dev, uint64_t card_capacity,
                    void* stream);
int qkv_assign_quantize_pack(const qkv_desc_t* desc, const void* k_dev, const void* v_dev,
                             const float* scores_dev, double avg_bits_budget, uint8_t* bits_dev,
                             int64_t counts_out[4], void* card_dev, uint64_t card_capacity, void* stream);

/*
 * Receiver-side injection (paper Sec. 4.2.2): unpack and dequantize a card into a
 * dense fp16 K/V cache.
 *   card_dev:   device, 256-byte aligned, card_bytes readable bytes.
 *   expect:     host; layers, kv_heads, head_dim, group_size, tokens the caller's
 *               output buffers were sized for (ids and position_offset ignored).
 *   k_out_dev, v_out_dev: device, fp16 [L][H][T][D], 16-byte aligned, written in full
 *               when the card is valid.
 *   status_dev: device uint32_t, may be NULL.  Set to 0 when the header matches
 *               `expect` and fits in card_bytes, else to QKV_STATUS_BAD_HEADER and
 *               the outputs are left untouched; QKV_STATUS_BAD_ORDER is or-ed in if
 *               a corrupt order[] entry was skipped.
 * The kernels read the class counts from the header on the device, so no host copy
 * of the card is needed.  Asynchronous on `stream`.
 */
int qkv_unpack_dequant(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                       void* k_out_dev, void* v_out_dev, uint32_t* status_dev, void* stream);

/*
 * Variant for uniform cards (every token at the same width 2, 4 or 8) with the keys grouped per
 * channel, after the per-channel key / per-token value scheme the paper cites as related work
 * (Sec. 2): key outliers live in a few channels, so a key group holds the 32 tokens
 * 32 tb .. 32 tb + 31 of ONE channel instead of 32 channels of one token; values keep per-token
 * groups.  Same quantizer, same card layout and sizes; in the key planes a code section reads
 * [plane][token block][channel][32 codes] and a pair section [plane][token block][channel]; the
 * header's flags word holds QKV_FLAG_KEYS_PER_CHANNEL.
 *
 * qkv_quantize_pack_kc / qkv_unpack_dequant_kc take the arguments of qkv_quantize_pack /
 * qkv_unpack_dequant and behave like them, with these extra conditions (QKV_ERR_SHAPE otherwise):
 * group_size 32, head_dim 64 or 128, tokens a multiple of 32 (of 64 at head_dim 64); and
 * (QKV_ERR_COUNTS) counts naming exactly one of the widths 2, 4, 8 for all tokens.  A card of
 * one grouping handed to the other grouping's call is refused on the device (QKV_STATUS_BAD_HEADER,
 * nothing written); qkv_inject_layers takes either grouping (its keys_per_channel field says
 * which), and qkv_card_attend_kc is qkv_card_attend for this grouping.
 */
int qkv_quantize_pack_kc(const qkv_desc_t* desc, const void* k_dev, const void* v_dev, const uint8_t* bits_dev,
                         const int64_t counts[4], void* card_dev, uint64_t card_capacity, void* stream);
int qkv_unpack_dequant_kc(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                          void* k_out_dev, void* v_out_dev, uint32_t* status_dev, void* stream);

/*
 * Receiver-side injection into per-layer caches (paper Sec. 4.2.2: the receiver rebuilds fp16
 * past_key_values, which frameworks keep as one key tensor and one value tensor per layer), for a
 * range of layers, so that injection can run layer by layer ahead of the receiver's forward
 * pass; optionally with the keys realigned to a shifted position (Sec. 3.2, challenge 2; the
 * card's position-offset field of Sec. 4.2.1 exists for this).
 *
 * Layer layer_begin + i of the card goes to k_layers[i] / v_layers[i]: device pointers to where
 * token 0 of head 0 lands; token t of head h lands h * head_stride + t * token_stride elements
 * further, as one contiguous row of head_dim fp16 values.  A cache of shape
 * [kv_heads][capacity][head_dim] that already holds a prefix of P tokens takes
 * head_stride = capacity * head_dim, token_stride = head_dim and pointers advanced by P rows.
 * Pointers 16-byte aligned, strides multiples of 8 elements, token_stride >= head_dim.  Any
 * other layout in which rows do not overlap works too (the library checks alignment and
 * token_stride only; it cannot see the tensors' extents).  The pointer arrays are host memory,
 * read before the call returns.
 *
 * Realignment (rope_base > 0): cached keys are assumed to carry rotary position embedding in the
 * half-split pairing (element i with i + head_dim/2, angle position * rope_base^(-2i/head_dim)).
 * Moving a key by rope_delta positions is one more rotation:
 *   theta_i = pow(rope_base, -2 i / head_dim)                      (double)
 *   c_i = (float)cos(rope_delta * theta_i), s_i = (float)sin(...)   (double, rounded to fp32)
 *   x'[i]     = fp16( fma(x[i],     c_i, -fl32(x[i+D/2] * s_i)) )
 *   x'[i+D/2] = fp16( fma(x[i+D/2], c_i, +fl32(x[i]     * s_i)) )
 * applied to the dequantized fp16 key values (and to 16-bit key rows, which must then be finite);
 * values are never rotated.  rope_base == 0 copies the keys as qkv_unpack_dequant does.
 *
 * Validation, status_dev and asynchrony as for qkv_unpack_dequant.  Allocates nothing.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE (layer range outside the card, layer_count < 1 or
 * > QKV_INJECT_MAX_LAYERS, bad strides - negative, not multiples of 8, token_stride < head_dim,
 * token_stride * tokens or head_stride * kv_heads >= 2^46 -, rope_base < 0 or not finite, |rope_delta| >= 2^31),
 * QKV_ERR_GROUP, QKV_ERR_CAPACITY, QKV_ERR_ALIGN, QKV_ERR_HIP.
 */
#define QKV_INJECT_MAX_LAYERS 64

typedef struct qkv_inject {
  int32_t layer_begin, layer_count;
  void* const* k_layers;            /* host array [layer_count] of device pointers */
  void* const* v_layers;
  int64_t head_stride, token_stride;  /* in fp16 elements */
  double rope_base;                 /* 0: no realignment */
  int64_t rope_delta;               /* positions to move the keys by */
  int32_t keys_per_channel;         /* 1: the card was made by qkv_quantize_pack_kc (its shape rules apply), else 0 */
  int32_t reserved;                 /* 0 */
} qkv_inject_t;

int qkv_inject_layers(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                      const qkv_inject_t* where, uint32_t* status_dev, void* stream);

/*
 * One hop of a multi-hop chain without the dense cache in between (paper Sec. 3.2, challenge 3:
 * error accumulates as a cache is forwarded from agent to agent; Sec. 4.2: the card is what
 * travels).  Builds, from an incoming card and new bit widths, exactly the card that
 * qkv_quantize_pack would build from the cache qkv_unpack_dequant rebuilds - byte for byte -
 * but moves only the two cards' bytes: every span is decoded and quantized again in registers.
 *   card_in_dev, card_in_bytes: the incoming card (device, 256-byte aligned, per-token groups);
 *               validated on the device like qkv_unpack_dequant does.  Where the card sits in a longer buffer, its own
 *               length is the better argument: results are the same, but the kernel is chosen by it.
 *   desc:       host; shape of both cards (must match the incoming header) and the identifiers
 *               and position offset that go into the outgoing header.
 *   bits_dev, counts: the new widths, as for qkv_quantize_pack.
 *   card_out_dev, card_out_capacity: as for qkv_quantize_pack; must not overlap the incoming card.
 *   status_dev: device uint32_t, may be NULL.  0, or QKV_STATUS_BAD_HEADER when the incoming
 *               card was refused (the outgoing card then holds header and tables but no rows),
 *               QKV_STATUS_BAD_ORDER or-ed in when a corrupt table entry of the incoming card was
 *               skipped (its rows are then zeros).
 * Asynchronous on `stream`; allocates nothing.
 * Errors: as qkv_quantize_pack; QKV_ERR_OVERLAP when the two cards' byte ranges intersect.
 */
int qkv_requantize(const void* card_in_dev, uint64_t card_in_bytes, const qkv_desc_t* desc,
                   const uint8_t* bits_dev, const int64_t counts[4], void* card_out_dev,
                   uint64_t card_out_capacity, uint32_t* status_dev, void* stream);

/*
 * Decode-step attention of one new query token directly over a card, without rebuilding
 * the dense cache (paper Sec. 4.3: consuming a foreign quantized cache inside attention,
 * which the paper names as its long-term goal).  For every layer l and query head hq, with
 * kv head h = hq / (q_heads / kv_heads):
 *     s_t = softmax_scale * <q[l][hq], K^[l][h][t]>,   t = 0 .. T-1
 *     out[l][hq] = sum_t softmax(s)_t * V^[l][h][t],   lse[l][hq] = log sum_t exp(s_t)
 * where K^, V^ are the dequantized fp16 values, exactly those qkv_unpack_dequant would
 * write (raw 16-bit rows as they are).  Scores are accumulated in fp32 from fp16 products,
 * the softmax and the weighted sum run in fp32; against the float64 definition a score is off
 * by at most head_dim * 2^-24 * softmax_scale * sum_i |q_i K^_ti| (summation order only), which
 * for caches of ordinary magnitude leaves out within a few units in 1e-6 of max|V^|.
 * Raw rows may hold anything: a score of -inf has a weight of zero, a value that is infinite or no number
 * makes its own dimension of out one; a head with a score that is +inf or no number has unspecified results.
 *   card_dev, card_bytes, expect, status_dev: as for qkv_unpack_dequant; head_dim 64, 128 or 256
 *             (the kernel is laid out for 128: at 64 it takes twice the tokens at a time, at 256 the
 *             head dimension in two halves), keys grouped per token.
 *   q_dev:    device, fp16 [layers][q_heads][head_dim], 16-byte aligned.  q_heads is a multiple
 *             of kv_heads, at most 16 query heads per kv head.
 *   out_dev:  device, float [layers][q_heads][head_dim], 16-byte aligned, written in full.
 *   lse_dev:  device, float [layers][q_heads], may be NULL.  With (out, lse) the caller can
 *             merge this result with attention over its own tokens.
 *   workspace_dev: device scratch of qkv_card_attend_workspace() bytes or more, 16-byte
 *             aligned; contents on entry and exit are unspecified.  workspace_bytes beyond that
 *             change nothing.  Short cards (up to 4 query heads per kv head, head_dim up to 128) are cut
 *             into more tasks than the call needs at least, and that size has room for them; a
 *             smaller workspace is accepted down to the one for the least number of tasks
 *             (QKV_ERR_CAPACITY below it).  With less than the full size the sums are taken in another
 *             order: out and lse then differ in their last bits, within the bound above, and the
 *             call takes longer.
 * When the header does not match, out / lse are left untouched (status_dev says so).
 * Asynchronous on `stream`.
 *
 * Several new tokens at once (a speculative window, a short suffix): every card token precedes
 * all of them, so no mask is needed and a "query head" may just as well be a (token, head) pair.
 * With S tokens and R = query heads per kv head, S * R <= 16, lay q out as
 * [layers][kv_heads][S][R][head_dim] and pass q_heads = kv_heads * S * R; out and lse come back in
 * the same order.  The card is then read once for all S tokens.
 */
int qkv_card_attend_workspace(const qkv_desc_t* expect, int32_t q_heads, uint64_t* bytes_out);
int qkv_card_attend(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                    const void* q_dev, int32_t q_heads, float softmax_scale,
                    float* out_dev, float* lse_dev, void* workspace_dev, uint64_t workspace_bytes,
                    uint32_t* status_dev, void* stream);

/*
 * qkv_card_attend for cards whose keys are grouped per channel (those of qkv_quantize_pack_kc; paper
 * Sec. 2 names the scheme, Sec. 4.3 the goal).  Same arguments, same results to the same bound, under
 * the shape rules of qkv_quantize_pack_kc (group_size 32: QKV_ERR_GROUP otherwise; head_dim 64 or 128,
 * tokens a multiple of 32, of 64 at head_dim 64: QKV_ERR_SHAPE otherwise).  There a key group holds 32
 * tokens of one channel, so the scores contract over the card's rows, the way the weighted sum of the
 * values does.  A card of the other grouping is refused on the device (QKV_STATUS_BAD_HEADER, nothing
 * written), and so does qkv_card_attend refuse a card of this one; qkv_card_flags says which a card is.
 */
int qkv_card_attend_kc(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                       const void* q_dev, int32_t q_heads, float softmax_scale,
                       float* out_dev, float* lse_dev, void* workspace_dev, uint64_t workspace_bytes,
                       uint32_t* status_dev, void* stream);

/*
 * qkv_card_attend for callers that cannot allocate device memory - code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc: the same kernels, the same results bit for
 * bit as with a workspace of at least qkv_card_attend_workspace() bytes, with the partials kept in a
 * fixed array inside the library instead of a caller's workspace.
 * Arguments as for qkv_card_attend, without the workspace.  The call allocates and frees nothing.
 *   - The array holds QKV_ATTEND_STATIC_SCRATCH_BYTES per GPU the library runs on, from the first
 *     call on that GPU until the process ends.  A shape whose qkv_card_attend_workspace() exceeds it
 *     is refused with QKV_ERR_CAPACITY (the Llama-3.1-8B shape at 8192 tokens with 32 query heads
 *     needs 13.3 MB; at 32768 tokens use qkv_card_attend with a workspace).
 *   - All calls on one GPU share the array: two calls that overlap in time on the same GPU (on
 *     different streams, or from different threads) race and give wrong results.  Calls on one
 *     stream are ordered by the stream.  Nothing in the array needs clearing between calls: every
 *     partial that counts has been written by the call itself.
 *   - The first call on a GPU looks the array's device address up with the runtime; make that
 *     first call outside a graph capture.
 */
#define QKV_ATTEND_STATIC_SCRATCH_BYTES (16u << 20)
int qkv_card_attend_static(const void* card_dev, uint64_t card_bytes, const qkv_desc_t* expect,
                           const void* q_dev, int32_t q_heads, float softmax_scale,
                           float* out_dev, float* lse_dev, uint32_t* status_dev, void* stream);

/*
 * A receiver's own cache, in pages, and the attention that reads it (paper Sec. 4.2.2: the receiver goes on from the injected cache
 * with tokens of its own; Sec. 4.3: attention over a card gives (out, lse), to be joined with attention over those tokens).
 * Several agents can go on from one injected context: their rows share its pages.
 *
 * The pool: per layer one tensor of keys and one of values, `pages` pages of page_tokens tokens.  Token i of page p, kv head h, starts
 * p * page_stride + h * head_stride + i * token_stride elements behind the layer's pointer and is one contiguous row of head_dim
 * 16-bit values.  Which sequence holds what is device memory of the caller's:
 *   lens_dev   [rows]              tokens of each sequence; 0 for a place that is not in use
 *   table_dev  [rows][row_pages]   entry j of a row: the page of tokens j * page_tokens and on.  Entries behind the last page a
 *                                  length needs mean nothing and are never looked at.
 *   refs_dev   [pages]             how many entries name the page; 0 is free.  Only qkv_pages_reserve / _fork / _free / _compact need it.
 * A page whose last tokens are not written yet belongs to one row only; the calls below keep it so.
 * The pointer arrays are host memory, read before a call returns.
 *
 * Shapes: layers 1 .. 64; head_dim 64, 128, 256; page_tokens a power of two up to 2^20; pages < 2^31; rows <= 65536; row_pages * page_tokens
 * (room for one sequence) and rows * row_pages < 2^31; strides multiples of 8 elements below 2^31, token_stride >= head_dim,
 * page_tokens * token_stride <= 2^30; layer pointers 16-byte aligned, others 4 (QKV_ERR_SHAPE, QKV_ERR_ALIGN).  The library cannot see the tensors' extents.
 *
 * What only the device sees never makes a call leave these tensors: lengths count as 0 .. row_pages * page_tokens, an entry that names no
 * page is QKV_STATUS_BAD_PAGE.  Status words: qkv_pages_reserve, _fork and _compact need one and set it (0 when all is well); the
 * other calls or their bits into it, where one is given, and clear nothing.
 * All calls are asynchronous on `stream` and allocate nothing.  Calls that share a pool belong on one stream, or are ordered by the caller.
 */
#define QKV_VALUE_FP16 0
#define QKV_VALUE_BF16 1

typedef struct qkv_pages {
  int32_t layers, kv_heads, head_dim, page_tokens;
  int32_t value_type;                 /* QKV_VALUE_* of keys, values and queries */
  int32_t pages, rows, row_pages;
  void* const* k_layers;              /* host array [layers] of device pointers */
  void* const* v_layers;
  int64_t page_stride, head_stride, token_stride;   /* in elements */
  int32_t* table_dev;
  int32_t* lens_dev;
  int32_t* refs_dev;                  /* NULL where it is not needed */
} qkv_pages_t;

/*
 * Makes room for new tokens: row i grows by more_dev[i] (device, int32_t[rows]; NULL: every row by 1).  Rows take new pages in their
 * order, the lowest free page first, and lens_dev holds the new lengths afterwards; qkv_pages_append then writes the tokens.
 * All or nothing: with a negative number, a length that the row has no entries for (QKV_STATUS_BAD_ROW) or too few free pages
 * (QKV_STATUS_NO_PAGES) nothing changes.
 */
int qkv_pages_reserve(const qkv_pages_t* pages, const int32_t* more_dev, uint32_t* status_dev, void* stream);

/*
 * Rows of new tokens into the pages of the sequences' last places.  Token i of row b, i = starts_dev[b] .. starts_dev[b + 1] - 1 of the
 * batch, goes to place lens_dev[b] - (starts_dev[b + 1] - starts_dev[b]) + (i - starts_dev[b]): lengths count the new tokens already.
 *   starts_dev: device, int32_t[rows + 1], rising; NULL: one token for every row (tokens == rows), which a row of length 0 leaves out.
 *   tokens: below 2^27.
 *   k_dev, v_dev: device, the new rows: layer l (counted from layer_begin), token i, head h start l * layer_stride + i * token_stride +
 *             h * head_stride elements behind it; strides multiples of 8, below 2^40, pointers 16-byte aligned.  A dense cache of
 *             qkv_unpack_dequant goes in with layer_stride = H*T*D, head_stride = T*D, token_stride = D.
 * Tokens behind the last row's are left out.  A place in front of the sequence or behind its entries is QKV_STATUS_BAD_ROW, and nothing is written.
 */
typedef struct qkv_rows {
  const void* k_dev;
  const void* v_dev;
  int64_t tokens;
  int64_t layer_stride, head_stride, token_stride;
  const int32_t* starts_dev;
  int32_t layer_begin, layer_count;
} qkv_rows_t;

int qkv_pages_append(const qkv_pages_t* pages, const qkv_rows_t* rows, uint32_t* status_dev, void* stream);

/*
 * Sequences that go on from another one: row target_dev[i] becomes what row source_dev[i] is (device, int32_t[count], 1 <= count <= rows).
 * What the targets held is given back first.  Full pages are shared: tokens that a source has room for are written before it is forked.  A last
 * page that is not full is copied (its tokens, in all layers) to a new page, the lowest free one, in the order of the pairs.  Targets are all
 * different and none is a source, else QKV_STATUS_BAD_ROW; with too few free pages QKV_STATUS_NO_PAGES; in both cases nothing has changed when
 * the call's work is done.
 */
int qkv_pages_fork(const qkv_pages_t* pages, const int32_t* source_dev, const int32_t* target_dev, int32_t count, uint32_t* status_dev,
                   void* stream);

/*
 * Pages given back by rows rows_dev[0 .. count) (NULL: all rows, count == rows).  window == 0: the rows hold nothing afterwards, lengths
 * are 0.  window > 0: only pages none of whose tokens a query at the row's last place or later sees (see qkv_paged_attend); their
 * entries become -1, lengths stay.  A row that is listed twice counts once; one that is none is QKV_STATUS_BAD_ROW.
 */
int qkv_pages_free(const qkv_pages_t* pages, const int32_t* rows_dev, int32_t count, int32_t window, int32_t sinks, uint32_t* status_dev,
                   void* stream);

/*
 * Moves the pages in use (refs > 0) to the pages 0 .. n - 1: the k-th page in use from n on goes to the k-th free page below n, in all layers;
 * entries and refs follow, live_dev (device, may be NULL) gets n.  Pages moved from keep their contents.
 * workspace_dev: device scratch of qkv_pages_compact_workspace() bytes, 16-byte aligned, contents unspecified (QKV_ERR_CAPACITY if smaller).
 */
int qkv_pages_compact_workspace(const qkv_pages_t* pages, uint64_t* bytes_out);
int qkv_pages_compact(const qkv_pages_t* pages, int32_t* live_dev, void* workspace_dev, uint64_t workspace_bytes, uint32_t* status_dev,
                      void* stream);

/*
 * Attention over the pages of one layer.  With R = q_heads / kv_heads (at most QKV_PAGED_MAX_REP) query head hq reads kv head hq / R; a query
 * at place p of its sequence sees the tokens t <= p and, with window > 0, of those only t > p - window and t < sinks:
 *     s_t = softmax_scale * <q, K_t>,   out = sum_t softmax(s)_t * V_t,   lse = log sum_t exp(s_t)
 * A query that sees nothing has out = 0, lse = -inf.  Tokens that are not seen count for nothing, whatever their rows hold.  Of those that are seen, one with
 * a score of -inf weighs nothing, a value that is infinite or no number makes its own dimension of out one; a head with a score that is +inf or no number has
 * unspecified results.
 *   q_dev:    device, values of the pages' type: query i, head hq start i * q_token_stride + hq * q_head_stride elements behind it; strides
 *             multiples of 8, 16-byte aligned, so a part of a fused projection's result will do.
 *   lse_dev:  device, float [tokens][q_heads], may be NULL.
 *   workspace_dev: device scratch, 16-byte aligned, contents unspecified, of the bytes the call's _workspace function names; NULL where
 *             that is 0.  Two calls that may run at once, graphs among them, need one each.  What qkv_paged_prompt_workspace names for a
 *             number of tokens is enough for every batch of that pool and q_heads with as many tokens or fewer.
 *
 * qkv_paged_attend: one new token of every sequence, p = lens_dev[i] - 1; tokens == rows, starts_dev NULL.  out is float
 * [rows][q_heads][head_dim], 16-byte aligned.  prior_out / prior_lse (float, shapes of out / lse, both or neither): the result of
 * attention over tokens that are somewhere else, qkv_card_attend's over a card above all; out and lse are then those of both together.
 * (prior_out may be out itself, and prior_lse lse.)  All sums in fp32; weights held to 22 bits, in fp16 those
 * below 2^-18 of the largest to 2^-40 of it.
 *
 * qkv_paged_prompt: many new tokens, whose keys and values are in the pages already: token i of row b (starts_dev as for qkv_pages_append,
 * here required, tokens >= 1) stands at place lens_dev[b] - n_b + (i - starts_dev[b]).  out is of the pages' type,
 * [tokens][q_heads][head_dim]; weights are rounded to that type for the product with the values, sums and lse are fp32.  out and lse of tokens
 * behind the last row's are left as they were; a row with more new tokens than length is QKV_STATUS_BAD_ROW (those in front see nothing).
 *
 * Limits: tokens * q_heads < 2^31; with G = ceil(R / 16) rows * kv_heads * G < 2^22 and rows * kv_heads * G * (row_pages * page_tokens / 32 + 3) < 2^31 for
 * qkv_paged_attend; with P = 128 / R, rounded down, (tokens / P + rows) * kv_heads < 2^23 for qkv_paged_prompt.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE (also: window < 0, sinks without a window, a scale that is not finite), QKV_ERR_ALIGN,
 * QKV_ERR_CAPACITY, QKV_ERR_HIP.
 */
#define QKV_PAGED_MAX_REP 128

typedef struct qkv_paged_query {
  const void* q_dev;
  int64_t q_token_stride, q_head_stride;   /* in elements */
  int64_t tokens;
  const int32_t* starts_dev;
  void* out_dev;
  float* lse_dev;
  const float* prior_out_dev;
  const float* prior_lse_dev;
  void* workspace_dev;
  uint64_t workspace_bytes;
  uint32_t* status_dev;
  int32_t layer, q_heads;
  int32_t window, sinks;
  float softmax_scale;
  int32_t reserved;                        /* 0 */
} qkv_paged_query_t;

int qkv_paged_attend_workspace(const qkv_pages_t* pages, int32_t q_heads, uint64_t* bytes_out);
int qkv_paged_attend(const qkv_pages_t* pages, const qkv_paged_query_t* query, void* stream);
int qkv_paged_prompt_workspace(const qkv_pages_t* pages, int32_t q_heads, int64_t tokens, uint64_t* bytes_out);
int qkv_paged_prompt(const qkv_pages_t* pages, const qkv_paged_query_t* query, void* stream);

/*
 * Attention over pages that a cheap score chooses for each query: where sequences are long - a whole injected context in front of the receiver's own
 * tokens (paper Sec. 4.2.2) - most pages weigh next to nothing for a given query.  Three steps, each a call:
 *   qkv_pages_digest           bounds of the keys of a page, once, when it has been filled
 *   qkv_paged_choose           the pages of every (query token, kv head), from those bounds
 *   qkv_paged_attend_chosen,   qkv_paged_attend and qkv_paged_prompt over the chosen pages
 *   qkv_paged_prompt_chosen
 *
 * A digest of a page, for one layer and kv head: per channel d an upper bound of its keys' values, then (head_dim further on) a lower one, as codes of the
 * step 2^e(d):
 *     hi(d) = sat8(ceil(max_t K_t(d) * 2^-e(d))),   lo(d) = sat8(floor(min_t K_t(d) * 2^-e(d))),   sat8: to -128 .. 127
 * A channel in which a key is no number has 127 and -128.  The steps are the caller's, the same for all pages of a layer, for instance for every channel
 * the smallest e with max |K(d)| <= 127 * 2^e over the first prompt; all int8_t values are allowed.  A digest belongs to the page: qkv_pages_fork needs
 * nothing for the pages it shares (and a page that is copied is not full), but after qkv_pages_compact digests are to be made again.
 *
 * A choice is a bit for each page of a sequence, bit j % 32 of word j / 32 for its page j, [tokens][kv_heads][(row_pages + 31) / 32] words.
 */
typedef struct qkv_digests {
  void* const* layers;                     /* host array [layers] of device pointers, 16-byte aligned: int8_t [pages][kv_heads][2][head_dim] */
  const int8_t* exponents_dev;             /* device, [layers][kv_heads][head_dim], 16-byte aligned: e */
} qkv_digests_t;

/*
 * Digests of the pages that new tokens have filled, in layers layer_begin .. layer_begin + layer_count - 1: of row b the full pages with a token among the
 * last n_b = starts_dev[b + 1] - starts_dev[b] of its lens_dev[b] (starts_dev and tokens as for qkv_pages_append, whose call has written them; starts_dev
 * NULL: one token for every row that has any, tokens == rows).  With n_b = lens_dev[b] that is all full pages of the row.  Digests of other pages stay.
 * An entry that names no page is QKV_STATUS_BAD_PAGE; a row whose starts lie outside the tokens or apart by more than its length is QKV_STATUS_BAD_ROW; both
 * are left out.  Limit: (tokens / page_tokens + rows) * kv_heads < 2^24.
 */
int qkv_pages_digest(const qkv_pages_t* pages, const qkv_digests_t* digests, const int32_t* starts_dev, int64_t tokens, int32_t layer_begin,
                     int32_t layer_count, uint32_t* status_dev, void* stream);

/*
 * Chooses pages for every query token and kv head, in whole numbers, so the result hangs on no order of summation.  A query at place p of its sequence has the
 * pages 0 .. o, o = p / page_tokens; those whose entry names no page are not there.  Of the others the first `first` (j < first) and the last `last` ones
 * (j > o - last) are chosen, and as many more as make `most` together: those with the highest score, of equal scores the lowest j.
 *   Query codes.  With the query heads r = 0 .. R - 1 of the kv head, in this order, in fp32:   P(d) = sum_r max(q_r(d), 0),   N(d) = sum_r min(q_r(d), 0)
 *   (a value that is no number counts as 0; sums are held to the largest finite numbers);   x = max_d (floor(log2(max(P(d), -N(d)))) + e(d)) over the d where that is not 0;
 *   p(d) = min(127, rne(P(d) * 2^(e(d) - x + 6))),   n(d) = max(-127, rne(N(d) * 2^(e(d) - x + 6)))    (all 0 where P and N are).
 *   Score of page j:   sum_d p(d) hi_j(d) + n(d) lo_j(d).   But for the rounding of the codes it bounds sum_r <q_r, K_t> over the page's tokens, for a
 *   softmax scale above 0.
 *   q_dev, strides, tokens, starts_dev, layer, q_heads: as for qkv_paged_prompt, or with starts_dev NULL as for qkv_paged_attend.
 *   most >= first + last, first >= 0, last >= 1: a query's own page, which need not be full, is never scored.  Digests of the full pages in front of it have to be there.
 *   choice_dev: device, uint32_t [tokens][kv_heads][(row_pages + 31) / 32], written in full; where a query has no place (p < 0) all bits are 0.  Words of tokens behind
 *             the last row's are left as they were.
 *   workspace_dev: device scratch of qkv_paged_choose_workspace() bytes, 16-byte aligned, contents unspecified; NULL where that is 0.  What is named for a number
 *             of tokens is enough for fewer.  Two calls that may run at once need one each.
 * Limits: row_pages < 2^20; tokens * kv_heads * 64 < 2^31; rows * kv_heads < 2^23, and for prompts (tokens / 16 + rows) * kv_heads < 2^23.
 * Errors: QKV_ERR_NULL, QKV_ERR_SHAPE, QKV_ERR_ALIGN, QKV_ERR_CAPACITY, QKV_ERR_HIP.
 */
typedef struct qkv_choose {
  const void* q_dev;
  int64_t q_token_stride, q_head_stride;   /* in elements */
  int64_t tokens;
  const int32_t* starts_dev;
  uint32_t* choice_dev;
  void* workspace_dev;
  uint64_t workspace_bytes;
  uint32_t* status_dev;
  int32_t layer, q_heads;
  int32_t most, first, last;
  int32_t reserved;                        /* 0 */
} qkv_choose_t;

int qkv_paged_choose_workspace(const qkv_pages_t* pages, int64_t tokens, uint64_t* bytes_out);
int qkv_paged_choose(const qkv_pages_t* pages, const qkv_digests_t* digests, const qkv_choose_t* choose, void* stream);

/*
 * qkv_paged_attend and qkv_paged_prompt over chosen pages: a query at place p sees the tokens t <= p of the pages j whose bit is set.  Everything else - arguments,
 * results, rounding, what is not seen, limits, errors - is as it is there; window and sinks are 0 (QKV_ERR_SHAPE).  Any bits will do: none, all, or a choice of the
 * caller's own.  Bits of pages behind a query's own mean nothing, as do those behind row_pages in a last word.
 *   choice_dev: device, uint32_t [tokens][kv_heads][(row_pages + 31) / 32].
 * Where sequences are short there is little to leave out, and finding it costs more than it saves: of prompts, 510 tokens of six sequences of up to 368 tokens take 25 us
 * with 8 pages of 16 each, where qkv_paged_prompt takes 17 over all of their tokens, and 1000 tokens behind 4000 58, where it takes 114 (32 / 8 heads of 128 dimensions, the
 * choice itself not counted; the two are even near 2000 tokens).
 *   most:     how many bits of a query are set, about; 0 if that is not known.  It guides how the work is cut, and decides with the shape how large
 *             the workspace has to be; results are right whatever is set.
 */
int qkv_paged_attend_chosen_workspace(const qkv_pages_t* pages, int32_t q_heads, int32_t most, uint64_t* bytes_out);
int qkv_paged_attend_chosen(const qkv_pages_t* pages, const qkv_paged_query_t* query, const uint32_t* choice_dev, int32_t most, void* stream);
int qkv_paged_prompt_chosen_workspace(const qkv_pages_t* pages, int32_t q_heads, int64_t tokens, uint64_t* bytes_out);
int qkv_paged_prompt_chosen(const qkv_pages_t* pages, const qkv_paged_query_t* query, const uint32_t* choice_dev, void* stream);

/*
 * The maps of a ragged batch, made on the device from how many new tokens each row has: what qkv_pages_append, qkv_pages_digest, qkv_paged_choose and
 * qkv_paged_prompt take as starts_dev, and where every token stands, for kernels of the caller's own (position embedding, a projection that writes its rows
 * into the pages itself).  Lengths count the new tokens already (qkv_pages_reserve).
 *   more_dev:   device, int32_t [rows]; NULL: one token for every row that has any.
 *   tokens:     room for tokens in the maps, 1 .. 2^27 - 1.
 *   starts_dev: device, int32_t [rows + 1], written: row b's tokens are starts_dev[b] .. starts_dev[b + 1] - 1 of the batch.
 *   row_dev, place_dev: device, int32_t [tokens], may be NULL: the token's row and its place in the sequence.
 *   slot_dev:   device, int64_t [tokens], 8-byte aligned, may be NULL: page * page_tokens + place % page_tokens; -1 where the entry names no page (QKV_STATUS_BAD_PAGE).
 * Maps hold -1 behind the last row's tokens, so that a batch may be padded to a fixed size.  A number below 0 or above the row's length counts as 0; a row whose
 * tokens do not fit has none, and neither have those behind it.  Both are QKV_STATUS_BAD_ROW.
 */
typedef struct qkv_slots {
  const int32_t* more_dev;
  int64_t tokens;
  int32_t* starts_dev;
  int32_t* row_dev;
  int32_t* place_dev;
  int64_t* slot_dev;
} qkv_slots_t;

int qkv_pages_slots(const qkv_pages_t* pages, const qkv_slots_t* slots, uint32_t* status_dev, void* stream);

/*
 * Read a card's header back to the host (paper Sec. 4.2.1: the card is self-describing - sequence length, identifiers,
 * position offset, achieved average bit width) and validate it (magic, version, shape
 * domain, counts summing to tokens, section offsets equal to the closed form,
 * total_bytes <= card_bytes).  Any out pointer may be NULL.  SYNCHRONISES `stream`.
 * Returns QKV_ERR_FORMAT for an invalid header (out values are then not written).
 */
int qkv_card_peek(const void* card_dev, uint64_t card_bytes, qkv_desc_t* desc_out,
                  int64_t counts_out[4], float* avg_bits_out, uint32_t* status_out,
                  void* stream);

/*
 * The flags word of a card's header: 0, or QKV_FLAG_KEYS_PER_CHANNEL for a card whose keys are
 * grouped per channel.  It tells a receiver which of qkv_unpack_dequant / qkv_unpack_dequant_kc
 * (and which keys_per_channel value of qkv_inject_layers) the card is for - the card is
 * self-describing (paper Sec. 4.2.1).  Validates the header like qkv_card_peek, and also that a
 * flagged card has a shape and widths that grouping allows; flags_out (host) is written only on
 * QKV_OK.  SYNCHRONISES `stream`.
 * Errors: QKV_ERR_NULL, QKV_ERR_FORMAT, QKV_ERR_HIP.
 */
int qkv_card_flags(const void* card_dev, uint64_t card_bytes, uint32_t* flags_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QKVCARD_H */
