/*
 * cocktail.h - C ABI of the chunk-level KV cache computation of Cocktail
 * (arXiv 2503.23294, Sec. III-C, Algorithm 1) for AMD MI355X (gfx950).
 *
 * The library covers the data-parallel hot path of the paper's second module.
 * Given the bitwidth (FP16 / INT8 / INT4 / INT2) that the chunk-level quantization
 * search (Sec. III-B) chose for every context chunk, it
 *   1. reorders the KV chunks so that every bitwidth class is contiguous in
 *      memory (Alg. 1, prefill loop; Fig. 3),
 *   2. quantizes and packs the INT2, INT4 and INT8 classes (Alg. 1, `quant`),
 *   3. runs single-query decode attention over the classes: logits of the
 *      INT2, INT4 (INT8) and FP16 blocks, one softmax over their concatenation, the
 *      att x V products of the blocks summed (Alg. 1, decode phase).  The concatenation is
 *      never materialised: each worker keeps a partial softmax state
 *      (max, sum, weighted V sum) and the states are merged exactly, which
 *      gives the same result because the softmax-weighted sum does not depend
 *      on the order or grouping of the tokens (Sec. III-C, Eq. 4-5).
 *
 * Conventions
 *   - Every pointer is marked HOST or DEVICE.  The library never allocates,
 *     frees or copies device memory and never synchronises the device (the one
 *     exception, cocktail_decode_check, says so); the GPU entry points only
 *     enqueue kernels on the caller's stream.
 *   - All functions return a cocktail_status; on failure a message is kept in
 *     thread-local storage (cocktail_last_error).  Arguments are validated on
 *     the host before anything is launched.
 *   - class index 0 = INT2, 1 = INT4, 2 = INT8, 3 = FP16: the concatenation order of Alg. 1 (INT2, INT4,
 *     FP16) with INT8, which Sec. I names as a further bitwidth, in its place by precision.
 *
 * Packed cache layout (an encoding defined by this library; the paper does not
 * fix one).  For each class c the K data and the V data live in one device
 * buffer each.  A buffer is a sequence of 64-token blocks ordered by
 * (sequence b, kv head h, block j); sequence b owns ceil(n_{b,c}/64) blocks per
 * head, n_{b,c} being its token count in class c (the FP16 runs of a plan made with
 * cocktail_plan_options::max_seq_lens own more: room for the tokens that may be folded in later, zero blocks
 * until then).  Inside a block:
 *   codes   the row of token i (i = 0..63) is cut into 16-byte pieces; piece p
 *           of token i is at byte (p*64 + i)*16.  Row size: D*bits/8 bytes for
 *           INT2/INT4/INT8, 2*D bytes (raw fp16, channel order) for FP16.
 *           A quantized row is a sequence of little-endian 32-bit words; word k
 *           covers the n = 32/bits channels k*n .. k*n+n-1, channel k*n+2f in
 *           bits [f*bits, f*bits+bits) and channel k*n+2f+1 in bits
 *           [16+f*bits, 16+f*bits+bits).
 *   meta    (quantized classes only) after the codes, at byte 64*rowbytes: for token i
 *           and group g of G consecutive channels, 4 bytes at (i*(D/G)+g)*4 =
 *           fp16 scale, then fp16 zero.  Value of a code: zero + code*scale.
 *   Tokens past n_{b,c} in the last block of a head are zero bytes.
 *   (At head_dim 64 a row is half as long, everything else is the same; group_size is then 32 or 64.)
 *   V in token quads (cocktail_sizes::v_layout == COCKTAIL_V_TOKEN_QUADS; chosen
 *   wherever a matrix kernel runs (Hq/Hkv >= 2 unless the plan is vector-ALU-only or Hq/Hkv > 8 has no divisor from
 *   2 to 8), where a wave serves several query heads of a kv head with matrix instructions and needs four tokens of a
 *   channel side by side):
 *   same block size, piece addressing and meta as above, but the 16-byte piece at
 *   slot sl no longer holds one token.  With n = 16/bits values per half-word,
 *   token i of the block and channel c are found at
 *     h = c / 64, j = (c % 32) / 8, e = 8 * ((c % 64) / 32) + c % 8,
 *     slot sl = 4 * (i / 4) + j, word w = 2 * (e / n) + (i % 4) / 2,
 *     piece (bits / 2) * h + w / 4 (a 64-channel half of a row is bits / 2 pieces), 32-bit word w % 4 of the piece, low (i even)
 *     or high (i odd) half-word, bits [(e % n) * bits, +bits).
 *   K always uses the row form.
 *
 * Quantizer (the paper names `quant` without defining it; this is the reading
 * used): per token, per group of G channels along head_dim, asymmetric min/max.
 * Every step is one IEEE binary32 operation, round-to-nearest-even, unfused:
 *   mn, mx = min, max of the group (zeros of either sign compare equal: a zero minimum or maximum is +0)
 *   scale  = fp16((f32(mx) - f32(mn)) / (2^bits - 1)),  zero = mn
 *   code   = 0 if scale == 0, else
 *            clamp(rint((f32(x) - f32(mn)) * (1.0f / f32(scale))), 0, 2^bits - 1)
 */
#ifndef COCKTAIL_H
#define COCKTAIL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define COCKTAIL_NUM_CLASSES 4
#define COCKTAIL_TOKENS_PER_BLOCK 64
#define COCKTAIL_MAX_Q_PER_KV 64
#define COCKTAIL_V_ROWS 0
#define COCKTAIL_V_TOKEN_QUADS 1

typedef enum cocktail_status {
  COCKTAIL_OK = 0,
  COCKTAIL_EINVAL = -1,       /* NULL pointer, non-positive size, bad chunk bit value, ...    */
  COCKTAIL_EUNSUPPORTED = -2, /* valid request this build has no kernel for                    */
  COCKTAIL_EALIGN = -3,       /* a device pointer is not 16-byte aligned                       */
  COCKTAIL_ENOSPACE = -4,     /* plan or workspace buffer smaller than required                */
  COCKTAIL_EHIP = -5,         /* the HIP runtime reported an error at launch                   */
  COCKTAIL_ESTATE = -6        /* cocktail_decode_check: the last decode call did not attend to every token once */
} cocktail_status;

/* Geometry of one attention layer call.  group_size divides head_dim. */
typedef struct cocktail_shape {
  int32_t batch;        /* B  sequences                                        */
  int32_t num_q_heads;  /* Hq query heads, a multiple of num_kv_heads          */
  int32_t num_kv_heads; /* Hkv                                                 */
  int32_t head_dim;     /* D, a multiple of 64 (kernels: 64 and 128)           */
  int32_t chunk_size;   /* C tokens per context chunk (Sec. III-A)             */
  int32_t group_size;   /* G in {32, 64, 128}: channels per scale/zero pair    */
} cocktail_shape;

/* Sizes the caller needs to allocate buffers; filled by cocktail_plan. */
typedef struct cocktail_sizes {
  int64_t total_chunks;                        /* sum_b floor(T_b / C): entries of perm            */
  int64_t class_tokens[COCKTAIL_NUM_CLASSES];  /* sum_b n_{b,c}                                    */
  int64_t class_blocks[COCKTAIL_NUM_CLASSES];  /* 64-token blocks in the K (= V) buffer of class c */
  int64_t class_bytes[COCKTAIL_NUM_CLASSES];   /* bytes of the K buffer, and of the V buffer       */
  int64_t plan_bytes;                          /* bytes of the plan blob                           */
  int64_t workspace_bytes;                     /* bytes of the decode-attention workspace          */
  int64_t packed_bytes;                        /* K+V bytes of codes + scale/zero, padding excluded */
  int32_t num_workers;                         /* waves the decode kernel is launched with, without those
                                                  of the append buffers                            */
  int32_t num_partials;                        /* partial softmax states written per call          */
  int32_t num_segments;
  int32_t append_capacity;                     /* tokens per sequence the append buffers can take  */
  int64_t append_bytes;                        /* bytes of the K append buffer, and of the V one   */
  int32_t v_layout;                            /* COCKTAIL_V_ROWS or COCKTAIL_V_TOKEN_QUADS: form of the V blocks */
  int32_t reserved;
} cocktail_sizes;

/* The packed mixed-precision cache of one layer: the six lists of Alg. 1
 * (K_q2, K_q4, K_fp16, V_q2, V_q4, V_fp16), an INT8 pair between the INT4 and the FP16 ones, and the plan
 * that describes them. */
typedef struct cocktail_cache {
  void* k[COCKTAIL_NUM_CLASSES]; /* DEVICE, class_bytes[c] each, 256-byte aligned; may be NULL iff 0 bytes */
  void* v[COCKTAIL_NUM_CLASSES]; /* DEVICE, same sizes                                                     */
  const void* plan_host;         /* HOST   plan blob written by cocktail_plan                              */
  void* plan_dev;                /* DEVICE byte-for-byte copy of the plan blob, 16-byte aligned; also holds
                                    the decode kernels' counters, the only part kernels write
                                    (see cocktail_decode_attention)                                        */
  void* k_app;                   /* DEVICE append_bytes each, 256-byte aligned: K/V rows of the tokens     */
  void* v_app;                   /*        generated during decoding; NULL iff append_capacity == 0         */
  int32_t num_appended;          /* tokens appended so far to every sequence, 0 .. append_capacity (batches
                                    that generate in lockstep); 0 if appended_dev is used                  */
  int32_t reserved;
  int32_t* appended_dev;         /* DEVICE int32 [B], or NULL: tokens appended so far per sequence, for batches
                                    whose sequences stop generating at different steps; read by
                                    cocktail_decode_attention, advanced by cocktail_append_fp16_ragged      */
} cocktail_cache;

/*
 * Host-only planning step (Alg. 1, prefill loop).
 * Computes the stable partition of every sequence's chunks by bitwidth, the token
 * count of every class (the FP16 class also receives the T_b mod C tail tokens,
 * Sec. III-A), the block layout of the packed cache and the static split of the
 * decode work over `num_workers` workers (waves).
 *
 *   seq_lens     HOST [B]           context tokens T_b >= 0
 *   chunk_bits   HOST [sum_b N_b]   N_b = floor(T_b / C) values in {2, 4, 8, 16}, sequence after sequence
 *   num_workers  most workers the decode kernel may be launched with (> 0), normally
 *                cocktail_default_workers(); a plan never has more workers than 32-token
 *                (head_dim 64: 64-token) units of work, rounded up to a multiple of 64:
 *                sizes->num_workers says how many it has
 *   sizes        HOST out, always written on success
 *   plan_host    HOST out, plan_capacity bytes, or NULL to query sizes only
 *   class_tokens HOST out [B][COCKTAIL_NUM_CLASSES] n_{b,c}, or NULL
 *   perm         HOST out [sum_b N_b]: position j of sequence b's reordered chunk
 *                list holds original chunk perm[off_b + j] (the x_j of Eq. 5), or NULL
 *
 * Errors: EINVAL (NULL, bad shape, bad bit value), ENOSPACE (plan_capacity too small).
 * The plan blob is position independent: copy its plan_bytes bytes to the device
 * unchanged.  The host arrays may be freed on return.
 */
int cocktail_plan(const cocktail_shape* shape, const int32_t* seq_lens, const uint8_t* chunk_bits,
                  int32_t num_workers, cocktail_sizes* sizes, void* plan_host, size_t plan_capacity,
                  int32_t* class_tokens, int32_t* perm);

/* Options of cocktail_plan_ex; zero-initialise, then set what is needed. */
typedef struct cocktail_plan_options {
  int32_t append_capacity; /* >= 0: generated tokens per sequence the cache can take (Sec. III-A keeps their K/V
                              in FP16 behind the context).  They live in two extra buffers
                              (cocktail_cache::k_app, v_app; sizes->append_bytes each): per (sequence, kv head)
                              ceil(append_capacity / 64) blocks in the block layout of the FP16 class, ordered
                              (b, h, block).                                                                  */
  int32_t reproducible;    /* != 0: purely static split of the decode work (no shared pools): calls on the same
                              inputs then agree bit for bit, at some cost in speed                            */
  int32_t vector_alu_only; /* != 0: grouped-query shapes are planned for the kernel that runs one query head per wave
                              on the vector ALU alone (no matrix instructions, V in token rows); every query head
                              then reads the blocks of its kv head by itself                                    */
  int32_t reserved0;       /* must be zero                                                                    */
  const int32_t* max_seq_lens; /* HOST [B] or NULL: the context length every sequence may reach when generated tokens
                              are folded into the packed cache (cocktail_fold_appended; Sec. III-A: they stay FP16).
                              The FP16 run of every (sequence, kv head) is laid out with room for
                              max_seq_lens[b] - seq_lens[b] more tokens (zero blocks after reorder+quantize), so a
                              plan for a longer context with the same max_seq_lens has the same cache layout.
                              max_seq_lens[b] >= seq_lens[b].                                                   */
  int32_t reserved[2];     /* must be zero                                                                    */
} cocktail_plan_options;

/* cocktail_plan with options (NULL = defaults = cocktail_plan). */
int cocktail_plan_ex(const cocktail_shape* shape, const int32_t* seq_lens, const uint8_t* chunk_bits,
                     int32_t num_workers, const cocktail_plan_options* options, cocktail_sizes* sizes,
                     void* plan_host, size_t plan_capacity, int32_t* class_tokens, int32_t* perm);

/* Source layouts accepted by cocktail_reorder_quantize (element = one fp16). */
#define COCKTAIL_SRC_STRIDED 0 /* element (b,h,t,d) at b*stride_b + h*stride_h + t*stride_t + d        */
#define COCKTAIL_SRC_RAGGED 1  /* sequences concatenated; sequence b is [Hkv][T_b] rows of stride_t
                                  elements, starting at (sum_{b'<b} T_b') * Hkv * stride_t              */

/*
 * Prefill side of Alg. 1: gather every chunk into its class (reorder), then
 * quantize and pack the INT2, INT4 and INT8 classes; FP16 chunks and the tail are
 * copied.  One kernel launch handles K and V of all classes.
 *
 *   k_src, v_src  DEVICE fp16, 16-byte aligned, head_dim contiguous; strides in
 *                 elements, multiples of 8
 *   cache         k/v buffers are written completely (padding included), the append
 *                 buffers (if any) are zeroed; num_appended is not read;
 *                 plan_host/plan_dev must come from cocktail_plan for this shape
 *   stream        hipStream_t (NULL = default stream)
 *
 * Inputs must be finite.  Errors: EINVAL, EUNSUPPORTED (head_dim other than 64 or 128),
 * EALIGN, EHIP.  Nothing is launched when an error is returned.
 */
int cocktail_reorder_quantize(const cocktail_shape* shape, const void* k_src, const void* v_src,
                              int32_t src_layout, int64_t stride_b, int64_t stride_h, int64_t stride_t,
                              const cocktail_cache* cache, void* stream);

/*
 * The same prefill step from a paged KV cache, the way serving stacks keep K and V between prefill and
 * decode: two pools of fixed-size pages (one for K, one for V, same geometry) and a page table per
 * sequence.  Token t of sequence b, kv head h, channel d is the fp16 element at
 *     page_table[b * table_stride + t / page_size] * stride_page + h * stride_h + (t % page_size) * stride_t + d
 * of k_pages (v_pages).  Blocks whose 64 tokens lie inside one page are read with one base address, the
 * others row by row; any page_size >= 1 works, multiples of 64 are fastest.
 *
 *   k_pages, v_pages  DEVICE fp16, 16-byte aligned; strides in elements, multiples of 8, stride_t >= head_dim
 *   page_table        DEVICE int32 [B][table_stride]; row b names the ceil(T_b / page_size) pages of sequence b
 *                     in token order; entries behind them are not read.  An entry outside [0, num_pages) is
 *                     not followed: the rows of that page are quantized as zeros.
 *   cache, stream     as cocktail_reorder_quantize
 *
 * Errors: EINVAL (NULL, bad page geometry, a page table row too short for its sequence), EUNSUPPORTED, EALIGN, EHIP.
 */
typedef struct cocktail_paged_source {
  const void* k_pages;
  const void* v_pages;
  const int32_t* page_table;
  int32_t table_stride; /* entries per page table row                      */
  int32_t page_size;    /* tokens per page                                 */
  int32_t num_pages;    /* pages in each pool                              */
  int32_t reserved;     /* must be zero                                    */
  int64_t stride_page, stride_h, stride_t;
} cocktail_paged_source;

int cocktail_reorder_quantize_paged(const cocktail_shape* shape, const cocktail_paged_source* src,
                                    const cocktail_cache* cache, void* stream);

/*
 * Decode side of Alg. 1: out[b,h] = softmax(sm_scale * q[b,h] . K^_b^T) V^_b over
 * all tokens of all classes of sequence b, K^/V^ being the dequantized
 * (or raw fp16) rows of kv head h / (Hq/Hkv).  Two launches: partial states per
 * worker, then the exact merge.  Short contexts take one launch (plans whose cocktail_plan_field "short_groups" is not 0): the workgroups of a
 * (sequence, set of query heads that a wave serves) count themselves in the device copy of the plan, and the last one merges.  Workers that finish their own share early take
 * further pieces from a pool shared by a few neighbouring workers; the pools are
 * handed out through ticket counters that live in the device copy of the plan as well.
 * All these counters are zero in the blob cocktail_plan writes and every call leaves
 * them zero again, so calls on the same plan_dev must not overlap in time (calls
 * on one stream never do), and a plan_dev whose call was aborted has to be
 * re-uploaded.  A call that breaks this rule is not silently wrong: every partial
 * state records how many tokens it covers, the merge compares their sum with the
 * token count of the sequence, and a (sequence, query head) row that does not add
 * up gets NaN in out and lse and a non-zero status word (cocktail_decode_check);
 * the call after it finds the ticket counters at zero again.  The workgroups of the one
 * launch notice a counter that was not zero, or that another call adds to, and put it back
 * to zero: calls one behind the other are right whatever it was, and of calls that overlap
 * a row may end up merged by nobody, which is NaN and reported like the above.  Which worker takes which pool piece differs from call to call, so
 * two calls on the same inputs agree to fp32 summation order, not bit for bit
 * (plans made with cocktail_plan_options::reproducible use no pools and are reproducible bit for bit, and so are
 * plans on matrix instructions whose waves serve five to eight query heads: Hq/Hkv of 5 to 8, and the larger
 * ratios whose largest divisor up to 8 is at least 5, such as 10, 12 and 16 but not 9, 11 or 13.  Which other plans
 * have pools is a matter of speed and no contract; cocktail_plan_field "num_pool_segs" is 0 for one without).  Shapes with
 * Hq = Hkv run one query head per wave on the vector ALU; 2 <= Hq/Hkv <= 8 run all query heads of a kv head in one
 * wave on matrix instructions (4x4x4 up to four heads, 16x16x32 beyond; V in token quads), unless the plan asks for
 * the vector ALU only; for larger ratios (up to COCKTAIL_MAX_Q_PER_KV) the query heads of a kv head are cut into equal
 * sets, of as many heads as that divisor, that each read the kv head's blocks (one head per wave if it is 1).
 *
 *   cache      the appended tokens (num_appended of every sequence, or appended_dev[b] of sequence b) are
 *              attended to after the context
 *   q          DEVICE fp16 [B][Hq][D], 16-byte aligned
 *   sm_scale   softmax scale; <= 0 selects 1/sqrt(D)
 *   out        DEVICE fp16 [B][Hq][D]; a sequence with no tokens yields zeros
 *   lse        DEVICE fp32 [B][Hq] natural-log-sum-exp of the scaled logits
 *              (-inf for an empty sequence), or NULL
 *   workspace  DEVICE, workspace_bytes >= sizes.workspace_bytes, 16-byte aligned;
 *              contents need not be initialised and are overwritten (partial states,
 *              then one status word per (sequence, query head)).  Calls that share a
 *              workspace must not overlap in time.
 *
 * The packed K/V data is not modified.  Errors: EINVAL, EUNSUPPORTED (head_dim other than 64 or 128,
 * Hq/Hkv > COCKTAIL_MAX_Q_PER_KV), EALIGN, ENOSPACE, EHIP.
 */
int cocktail_decode_attention(const cocktail_shape* shape, const void* q, const cocktail_cache* cache,
                              float sm_scale, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * Measurement aid: cocktail_decode_attention that also records `event_between` (a hipEvent_t created by the
 * caller with timing enabled) on `stream` between its two kernels, so that the partial-state kernel (Alg. 1
 * decode phase, the kernel that streams the cache) and the merge can be timed apart with events on the launch
 * stream.  The record itself sits between the kernels: time whole calls with cocktail_decode_attention, which
 * takes one launch for short contexts where this call always takes two.
 * Errors: as cocktail_decode_attention; EINVAL if event_between is NULL; EHIP if the record fails.
 */
int cocktail_decode_attention_marked(const cocktail_shape* shape, const void* q, const cocktail_cache* cache,
                                     float sm_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                     void* stream, void* event_between);

/*
 * cocktail_decode_attention for callers that cannot allocate device memory or hand over a workspace: code
 * that runs under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * same kernels and same results, but the partial states go to a workspace built into the library: a
 * static device array of COCKTAIL_STATIC_WORKSPACE_BYTES_TILES that every GPU the library runs on holds until the
 * process ends.  The call allocates and frees nothing, on the device or through any library.
 *
 * Every call on a GPU shares that GPU's array, so calls that overlap in time on one GPU (two streams, two
 * threads) race; nothing in it has to survive from one call to the next.  The array's address is looked up
 * on the first call on each device (with that device current): make that call outside a graph capture.
 *
 * Errors: as cocktail_decode_attention, and ENOSPACE if the plan's workspace_bytes exceeds
 * COCKTAIL_STATIC_WORKSPACE_BYTES (the five benchmark shapes need 0.1 to 5.2 MB), or
 * COCKTAIL_STATIC_WORKSPACE_BYTES_TILES where one wave serves five to eight query heads (more and larger partial states) or
 * the query heads of a kv head are cut into sets on matrix instructions (Hq/Hkv > 8: more partial states).
 */
#define COCKTAIL_STATIC_WORKSPACE_BYTES (16u << 20)
#define COCKTAIL_STATIC_WORKSPACE_BYTES_TILES (24u << 20)
int cocktail_decode_attention_static(const cocktail_shape* shape, const void* q, const cocktail_cache* cache,
                                     float sm_scale, void* out, float* lse, void* stream);

/*
 * Diagnostic: waits for `stream`, then reads the status words the last decode call on `workspace` left
 * (the only entry point that synchronises and copies).  The softmax of Alg. 1's decode phase runs over the
 * concatenation of all classes, i.e. over every token of the sequence exactly once; the status word
 * of a (sequence, query head) is the number of tokens its partial states covered minus the sequence length (a row
 * that was not merged at all: one less than if they had covered none).
 *
 *   workspace  DEVICE, the workspace of that call; NULL = the built-in one of cocktail_decode_attention_static
 *
 * Nothing is written.  Returns COCKTAIL_OK if every word is zero, else COCKTAIL_ESTATE with a message naming the first bad row
 * (see cocktail_decode_attention for the causes).  Other errors: EINVAL, EHIP.
 */
int cocktail_decode_check(const cocktail_shape* shape, const cocktail_cache* cache, const void* workspace,
                          void* stream);

/*
 * Sec. III-A: stores the K/V rows of one generated token per sequence, in FP16, as token `position`
 * (0-based) of the append buffers.  The caller then sets cache->num_appended = position + 1 (or higher)
 * for the following cocktail_decode_attention calls, which attend to the context and to the first
 * num_appended appended tokens of every sequence.
 *
 *   k_new, v_new  DEVICE fp16 [B][Hkv][D], 16-byte aligned
 *   position      0 <= position < append_capacity of the plan
 *
 * One kernel launch.  Errors: EINVAL (no append buffers, position out of range, NULL), EALIGN, EHIP.
 */
int cocktail_append_fp16(const cocktail_shape* shape, const void* k_new, const void* v_new,
                         const cocktail_cache* cache, int32_t position, void* stream);

/*
 * Sec. III-A for a batch whose sequences generate (and stop) independently: for every sequence b with
 * active_dev[b] != 0 the K/V rows of its new token are stored as appended token cache->appended_dev[b] of that
 * sequence, then appended_dev[b] is advanced by one; the rows of the other sequences are ignored.  A sequence
 * whose append buffer is full (appended_dev[b] == append_capacity) is left as it is.  The following
 * cocktail_decode_attention calls attend to the context and to the first appended_dev[b] appended tokens of
 * every sequence.  Counts and flags live on the device, so a decode loop needs no host round trip.
 *
 *   k_new, v_new  DEVICE fp16 [B][Hkv][D], 16-byte aligned
 *   cache         appended_dev must not be NULL (zero it before the first token; cocktail_reorder_quantize
 *                 does not touch it)
 *   active_dev    DEVICE uint8 [B], or NULL = every sequence
 *
 * Two kernel launches (store, then advance the counts).  Errors: EINVAL, EUNSUPPORTED, EALIGN, EHIP.
 */
int cocktail_append_fp16_ragged(const cocktail_shape* shape, const void* k_new, const void* v_new,
                                const cocktail_cache* cache, const uint8_t* active_dev, void* stream);

/*
 * Sec. III-A, for long generations: the tokens appended so far become context.  Their K/V rows move from the
 * append buffers into the packed cache, behind the FP16 rows of their (sequence, kv head) (they stay FP16 and keep
 * their place in the order of the tokens: the FP16 list of Alg. 1 grows at its end, nothing is quantized again), so
 * that the decode work split of a new plan covers them like any other token instead of leaving them to the few
 * waves that serve the append buffers.
 *
 *   cache          the cache as it is: plan_host / plan_dev = the plan in use (made with append buffers and with
 *                  cocktail_plan_options::max_seq_lens), class and append buffers, appended_dev or num_appended
 *   new_plan_host  HOST plan of the longer contexts: seq_lens[b] + (tokens appended to sequence b), chunk_bits
 *                  extended by 16 for every chunk the new tokens complete, the same shape and the same
 *                  max_seq_lens, hence the same cache layout (checked)
 *   new_plan_dev   DEVICE copy of new_plan_host, 16-byte aligned, complete before this call runs on `stream`
 *
 * Every sequence is folded completely: new seq_lens[b] - old seq_lens[b] has to be the number of tokens appended
 * to sequence b (checked against num_appended for batches in lockstep; with appended_dev the counts live on the
 * device and are the caller's to match).  Afterwards the caller switches cache->plan_host and cache->plan_dev to
 * the new plan and sets num_appended = 0; appended_dev is cleared by this call.  The workspace of the new plan may
 * be larger than the old one's.
 *
 * One or two kernel launches.  Errors: EINVAL (plans that differ in more than FP16 tokens at the end, counts out of
 * range, NULL), EUNSUPPORTED, EALIGN, EHIP.
 */
int cocktail_fold_appended(const cocktail_shape* shape, const cocktail_cache* cache, const void* new_plan_host,
                           const void* new_plan_dev, void* stream);

/*
 * Chunk-level quantization search (Sec. III-B): scores[i] = cosine similarity of sequence b's query
 * embedding with chunk embedding i (Eq. 1); per sequence T_low = s_min + (s_max - s_min) * alpha and
 * T_high = s_max - (s_max - s_min) * beta (Eq. 2-3); chunk_bits[i] = 2 if scores[i] < T_low, else 16
 * if scores[i] > T_high, else 4 (the comparisons of Alg. 1's prefill loop, in that order).  The
 * embeddings come from the caller's encoder.  Arithmetic: sums in binary64, the score rounded once
 * to binary32 (0 if either vector is zero), thresholds and comparisons in unfused binary32.
 *
 *   chunk_off   DEVICE int32 [B+1]  prefix sum of the chunk counts N_b (chunk_off[B] = total_chunks)
 *   query_emb   DEVICE fp32 [B][E]
 *   chunk_emb   DEVICE fp32 [total_chunks][E], sequence after sequence
 *   alpha, beta in [0, 1] (the paper uses 0.6 and 0.1)
 *   scores      DEVICE fp32 [total_chunks] out
 *   chunk_bits  DEVICE uint8 [total_chunks] out, values 2 / 4 / 16: copy to the host for cocktail_plan
 *
 * Two kernel launches.  Errors: EINVAL, EALIGN, EHIP.
 */
int cocktail_chunk_bitwidths(int32_t batch, int32_t embed_dim, int32_t total_chunks, const int32_t* chunk_off,
                             const float* query_emb, const float* chunk_emb, float alpha, float beta, float* scores,
                             uint8_t* chunk_bits, void* stream);

/*
 * Number of decode workers (waves) that fills the current HIP device for this shape
 * (compute units x resident waves per unit).  Needs a GPU: EHIP otherwise.
 */
int cocktail_default_workers(const cocktail_shape* shape, int32_t* num_workers);

/*
 * Measurement aid, not a step of the method: enqueues a plain 128-bit streaming read of
 * `buf` (2048 single-wave workgroups, each over one contiguous range), so that a benchmark
 * can report the HBM read rate this GPU reaches with loads alone beside the rate of the
 * decode kernel (whose cost the paper attributes to loading the KV cache, Sec. I).
 *
 *   buf         DEVICE, 16-byte aligned, `bytes` >= 16 MiB readable bytes
 *   sink        DEVICE, 4 bytes the kernel may write
 *   bytes_read  HOST out: bytes the launch reads (`bytes` rounded down to 16 MiB)
 *
 * Errors: EINVAL, EALIGN, EHIP.
 */
int cocktail_stream_read_probe(const void* buf, size_t bytes, void* sink, size_t* bytes_read, void* stream);

/*
 * Diagnostic, not a step of the method.  The quantizer (top of this file) is defined by IEEE binary32
 * divisions; the kernel replaces them by shorter sequences that are exact on the operands that can
 * occur.  This call checks that claim on the device for every such operand: all floats in [0, 131008]
 * for (mx - mn) / 3, / 15 and / 255, and every positive finite fp16 value for 1 / scale.
 *
 *   mismatches  DEVICE uint64 [4] out, 16-byte aligned: operands on which the result differs from the
 *               division, for / 3, / 15, 1 / scale, / 255.  All zero on a correct device.
 *
 * Two kernel launches (about a millisecond).  Errors: EINVAL, EALIGN, EHIP.
 */
int cocktail_selftest_arithmetic(uint64_t* mismatches, void* stream);

/*
 * Debugging aid: value of one field of the plan header (the internal layout of the blob cocktail_plan writes),
 * by the name it has in the library's source, e.g. "off_counters", "num_groups", "class_blocks" (index =
 * class), plus a few constants of the layout ("counter_stride_bytes", "iter_units", "sizeof_worker_rec", ...) and the waves
 * per workgroup a decode call on the plan is launched with ("workgroup_waves").
 * Errors: EINVAL (not a plan of this library version, unknown name, index out of range).
 */
int cocktail_plan_field(const void* plan_host, const char* name, int32_t index, int64_t* value);

/* ======================================= A paged cache in 4 bits ======================================= */

/*
 * Sequences of a serving batch whose K and V live in pages: which pages a sequence has, how long it is, and how many sequences
 * hold a page.  All of it lives on the device, so that a generation loop needs no host round trip and can be captured into a
 * graph.  Any number of pools (K and V of every layer) can be addressed by one table.
 *
 *   table     page of every page_size tokens of a sequence, in token order; -1 behind the ceil(len / page_size) pages it has
 *   seq_lens  tokens of the sequence
 *   refs      table entries that name the page; 0 = free
 *   status    [0]: 0, or why the last cocktail_pages_resize did nothing: the number of pages that were missing, -1 if a row of
 *             the table was too short, -2 if a shared page had to be copied and no pools were given; [1..3] zero
 * To start with every entry of the table is -1 and the rest is zero.
 */
#define COCKTAIL_MAX_SEQS 4096
#define COCKTAIL_MAX_POOLS 256
typedef struct cocktail_page_table {
  int32_t* table;       /* DEVICE [num_seqs][table_stride]                                            */
  int32_t* seq_lens;    /* DEVICE [num_seqs]                                                          */
  int32_t* refs;        /* DEVICE [num_pages]                                                         */
  int32_t* status;      /* DEVICE [4]                                                                 */
  int32_t num_seqs;     /* 1 .. COCKTAIL_MAX_SEQS                                                     */
  int32_t table_stride; /* pages a sequence can have; table_stride * page_size and num_seqs * table_stride < 2^31 */
  int32_t page_size;    /* tokens per page                                                            */
  int32_t num_pages;    /* pages of every pool                                                        */
} cocktail_page_table;

/* Bytes of the workspace that cocktail_pages_resize and cocktail_pages_compact take (host only). */
int cocktail_pages_workspace(const cocktail_page_table* pages, size_t* bytes);

/*
 * Every sequence b becomes delta[b] tokens longer (shorter if negative; never shorter than 0, so that a large negative value
 * frees the sequence).  Pages behind the new end are given back (refs - 1).  Pages that are lacking are taken: the lowest-numbered
 * ones that were free when the call began, sequence after sequence.  A sequence that grows out of a partly filled page which
 * other sequences hold takes a copy of it first (before its further pages), so that what it stores there is its own; where a page
 * is held by growing sequences only, the last of them keeps it.  The copies are made in all `num_pools` pools.
 * All or nothing: if pages are lacking, or the table has too few columns, nothing changes and status[0] says so; the
 * cocktail_fp4_store calls that follow then store nothing, until a resize succeeds; all other calls go by the lengths as they are (cocktail_pages_check
 * tells).
 *
 *   delta       DEVICE int32 [num_seqs]
 *   pools       HOST array of DEVICE pointers to pools of num_pages pages of page_bytes bytes each; 16-byte aligned
 *   num_pools   0 .. COCKTAIL_MAX_POOLS; with 0 nothing can be copied: for callers whose sequences share no partly filled pages
 *               (where one has to be, nothing is done and status[0] is -2)
 *   page_bytes  a multiple of 16
 *   workspace   DEVICE, cocktail_pages_workspace bytes, 16-byte aligned, not initialised; shared between calls as that of
 *               cocktail_fp4_attention
 *
 * One launch, and one for the copies if there are pools.  Errors: EINVAL, EALIGN, ENOSPACE, EHIP.
 */
int cocktail_pages_resize(const cocktail_page_table* pages, const int32_t* delta, void* const* pools, int32_t num_pools,
                          int64_t page_bytes, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Forks: sequence b becomes what sequence source[b] was before the call, sharing its pages (also a partly filled last one, see
 * cocktail_pages_resize).  source[b] == b leaves it as it is, a negative source frees it; a source that is no sequence
 * (>= num_seqs) leaves it as it is too.  A step of a beam search is one call; no page is copied.
 *
 *   source  DEVICE int32 [num_seqs]
 *
 * One launch.  Errors: EINVAL, EALIGN, EHIP.
 */
int cocktail_pages_fork(const cocktail_page_table* pages, const int32_t* source, void* stream);

/*
 * Compaction: with n pages in use, the i-th page in use behind the first n moves to the i-th free page among them, in all pools,
 * and the table and the references follow; afterwards pages 0 .. n-1 are in use.  Arguments as cocktail_pages_resize.
 * Two launches.  Errors: EINVAL, EALIGN, ENOSPACE, EHIP.
 */
int cocktail_pages_compact(const cocktail_page_table* pages, void* const* pools, int32_t num_pools, int64_t page_bytes,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Diagnostic: waits for `stream` and reads status[0] (synchronises and copies).  COCKTAIL_OK, or COCKTAIL_ESTATE if the last
 * cocktail_pages_resize could not be done.  Other errors: EINVAL, EHIP. */
int cocktail_pages_check(const cocktail_page_table* pages, void* stream);

/*
 * A paged cache that holds K and V in microscaled 4-bit floating point (1 bit sign, 2 bits exponent, 1 bit mantissa, and an
 * 8-bit power of two per 32 channels), from the first token on and for every token: 4.25 bits a value.  One pool per layer.
 *
 * Page: num_kv_heads runs, one per head, each of page_size * (D + D/16) bytes:
 *   K codes   token i, channel c: byte i * D/2 + c/2, low half for even channels
 *   V codes   in quads of tokens: token i, byte y = c/2: (i/4) * 2D + (y/4) * 16 + (i%4) * 4 + y%4, low half for even channels
 *   K scales  token i, group g of 32 channels: byte i * D/32 + g
 *   V scales  token i, group g: byte (i/4) * D/8 + g * 4 + i%4
 * (Sixteen tokens of K are what the lanes of a wave hold as one operand of a matrix instruction, 16 bytes of contiguous memory
 * each; a quad of V is a piece of sixteen bytes per eight channels, so that a lane has tokens side by side.  No byte
 * is shared by two tokens.)
 *
 * Quantizer, per token, kv head and group of 32 channels, K and V alike (every step exact in binary32):
 *   e     = clamp(floor(log2(max |x|)) - 2, -23, 13); -23 if all are zero; scale byte = e + 127
 *   code  = sign of x, and the number of the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| * 2^-e (ties to the even number,
 *           6 beyond 6)
 * Value of a code: exact in fp16 and bf16.  Beyond 49152 = 6 * 2^13 values saturate (infinities too); NaN is stored as 0.
 */
typedef struct cocktail_fp4_cache {
  cocktail_page_table pages; /* page_size a multiple of 16 up to 65536, table_stride * page_size <= 2^31 - 256 */
  void* pool;                /* DEVICE num_pages pages of cocktail_fp4_page_bytes, 16-byte aligned    */
  int32_t num_kv_heads;
  int32_t head_dim;          /* 64 or 128                                                             */
} cocktail_fp4_cache;

#define COCKTAIL_FP16 0
#define COCKTAIL_BF16 1

int cocktail_fp4_page_bytes(int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int64_t* bytes);

/*
 * Stores new tokens: row t of k and v, starts[b] <= t < starts[b+1], is quantized into the cache as one of the last
 * n = starts[b+1] - starts[b] tokens of sequence b (token seq_lens[b] - n + t - starts[b]).  Call cocktail_pages_resize first: it
 * makes the room and counts the tokens.  Rows for tokens before the first, or behind what the table row can hold, or on a page that
 * is no page of the pool, are left out.  Nothing else in the pool is written.
 *
 *   k, v      DEVICE, 16-byte aligned; element (t, h, d) at t * stride_t + h * stride_h + d; strides in elements, multiples of 8
 *   dtype     COCKTAIL_FP16 or COCKTAIL_BF16
 *   total     rows; 0 is fine
 *   starts    DEVICE int32 [num_seqs + 1], ascending from 0 to total, or NULL: total / num_seqs rows for every sequence
 *             (total a multiple of num_seqs).  A sequence whose range is not within [0, total] is left out.  (Where starts descend, the
 *             rows of sequences that begin below an earlier start have no defined result.)
 *
 * One launch.  Errors: EINVAL, EUNSUPPORTED (head_dim), EALIGN, EHIP.
 */
int cocktail_fp4_store(const cocktail_fp4_cache* cache, const void* k, const void* v, int32_t dtype, int64_t stride_t,
                       int64_t stride_h, int64_t total, const int32_t* starts, void* stream);

/*
 * Reads tokens back as the values they stand for: the counterpart of cocktail_fp4_store, with the same rows and arguments.  Rows
 * that cocktail_fp4_store leaves out are zeros, but those of a sequence with a bad range are not written.  (With
 * starts = prefix sums of seq_lens: whole contexts, for instance for cocktail_reorder_quantize.)  One launch.
 */
int cocktail_fp4_gather(const cocktail_fp4_cache* cache, void* k, void* v, int32_t dtype, int64_t stride_t, int64_t stride_h,
                        int64_t total, const int32_t* starts, void* stream);

/*
 * Attention of the newest tokens of every sequence over its cached keys, themselves included (causal): with n = starts[b+1] -
 * starts[b] queries and len = seq_lens[b], query i of sequence b attends to tokens 0 .. len - n + i.  One query per sequence is a
 * decode step, some are the verification of drafts, many a prompt or a part of one; a batch may mix them.
 *     out[t,h] = softmax(sm_scale * q[t,h] . K^T) V,   kv head h / (num_q_heads / num_kv_heads)
 * Products and sums in binary32, K and V as stored, softmax weights rounded to fp16: by 2^-11 of themselves, or, where they are below 2^-25 of the
 * largest, by 2^-36 of that at most (in calls with max_new * num_q_heads / num_kv_heads > 64: below 2^-21, by 2^-32).  bf16 queries are used as fp16
 * times a power of two of their own (exact, but for channels below 2^-14 of the largest).
 *
 *   q         DEVICE, 16-byte aligned; element (t, h, d) at t * stride_t + h * stride_h + d, strides multiples of 8
 *   dtype     of q and out
 *   total, starts   as cocktail_fp4_store
 *   max_new   no sequence has more queries (a sequence that has is left out); with starts == NULL it has to be total / num_seqs
 *   max_len   about the length of the longest sequence, for the split of the work only (results do not depend on it but for the order
 *             of sums); <= 0: as many as the table can hold
 *   sm_scale  <= 0 selects 1/sqrt(D)
 *   out       DEVICE [total][num_q_heads][D], 16-byte aligned; zeros for a query without keys
 *   lse       DEVICE fp32 [total][num_q_heads] natural log-sum-exp (-inf without keys), or NULL
 *   workspace DEVICE, at least cocktail_fp4_attention_workspace bytes for the same sizes, 16-byte aligned, not initialised; calls
 *             that share one must not overlap in time, nor be made by two threads at once (a call is several launches)
 *
 * Keys on a page that is no page of the pool, or behind what the table row can hold, are left out.  Calls on the same inputs agree bit for bit.
 * num_q_heads / num_kv_heads from 1 to COCKTAIL_MAX_Q_PER_KV.  Up to four launches.  Errors: EINVAL, EUNSUPPORTED, EALIGN, ENOSPACE, EHIP.
 */
int cocktail_fp4_attention_workspace(const cocktail_fp4_cache* cache, int32_t num_q_heads, int64_t total, int32_t max_new,
                                     int32_t max_len, int32_t uniform, size_t* bytes);
int cocktail_fp4_attention(const cocktail_fp4_cache* cache, int32_t num_q_heads, const void* q, int32_t dtype, int64_t stride_t,
                           int64_t stride_h, int64_t total, const int32_t* starts, int32_t max_new, int32_t max_len,
                           float sm_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* ======================================= A paged cache in 16 bits ======================================= */

/*
 * A paged cache that holds K and V as they are, in fp16 or bf16, on the same page tables: for a prefill whose context is quantized later
 * (cocktail_reorder_quantize_paged reads these pages: stride_t = D, stride_h = page_size * D, stride_page = num_kv_heads * page_size * D), and
 * for layers that stay in 16 bits.  A pool for K and one for V per layer; both are pools of cocktail_pages_resize and
 * cocktail_pages_compact, pages of num_kv_heads * page_size * D * 2 bytes.
 *
 * Page: [num_kv_heads][page_size][D].
 */
typedef struct cocktail_kv16_cache {
  cocktail_page_table pages; /* page_size a multiple of 16 up to 65536, table_stride * page_size <= 2^31 - 256 */
  void* k;                   /* DEVICE num_pages pages, 16-byte aligned                               */
  void* v;                   /* DEVICE num_pages pages, 16-byte aligned                               */
  int32_t num_kv_heads;      /* 1 .. 1024                                                             */
  int32_t head_dim;          /* 64 or 128                                                             */
  int32_t dtype;             /* COCKTAIL_FP16 or COCKTAIL_BF16                                        */
  int32_t reserved;          /* 0                                                                     */
} cocktail_kv16_cache;

/*
 * Rotation of channels by the position: pair i of the first rotary_dim channels of a head, (x, y) = channels (i, i + rotary_dim / 2), or
 * (2 i, 2 i + 1) if interleaved, becomes factor * (x cos a - y sin a, y cos a + x sin a) with a = position * inv_freq[i].  The angle is taken
 * in binary64 and brought into one turn there, so that it is as good at position 2^31 as at 1; the rest is binary32, rounded
 * once to the type of the rows.  The other channels stay as they are.
 */
typedef struct cocktail_rotation {
  const double* inv_freq; /* DEVICE [rotary_dim / 2], 8-byte aligned                                  */
  int32_t rotary_dim;     /* a multiple of 16 up to head_dim                                          */
  int32_t interleaved;    /* 0 or 1                                                                   */
  float factor;           /* finite; 1 for a plain rotation                                           */
  int32_t reserved;       /* 0                                                                        */
} cocktail_rotation;

/*
 * Appends new tokens: row t of k and v, starts[b] <= t < starts[b+1], becomes one of the last n = starts[b+1] - starts[b] tokens of
 * sequence b (token seq_lens[b] - n + t - starts[b]), k rotated on the way; the queries of the same tokens are rotated into q_out.
 * Call cocktail_pages_resize first, as for cocktail_fp4_store: where it found no room nothing is stored (the queries are rotated all
 * the same), and rows for tokens before the first, or behind what the table row can hold, or on a page that is no page of the
 * pool, are left out.  Nothing else in the pools is written.  The pools must not overlap; k, v and q may lie in them in places that the call does not store to.
 *
 *   k, v       DEVICE, 16-byte aligned; element (t, h, d) at t * stride_t + h * stride_h + d; strides in elements, multiples of 8; of the
 *              cache's dtype, as q and q_out are
 *   total, starts   as cocktail_fp4_store
 *   rotation   HOST, or NULL: K is stored as it is, q must be NULL
 *   positions  DEVICE int32 [total]: positions of the rows for the rotation, or NULL: the tokens' numbers in their sequences
 *   q          DEVICE, 16-byte aligned, strides as k's, or NULL
 *   q_out      DEVICE [total][num_q_heads][D], 16-byte aligned; may be q itself where that is laid out the same; must not overlap with
 *              anything else that the call reads or stores to.  Rows of a sequence with a bad range are not written.
 *   num_q_heads  1 .. 65536 with q, else 0
 *
 * One launch.  Errors: EINVAL, EUNSUPPORTED (head_dim, rotary_dim), EALIGN, EHIP.
 */
int cocktail_kv16_append(const cocktail_kv16_cache* cache, const void* k, const void* v, int64_t stride_t, int64_t stride_h,
                         int64_t total, const int32_t* starts, const cocktail_rotation* rotation, const int32_t* positions,
                         const void* q, int32_t num_q_heads, int64_t q_stride_t, int64_t q_stride_h, void* q_out, void* stream);

/*
 * Attention of the newest tokens of every sequence over its cached keys, themselves included (causal): rows, arguments, workspace and
 * what is left out as cocktail_fp4_attention; q and out are of the cache's dtype.  out may be q where that is laid out the same; otherwise
 * out, lse and workspace must not overlap with each other or with anything that the call reads.
 * Products and sums in binary32; softmax weights rounded to the cache's dtype (fp16: as there; bf16: by 2^-8 of themselves), and divided by the
 * sum of the rounded ones (calls with max_new * num_q_heads / num_kv_heads > 64: or of the others).  A value of V that is not finite spoils its channel for all queries of its sequence and kv head in the
 * call, also for those that do not see its token.  Calls on the same inputs agree bit for bit.  Up to four launches.
 * Batches with sequences of up to 64 rows (queries times num_q_heads / num_kv_heads): num_seqs * num_kv_heads * min(64, most rows) below 2^26.
 * Errors: EINVAL, EUNSUPPORTED, EALIGN, ENOSPACE, EHIP.
 */
int cocktail_kv16_attention_workspace(const cocktail_kv16_cache* cache, int32_t num_q_heads, int64_t total, int32_t max_new,
                                      int32_t max_len, int32_t uniform, size_t* bytes);
int cocktail_kv16_attention(const cocktail_kv16_cache* cache, int32_t num_q_heads, const void* q, int64_t stride_t, int64_t stride_h,
                            int64_t total, const int32_t* starts, int32_t max_new, int32_t max_len, float sm_scale, void* out,
                            float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* ============================================ Beam search ============================================ */

/*
 * Selection of a step of beam search: `groups` requests with `beams` hypotheses each, rows r = group * beams + beam of logits.
 *     logp[r, v] = logits[r, v] - log sum_u exp(logits[r, u])
 * Candidate (r, v) has the value scores[r] + logp[r, v]; a hypothesis that has ended (finished[r] != 0) has the one candidate (r, eos) of value
 * scores[r].  The `keep` candidates of a group with the largest values are selected, in descending order, ties by the lowest
 * (row, token); those of a row are in the order of their logits, also where binary64 cannot tell their values apart.  What has no probability is no candidate: logits that are -inf or NaN, rows whose score is -inf or NaN, rows without a
 * finite logit.  An infinite logit counts as the largest finite number.  Where a group has fewer than `keep` candidates the other places are
 * source -1, token -1, score -inf, finished 0.
 * With keep == beams `source` is what cocktail_pages_fork and cocktail_beam_reorder take (places without a candidate free their pages).
 *
 *   logits    DEVICE, aligned to its elements; element (r, v) at r * stride_row + v (stride_row >= vocab, in elements)
 *   dtype     COCKTAIL_FP16, COCKTAIL_BF16 or COCKTAIL_FP32
 *   groups, beams, vocab, keep   groups * beams <= 2^20, beams 1 .. 64, vocab 1 .. 2^24, keep 1 .. 64
 *   scores    DEVICE fp32 [groups * beams]
 *   finished  DEVICE uint8 [groups * beams], or NULL: none
 *   eos       token that ends a hypothesis, or -1: none (then finished must be NULL)
 *   source    DEVICE int32 [groups * keep] out: rows of logits
 *   token     DEVICE int32 [groups * keep] out
 *   score     DEVICE fp32 [groups * keep] out: the candidates' values
 *   finished_out  DEVICE uint8 [groups * keep] out, or NULL: finished[source] or token == eos
 *   workspace DEVICE, cocktail_beam_select_workspace bytes, 16-byte aligned, not initialised; shared between calls as that of
 *             cocktail_fp4_attention
 *
 * Exponentials and sums of up to eight of them in binary32, longer sums and the candidates' values in binary64.  Results and workspace may not overlap
 * with each other or the inputs, but for score over scores and finished_out over finished where keep == beams.
 * Calls on the same inputs agree bit for bit.  Two launches.  Errors: EINVAL, EALIGN, ENOSPACE, EHIP.
 */
#define COCKTAIL_FP32 2
#define COCKTAIL_MAX_KEEP 64
int cocktail_beam_select_workspace(int32_t groups, int32_t beams, int32_t vocab, int32_t keep, size_t* bytes);
int cocktail_beam_select(const void* logits, int32_t dtype, int64_t stride_row, int32_t groups, int32_t beams, int32_t vocab,
                         int32_t keep, const float* scores, const uint8_t* finished, int32_t eos, int32_t* source, int32_t* token,
                         float* score, uint8_t* finished_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Reorders what hypotheses carry: row r of every state becomes what row source[r] was before the call; rows whose source is negative,
 * or no row, stay as they are.  The counterpart of cocktail_pages_fork for tensors (token histories, recurrent states).
 *
 *   source     DEVICE int32 [rows]; no state may be written over it
 *   rows       1 .. COCKTAIL_MAX_SEQS
 *   from, to   HOST arrays of num_states DEVICE pointers to contiguous rows; to[i] == from[i] reorders in place.  No memory may be written
 *              twice in a call, and none that is copied to may be copied from (what is reordered in place may: the copies are made first)
 *   row_bytes  HOST int64 [num_states], bytes of a row of each state; any number up to 2^40 (whole pieces of 16 bytes are fastest, then of 4)
 *   num_states 0 .. COCKTAIL_MAX_STATES
 *
 * Up to two launches (states in place, others).  Errors: EINVAL, EALIGN, EHIP.
 */
#define COCKTAIL_MAX_STATES 64
int cocktail_beam_reorder(const int32_t* source, int32_t rows, const void* const* from, void* const* to, const int64_t* row_bytes,
                          int32_t num_states, void* stream);

/* Message of the last failure on the calling thread ("" if none).  Static storage. */
const char* cocktail_last_error(void);

/* Library version, (major << 16) | minor. */
int cocktail_version(void);

#ifdef __cplusplus
}
#endif
#endif /* COCKTAIL_H */
