/*
 * smha -- masked multi-head attention for AMD MI355X (gfx950), C ABI.
 *
 *   O = softmax(scale * Q K^T  restricted to the unmasked keys of each query) V
 *
 * computed only over the unmasked entries of a static mask.  The library follows the
 * "unified MHA module" of the STOF paper (Sec. 4.2): a mask is analysed once into a
 * per-row column-index format and a two-level block format (block-compressed sparse rows
 * plus a bitmap per partially filled tile, Sec. 4.2.1), an analytical selector
 * (Sec. 4.2.3, Eq. 1) picks a row-wise or a block-wise kernel, and the forward call runs
 * one fused kernel that never touches empty tiles (Sec. 4.2.2, Algorithm 1).
 *
 * Conventions
 *   - A mask entry of 1 means "query i attends key j".  A query with no unmasked key
 *     produces an all-zero output row (the paper does not define this case).
 *   - Self-attention has Sq = Sk = S; a dense mask may also have fewer or more queries than
 *     keys (smha_plan_from_dense_rect: cross-attention, a chunk of queries against cached
 *     keys).  head_dim d is a multiple of 8 up to 256 (the kernels exist for 32, 64, 96, 128, 160 and 256
 *     columns; a narrower head runs on the next of them, its missing columns read as zeros).  Q/K/V are IEEE binary16 or bfloat16.
 *   - All functions return a status code; nothing is printed, thrown or aborted.
 *     On error, output parameters are left untouched.
 *   - "host" / "device" is stated per pointer.  The library never frees or keeps
 *     Q/K/V/O; it owns everything reachable from a plan.
 */
#ifndef SMHA_H
#define SMHA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct smha_plan smha_plan_t; /* opaque; created by smha_plan_from_*, freed by smha_plan_destroy */

typedef enum {
    SMHA_OK = 0,
    SMHA_ERR_INVALID_ARG = 1, /* null pointer, negative size, unknown enum value            */
    SMHA_ERR_UNSUPPORTED = 2, /* head_dim / block size / dtype / alignment not supported    */
    SMHA_ERR_SHAPE = 3,       /* B/H do not match the plan's mask broadcast shape, S < 1    */
    SMHA_ERR_ALLOC = 4,       /* host or device allocation failed                           */
    SMHA_ERR_HIP = 5          /* no usable GPU, or a HIP runtime call failed                */
} smha_status_t;

typedef enum { SMHA_F16 = 0, SMHA_BF16 = 1, SMHA_F32 = 2 /* output only */ } smha_dtype_t;
typedef enum { SMHA_KERNEL_AUTO = 0, SMHA_KERNEL_ROW = 1, SMHA_KERNEL_BLOCK = 2 } smha_kernel_t;
typedef enum {
    SMHA_SELECTOR_CALIBRATED = 0, /* cost model fitted to MI355X measurements (default)       */
    SMHA_SELECTOR_PAPER_EQ1 = 1   /* the paper's formula verbatim (Sec. 4.2.3, Eq. 1)         */
} smha_selector_t;

/* Plan options.  Zero-initialise for defaults. */
typedef struct {
    int block;      /* tile edge of the exported block format: 16, 32 or 64; 0 = 64 (the paper's
                       OuterTile, Sec. 4.2.1)                                                  */
    int force;      /* smha_kernel_t; AUTO lets the selector decide                            */
    int selector;   /* smha_selector_t                                                         */
    int build_both; /* nonzero: keep both formats so either kernel can be forced at run time  */
    int device_id;  /* >= 0: upload index arrays to that GPU at plan time; -1: the current
                       device if there is one, otherwise stay host-only (forward then returns
                       SMHA_ERR_HIP); -2: host-only on purpose                                 */
    int head_dim;   /* hint for the calibrated selector (0 = 64)                               */
    int no_gather;  /* nonzero: the block kernel visits every non-empty 64x64 tile as it is; 0: tiles
                       with few used key columns are repacked into gathered tiles (block kernel
                       work lists only; the exported formats are never affected)               */
    int block_form; /* which form of the block-wise kernel runs where several exist: 0 = the library's choice
                       (at 128 columns form 3, unless nearly all tiles are full and the lists long: form 1;
                       at 160 and 256 columns form 3; at 32, 64 and 96 columns form 1, at 96 form 3
                       where nine tiles in ten are partly filled and a quarter of their 32 x 32 sub-tiles has
                       no keys; at all widths the wave form, one wave per 32 query rows, for calls that it
                       is estimated to run faster),
                       1 = four waves per workgroup, every wave forms scores, probabilities and output of
                       its 32 rows (one to four workgroups per compute unit); 2 = eight waves per workgroup,
                       score waves and value waves, one workgroup per compute unit (64 and 128 columns);
                       3 = eight waves of 16 rows per workgroup, two workgroups per compute unit at 96 to
                       160 columns, one at 256.  Plans with gathered tiles always run form 1, as does bfloat16
                       at 128 columns where form 2 is asked for.  For measurements and tests.             */
} smha_plan_opts_t;

/* Mask description: the atomic patterns of the paper (Sec. 2.1.2, Fig. 1) and their
 * compounds.  Composition:
 *     M = (WINDOW | GLOBAL | STRIDED | BLOCK_RANDOM | BIGBIRD   [all ones if none is set])
 *         & CAUSAL (if set) & PADDING (if set)
 * Random components use a counter-based generator: u = top 53 bits of
 * mix(mix(seed ^ mix(head)) ^ (block_row << 32 | block_col)) / 2^53 with mix = the
 * splitmix64 output function, head = 0 unless per_head. */
enum {
    SMHA_MASK_CAUSAL = 1,        /* keep j <= i                                                */
    SMHA_MASK_WINDOW = 2,        /* keep i - j <= window_left and j - i <= window_right        */
    SMHA_MASK_GLOBAL = 4,        /* keep rows i < n_global and columns j < n_global            */
    SMHA_MASK_STRIDED = 8,       /* keep j % stride == stride_phase                            */
    SMHA_MASK_BLOCK_RANDOM = 16, /* keep block (br, bc) iff u < keep_p, and every br == bc     */
    SMHA_MASK_BIGBIRD = 32,      /* per block row: n_window_blocks columns centred on br,
                                    the first n_global_blocks block rows and columns, and the
                                    n_random_blocks not-yet-kept columns of smallest (hash, bc) */
    SMHA_MASK_PADDING = 64       /* keep only i < valid_len[b] and j < valid_len[b]            */
};

typedef struct {
    uint32_t flags;
    int window_left, window_right;
    int n_global;
    int stride, stride_phase;
    int block; /* block edge of BLOCK_RANDOM / BIGBIRD (any positive size)                    */
    double keep_p;
    int n_window_blocks, n_global_blocks, n_random_blocks;
    uint64_t seed;
    int per_head;             /* random components differ per head: one mask per head          */
    const int32_t *valid_len; /* host, [B]; required with PADDING: one mask per batch entry    */
} smha_mask_desc_t;

typedef struct {
    int S, Bm, Hm;      /* queries per sequence; masks are [Bm][Hm][S][Sk], Bm in {1,B}, Hm in {1,H} */
    int block;          /* tile edge of the exported block format                               */
    int kernel;         /* SMHA_KERNEL_ROW or SMHA_KERNEL_BLOCK: what smha_forward will run     */
    int has_row_format, has_block_kernel_lists, on_device;
    int64_t nnz;        /* unmasked entries, summed over the Bm*Hm masks                         */
    int64_t n_valid, n_full, n_part; /* tiles of edge `block`, summed over masks                 */
    int64_t n_valid16;  /* non-empty 16x16 tiles, summed over masks (input of Eq. 1)             */
    int64_t n_tiles64;  /* non-empty 64x64 tiles the block kernel visits, summed over masks      */
    int64_t n_union;    /* K/V tile loads of the block kernel: union of the tile lists of the two
                           tile rows each 128-row workgroup covers, summed over masks             */
    int64_t n_items, n_split_rows; /* block-kernel work items / 128-row groups split along keys  */
    double eq1_threshold; /* Eq. 1 with valid16 averaged over masks; < 0 means row-wise          */
    double model_row_us, model_block_us; /* calibrated cost model, per (batch, head) pair         */
    int Sk;             /* keys per sequence (= S unless the plan came from smha_plan_from_dense_rect) */
    int64_t n_gathered; /* gathered tiles in the block kernel's lists (each replaces several sparse tiles) */
} smha_plan_info_t;

/* Arrays smha_plan_export can copy out (all host byte order, packed):
 *   ROW_PTR int32[S+1], COL_IDX int32[nnz]  -- per-row format, columns ascending in a row
 *   LOAD/FULL/PART_ROW_PTR int32[nbr+1], LOAD/FULL/PART_COL_IDX int32[...]  (Sec. 4.2.1;
 *     nbr = ceil(S/block); load = full U part, ascending inside a tile row)
 *   BLOCK_FLAGS uint8 per load entry: 1 = full (all block*block entries unmasked), 0 = part
 *   BITMAP uint64[n_part][block], part tiles in PART_COL_IDX order: word r = tile row r,
 *     bit c (LSB = 0) = tile column c; entries past S are 0, so a ragged tile is never full
 *   BITMAP_IT8 uint64[n_part][64] (block == 64 only): the paper's inner-tile layout, word
 *     ic*8+ir = 8x8 inner tile (ir, ic) (column-major over inner tiles), bit 8*r+c = entry (r,c)
 * The block kernel's own work lists (for inspection and tests; UNSUPPORTED if the plan has none):
 *   KERNEL_ITEMS int32[n_items of this mask][8]: {128-row group, first entry, end entry, workspace slot
 *     or -1, first gathered tile, gathered tiles, split group (index among this mask's split groups)
 *     or -1, 0}
 *   KERNEL_ITEMS_FINE: the same groups cut to at most 16 entries per item; smha_forward walks these
 *     instead when the call has too few items to fill the chip (few heads, long lists), so that the
 *     longest list does not set the launch's duration
 *   KERNEL_ENTRIES int32[n][4], all masks: {key tile, code for the group's first 64 rows, code for its
 *     second 64 rows, gathered tile + 1 or 0}; code -2 = nothing, -1 = every entry set, >= 0 = block
 *     of KERNEL_BITMAPS.  An ordinary entry covers keys 64*tile .. 64*tile+63; a gathered one the 64
 *     keys KERNEL_GATHER_KEYS[gathered tile][0..63] (keys >= Sk are padding)
 *   KERNEL_BITMAPS uint64[n][64]: word r = query row r of the 64, bit k = k-th key of the entry
 *   KERNEL_GATHER_KEYS int32[n][64]
 * The lists of the block kernel's wave form (UNSUPPORTED if the plan has none):
 *   WAVE_ITEMS int32[n of this mask][8]: {32-row group, first entry, entries, workspace slot or -1, split
 *     group (index among this mask's) or -1, the first entry's two words, 0}, longest first
 *   WAVE_ENTRIES int32[n][2], all masks: {first key of a 32-key tile, -1 = every entry set, else the block
 *     of KERNEL_BITMAPS that holds the tile: its rows 32 (group mod 2) .., its bits 32 (key / 32 mod 2) ..}
 */
typedef enum {
    SMHA_EXPORT_ROW_PTR = 0,
    SMHA_EXPORT_COL_IDX = 1,
    SMHA_EXPORT_LOAD_ROW_PTR = 2,
    SMHA_EXPORT_LOAD_COL_IDX = 3,
    SMHA_EXPORT_BLOCK_FLAGS = 4,
    SMHA_EXPORT_BITMAP = 5,
    SMHA_EXPORT_FULL_ROW_PTR = 6,
    SMHA_EXPORT_FULL_COL_IDX = 7,
    SMHA_EXPORT_PART_ROW_PTR = 8,
    SMHA_EXPORT_PART_COL_IDX = 9,
    SMHA_EXPORT_BITMAP_IT8 = 10,
    SMHA_EXPORT_KERNEL_ITEMS = 11,
    SMHA_EXPORT_KERNEL_ENTRIES = 12,
    SMHA_EXPORT_KERNEL_BITMAPS = 13,
    SMHA_EXPORT_KERNEL_GATHER_KEYS = 14,
    SMHA_EXPORT_KERNEL_ITEMS_FINE = 15,
    SMHA_EXPORT_WAVE_ITEMS = 16,
    SMHA_EXPORT_WAVE_ENTRIES = 17
} smha_export_t;

/* Mask analysis (Sec. 4.2.1) from a dense boolean mask.
 *   mask            uint8 [Bm][Hm][S][S], nonzero = attend; host pointer if mask_on_device
 *                   is 0, else a device pointer on the current device.  A device mask is
 *                   analysed by GPU kernels on the default stream: tile by tile (16 bytes per
 *                   64x64 tile and the bitmaps of partially filled tiles cross to the host) when
 *                   the plan needs no per-row lists and exports 64-wide tiles, else packed to bit
 *                   rows (1/8 of the bytes cross over) for the host analysis.  Either way the
 *                   plan equals the one built from the same mask in host memory, and the call
 *                   synchronises before returning
 *   opts            may be NULL (defaults)
 *   out             receives the plan
 * Errors: INVALID_ARG (null, Bm/Hm/S < 1), UNSUPPORTED (block), ALLOC, HIP. */
smha_status_t smha_plan_from_dense(const uint8_t *mask, int mask_on_device, int Bm, int Hm, int S,
                                   const smha_plan_opts_t *opts, smha_plan_t **out);

/* The same for a mask with Sq queries and Sk keys per sequence, uint8 [Bm][Hm][Sq][Sk] (the
 * per-row definition of attention does not need Sq = Sk; Sec. 2.1.1).  Row arrays then have Sq + 1
 * entries, tile rows cover queries and tile columns keys; for Eq. 1 the valid-tile ratio is taken
 * over the ceil(Sq/16) * ceil(Sk/16) tiles and n = ceil(Sk/16).  smha_forward takes Q and O with
 * Sq rows and K and V with Sk rows.  smha_plan_from_dense is the case Sq = Sk. */
smha_status_t smha_plan_from_dense_rect(const uint8_t *mask, int mask_on_device, int Bm, int Hm, int Sq, int Sk,
                                        const smha_plan_opts_t *opts, smha_plan_t **out);

/* Mask analysis from a pattern description; B and H fix how many distinct masks exist
 * (Bm = B with PADDING else 1; Hm = H with per_head and a random component, else 1). */
smha_status_t smha_plan_from_desc(const smha_mask_desc_t *desc, int B, int H, int S,
                                  const smha_plan_opts_t *opts, smha_plan_t **out);

smha_status_t smha_plan_info(const smha_plan_t *plan, smha_plan_info_t *out);

/* Copy one index array of mask `mask_index` (= bm*Hm + hm) to host memory.
 * *need receives the size in bytes; if cap < *need nothing is copied and the call still
 * returns SMHA_OK (query-then-copy).  host_dst may be NULL when cap is 0.
 * UNSUPPORTED if the plan does not hold that array (e.g. ROW_PTR of a block-only plan). */
smha_status_t smha_plan_export(const smha_plan_t *plan, int mask_index, smha_export_t which,
                               void *host_dst, size_t cap, size_t *need);

/* Fused masked attention (Sec. 4.2.2, Algorithm 1 for the block kernel; Sec. 4.1 for the
 * row-wise kernel).  Enqueues on `hip_stream` (a hipStream_t, NULL = default stream) and
 * returns without synchronising.
 *   Q               device, [B][H][S][d] of in_dtype, addressed through *_strides
 *   K, V            device, [B][H][Sk][d] of in_dtype (Sk = S for self-attention plans)
 *   O               device, [B][H][S][d] of out_dtype (same as in_dtype, or SMHA_F32)
 *   *_strides       host, {batch, head, seq} strides in elements, d is contiguous;
 *                   NULL = packed.  Pointers must be 16-byte aligned, strides multiples of
 *                   8 elements, the seq stride at least d, and one (batch, head) slice of
 *                   each tensor must span less than 2 GiB (UNSUPPORTED otherwise).
 *   scale           <= 0 selects 1/sqrt(d)
 *   kernel          AUTO = the plan's choice; ROW/BLOCK need that format in the plan
 * What the block kernel needs per call shape (B, H, d) beyond the plan's index arrays -- the work
 * order and the workspaces of split 128-row groups, see smha_plan_prepare -- is made by that
 * function or, if the shape was never prepared, by the first forward that uses it (that one call
 * allocates device memory and copies to it, so it must not be captured into a HIP graph; every later
 * call, and every call with a prepared shape, allocates, frees and synchronises nothing).  Nothing
 * made for a shape is freed or moved before smha_plan_destroy, so captured graphs and queued
 * launches stay valid whatever other shapes are used later.  Forwards on one plan may overlap on
 * different streams: successive calls with one shape take its 4 workspaces in turn, so up to 4 of
 * them may be in flight at once (a fifth would share the first one's workspace: serialise it
 * behind that call).
 * Errors: INVALID_ARG, UNSUPPORTED (d, dtype, alignment, missing format, more than 2^28
 * work items in one call), SHAPE, ALLOC, HIP. */
smha_status_t smha_forward(const smha_plan_t *plan, const void *Q, const void *K, const void *V,
                           void *O, int B, int H, int d, smha_dtype_t in_dtype,
                           smha_dtype_t out_dtype, const int64_t q_strides[3],
                           const int64_t k_strides[3], const int64_t v_strides[3],
                           const int64_t o_strides[3], float scale, smha_kernel_t kernel,
                           void *hip_stream);

/* smha_forward for callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): same arguments, same result, but the partial
 * results of split row groups go to an array inside the library's own image (32 MiB per GPU,
 * held until the process ends) instead of a workspace of the plan, and nothing is ever allocated,
 * freed or synchronised.  The call shape must have been prepared (smha_plan_prepare, or an earlier
 * smha_forward with the same B, H, d; what another d of the same 64, 128 or 256 columns prepared serves
 * too, see smha_plan_prepare): UNSUPPORTED otherwise, and also when the workspace (as there, with D the
 * kernel width that runs) exceeds the 32 MiB.  A small kernel clears the array's arrival counters
 * ahead of the attention kernel, on the same stream.  Every call on a GPU shares that GPU's one
 * array: calls that overlap in time on one GPU (two streams, two plans, two threads) race on it and
 * must be serialised by the caller; calls that follow each other on one stream are fine.  Plans that
 * split nothing, and the row-wise kernel, do not touch the array.
 * Errors: as smha_forward, plus UNSUPPORTED as described. */
smha_status_t smha_forward_static(const smha_plan_t *plan, const void *Q, const void *K, const void *V,
                                  void *O, int B, int H, int d, smha_dtype_t in_dtype,
                                  smha_dtype_t out_dtype, const int64_t q_strides[3],
                                  const int64_t k_strides[3], const int64_t v_strides[3],
                                  const int64_t o_strides[3], float scale, smha_kernel_t kernel,
                                  void *hip_stream);

/* Makes, once, everything smha_forward needs for calls with this batch size, head count and head
 * size on a plan that runs the block-wise kernel (Sec. 4.2.2): the form of the kernel is decided, the
 * work order made (which workgroup takes which work item, see smha_plan_call_order; the wave form has
 * an order of its own, and its lists, SMHA_EXPORT_WAVE_ITEMS, are made by the first shape that takes
 * it), and 4 workspaces that hold the partial results of row groups whose tile lists were split
 * (those are merged inside the same launch by whichever part finishes last): B*H * (split parts per
 * head) * (128 D + 1024) floats each for the 128-row groups of the older forms, (32 D + 128) for the
 * 32-row groups of the wave form, which may split where they do not, and one counter per split group
 * and head (8 for the older forms); D is 64, 128 or 256, the next above d.  Shapes that split
 * nothing get none.
 * Every kernel width (32, 64, 96, 128, 160 and 256 columns: the next above d) has a preparation of its own, which
 * smha_forward makes where there is none.  Only where nothing may be allocated (smha_forward_static, or smha_forward on a
 * stream that is captured) does a shape without one run on that of another d with the same D, at the wider of the two
 * kernel widths and in the form that was prepared: the same result within rounding.
 * Allocates device memory and copies to it (blocking); call it outside stream capture, on the plan's device.  Calling it again for the
 * same shape does nothing; plans that run the row-wise kernel need nothing and return SMHA_OK.
 * Errors: INVALID_ARG, UNSUPPORTED (d, more than 2^28 work items), SHAPE, ALLOC, HIP. */
smha_status_t smha_plan_prepare(const smha_plan_t *plan, int B, int H, int d);

/* A work order of the block kernel's older forms for B x H heads (smha_plan_call_order gives the one that
 * a forward walks when B * H is no multiple of 8) when workgroups_per_xcd workgroups are
 * resident on each of the chip's 8 XCDs (smha_forward uses for the first form 4 per compute unit at
 * 32 and 64 columns, 3 at 96, 2 at 128 and, without gathered tiles, at 160, else 1; for the third 2, at 256 columns 1): the plan's work items (the workgroup tiling of Algorithm 1's outer loop)
 * differ in length, and each head's items go, longest first, to the compute unit with the least
 * work so far and there to the workgroup with the least (the last heads are dealt together).
 * For inspection and tests; runs on the host.
 *   fine       0: the items of SMHA_EXPORT_KERNEL_ITEMS, 1: those of KERNEL_ITEMS_FINE
 *   host_dst   host, int32: 8 list starts (in pairs), 8 list lengths (in pairs), then the
 *              lists: (batch*head, index into that grain's items of all masks, masks in
 *              order) pairs.  XCD x serves the heads with batch*head mod 8 = x; the
 *              workgroup of rank r takes positions r, r + *per_xcd, ... of its XCD's list
 *              until the list ends or a pair with batch*head = -1 (no more work for this
 *              rank) comes up.
 *   cap, need  capacity of host_dst and the size needed, in int32 words (call with cap 0
 *              to learn the size); nothing is written if cap < *need
 *   per_xcd    workgroups per XCD actually used (<= workgroups_per_xcd); may be NULL
 * Errors: INVALID_ARG, SHAPE (B, H against the plan's masks), UNSUPPORTED (no block format). */
smha_status_t smha_plan_work_order(const smha_plan_t *plan, int B, int H, int workgroups_per_xcd,
                                   int fine, int32_t *host_dst, size_t cap, size_t *need,
                                   int *per_xcd);

/* The order that smha_forward's block kernel walks: as smha_plan_work_order, but heads that are left over when
 * B * H is no multiple of 8 are not kept on one XCD each (batch*head mod 8): their items are dealt over all
 * XCDs, each such head over a stretch of them.  The same arguments, table and errors. */
smha_status_t smha_plan_call_order(const smha_plan_t *plan, int B, int H, int workgroups_per_xcd,
                                   int fine, int32_t *host_dst, size_t cap, size_t *need,
                                   int *per_xcd);

/* Which form of the row kernel smha_forward runs for B x H heads of size d: how many query rows
 * share a wave (8, 4, 2 or 1), and how many keys each lane group of a row has in flight.  For
 * inspection and tests; runs on the host.
 * Errors: INVALID_ARG, UNSUPPORTED (d, no row format), SHAPE. */
smha_status_t smha_plan_row_form(const smha_plan_t *plan, int B, int H, int d, int *rows_per_wave,
                                 int *keys_in_flight);

void smha_plan_destroy(smha_plan_t *plan); /* NULL is allowed */

/* ---- Attention within a causal window and a few first keys that stay visible (sinks) ----
 *
 * No plan: which keys a query sees is arithmetic on positions.  H query heads share Hkv key heads, H / Hkv in a
 * row each.  Query i of sequence b stands at position p = offsets[b] + i and exists where 0 <= p < lengths[b]; it
 * sees key j iff j <= p and (p - j < window or j < n_sink).
 *   Q, O            device, [B][H][Sq][d]; K, V: [B][Hkv][Sk][d]; all of `dtype` (F16 or BF16); d a multiple of 8
 *                   up to 128.  *_strides, alignment and the 2 GiB limit as in smha_forward, but batch and head
 *                   strides of tensors that are only read may be zero
 *   lse             device, float [B][H][Sq], packed: log of the sum of the exponentials of the scaled scores, -inf
 *                   where a query sees nothing or does not exist; NULL in smha_sink_forward if it is not wanted
 *   O_rest          device, [B][H][Sq][d] of `dtype`, packed: what the rounding of O left out, for the backward pass, whose dQ and
 *                   dK are less exact without it; NULL if it is not wanted
 *   offsets         device, int32 [B]; NULL: Sk - Sq for every sequence (the queries are its last ones)
 *   lengths         device, int32 [B], keys per sequence, taken as 0 or Sk where outside 0 .. Sk; NULL: Sk
 *   window          keys that a query sees, itself included; 0: all before it
 *   n_sink          first keys that every later query sees
 *   scale           <= 0 selects 1/sqrt(d)
 * Scores, exponentials and sums are 32 bits; the probabilities, relative to about the largest, are rounded to `dtype` for the product with V (as in
 * smha_forward), which adds as much again to O's own rounding.
 * offsets and lengths are read by the kernels: nothing synchronises, and a captured call follows their values.
 * Queries that do not exist give zero rows in O and dQ, keys at and past a sequence's length zero rows in dK
 * and dV; neither's values are read into any result, whatever they are.  Values that are visible to some query have to
 * be finite (a NaN or infinity there may reach other queries of the same 128, and one in Q or dO of a query that exists the gradients of
 * keys that this query does not see).
 * Errors: INVALID_ARG (null, sizes, a negative window or n_sink, too small a workspace), SHAPE (H no multiple of Hkv),
 * UNSUPPORTED (d, dtype, alignment, strides, sizes), HIP.  Enqueues on hip_stream, on the current device. */
smha_status_t smha_sink_forward(const void *Q, const void *K, const void *V, void *O, float *lse, void *O_rest, int B, int H,
                                int Hkv, int Sq, int Sk, int d, smha_dtype_t dtype, const int64_t q_strides[3],
                                const int64_t k_strides[3], const int64_t v_strides[3], const int64_t o_strides[3],
                                const int32_t *offsets, const int32_t *lengths, int window, int n_sink, float scale,
                                void *hip_stream);

/* Bytes of device memory that smha_sink_backward needs for such a call. */
smha_status_t smha_sink_workspace(int B, int H, int Hkv, int Sq, int Sk, int d, int window, int n_sink, size_t *need);

/* Gradients of Q, K and V (of `dtype`, written whole) from O, O_rest (or NULL) and lse of the forward with the same arguments and dO, the
 * gradient of O.  The result does not depend on the order in which workgroups run: the parts of sums that were cut
 * are added in a fixed order.  P and dS = P (dP - delta) are rounded to `dtype` for the products that use them (of
 * at most 8192 queries in all that see few keys, dS to twice its digits).  In binary16 the gradient of O has to be scaled (as such training
 * does) so that dS keeps within that type's range, and P below 2^-14, where windows are very wide, has fewer digits (96 queries on 20000
 * keys: dV 1.64 times its own rounding from 64 bits, on 1024 keys 1.42).  workspace: device, 16-byte aligned, smha_sink_workspace bytes or more;
 * the call's alone until it has run. */
smha_status_t smha_sink_backward(const void *Q, const void *K, const void *V, const void *O, const void *O_rest,
                                 const float *lse, const void *dO, void *dQ, void *dK, void *dV, int B, int H, int Hkv, int Sq, int Sk, int d,
                                 smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3],
                                 const int64_t v_strides[3], const int64_t o_strides[3], const int64_t do_strides[3],
                                 const int64_t dq_strides[3], const int64_t dk_strides[3], const int64_t dv_strides[3],
                                 const int32_t *offsets, const int32_t *lengths, int window, int n_sink, float scale,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- Attention of new tokens on a cache ----
 *
 * The last T tokens of every sequence, whose keys are in the cache already; H query heads share Hkv key heads.
 *   Q, O            device, [B][H][T][d]; K, V: [B][Hkv][Sk][d], of which sequence b uses the first lengths[b] keys (device, int32
 *                   [B], taken as 0 or Sk where outside 0 .. Sk; the new tokens' keys are the last of them).
 *                   Types, head sizes, strides, alignment as in smha_sink_forward
 *   PK, PV          device, [Hkv][P][d], strides {head, key}: keys before those of every sequence, one copy for all; P = 0: none
 *   weights         device, float [B][Hkv][Sk], strides {batch, head} (NULL = packed; rows apart): what attention each of a sequence's own keys
 *                   received, summed over the T tokens and H / Hkv heads, is added; NULL: not wanted
 *   window, n_sink  as in smha_sink_forward, in a sequence's own keys; a window together with a prefix is UNSUPPORTED
 * (A position is a slot of the cache: where keys have moved, as smha_cache_evict moves them, `window` and `n_sink` still count slots, and a recent key
 * that went to a low slot is outside the window.  Without a window the order of keys does not matter.)
 * Token t of sequence b stands at own key lengths[b] - T + t and sees the keys up to it (in its window, or sinks) and all of the
 * prefix.  Below 0 there is no such token: its output row is zero and it adds to no weight.
 * Roundings are those of smha_sink_forward; accounts are sums in 32 bits of unrounded probabilities.
 * lengths are read by the kernels (nothing synchronises; a captured call follows them), which divide the keys of all sequences evenly
 * over the chip whatever the lengths are.  The result does not depend on the order in which workgroups run.  Keys and values before every
 * token's window, past the length and past Sk are never read into a result; those that some token sees have to be finite (a NaN there may reach
 * the sequence's other tokens).
 * workspace: device, 16-byte aligned, smha_cache_workspace bytes or more (0, and then NULL will do, where there are few
 * keys); the call's alone until it has run.  (weigh: nonzero with weights: 4 H T Sk bytes a sequence more.)
 * Errors as for smha_sink_forward. */
smha_status_t smha_cache_workspace(int B, int H, int Hkv, int T, int Sk, int P, int d, int window, int n_sink, int weigh,
                                   size_t *need);
smha_status_t smha_cache_forward(const void *Q, const void *K, const void *V, const void *PK, const void *PV, void *O,
                                 float *weights, const int32_t *lengths, int B, int H, int Hkv, int T, int Sk, int P, int d,
                                 smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3],
                                 const int64_t v_strides[3], const int64_t pk_strides[2], const int64_t pv_strides[2],
                                 const int64_t o_strides[3], const int64_t w_strides[2], int window, int n_sink, float scale,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- Eviction from a cache by accumulated attention ----
 *
 * Every key head of every sequence keeps min(lengths[b], budget) keys (lengths taken as 0 or Sk where outside 0 .. Sk).  Where it has more, keys stay in the order of
 * (recent first: position > highest position - recent; then by weight, falling; then by slot, rising); recent keys and weights of
 * +inf are equals, and so are NaN and -inf.  Keys that stay keep their slots, but those in slots from `budget` on move, in order, to
 * the slots before it that were freed, with their weights and positions.  Slots from the new length on get weight 0 and
 * position -1; their keys and values stay as they are.  (Slots are then no longer in the order of positions: smha_cache_forward with a window would count
 * slots.)
 *   K, V            device, [B][Hkv][Sk][d], any 16-bit type, changed in place; strides as in smha_forward, but a head may be of any size;
 *                   no two heads in one place
 *   weights         device, float [B][Hkv][Sk], positions: int32 [B][Hkv][Sk], lengths: int32 [B]; packed
 *   *_out           what they are then; each may be the input itself, or must not overlap any
 * Not affected by NaN or infinities among the weights beyond what is said above.  No floating-point sums: exact.
 * workspace: device, smha_cache_evict_workspace bytes or more; the call's alone until it has run.
 * Errors: INVALID_ARG (null, sizes, budget < 1, recent < 0, too small a workspace), UNSUPPORTED (d not a multiple of 8 up to 128, alignment,
 * strides, more than 65535 heads in all, Sk above 2^28), HIP. */
smha_status_t smha_cache_evict_workspace(int B, int Hkv, int Sk, int d, int budget, int recent, size_t *need);
smha_status_t smha_cache_evict(void *K, void *V, const float *weights, const int32_t *positions, const int32_t *lengths,
                               float *weights_out, int32_t *positions_out, int32_t *lengths_out, int B, int Hkv, int Sk, int d,
                               int budget, int recent, const int64_t k_strides[3], const int64_t v_strides[3], void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/* ---- A cache held in 4 bits ----
 *
 * A packed row stands for the d columns of one key or value (d a multiple of 8 up to 128), 32 at a time: each group of 32 columns (the last may have
 * 8, 16 or 24) has a step s and a base m, both binary16, and every column a code c of 0 .. 15, which stands for the binary16 nearest
 * (ties to even) to c s + m.  The row is smha_packed_row(d) = 4 ceil(d / 32) + d / 2 bytes: (s, m) of each group, then d / 8 words of 32 bits, little
 * endian, in which columns 0, 2, 4 and 6 of 8 begin at bits 0, 4, 8 and 12, and columns 1, 3, 5 and 7 at bits 16, 20, 24 and 28.  (80 bytes for
 * 128 columns: 5 bits a value.)
 * How rows are packed: values beyond +-65280, infinities among them, are taken as +-65280; m is the largest binary16 that is not above the group's
 * least value (-0 counts as 0), s the smallest with which 15 s + m is not below its largest; c is the number of k in 0 .. 14 for which the value is at
 * least m + (k + 1/2) s, and 0 where s is 0 (15 s + m is finite then: every code of such a group stands for something finite).  All of it exactly, so that equal inputs give equal bytes.  A value is packed within s / 2 and half a last place
 * of binary16.  A group that holds a NaN stands for NaN throughout.
 *
 *   K, V            device, [B][Hkv][Sk][row] bytes: packed rows; *_strides in bytes, {batch, head, key} (NULL = packed), multiples of 4, no row
 *                   over another where they are written; 4-byte aligned; less than 2 GiB between a head's first and last byte
 *   lengths         device, int32 [B]: keys of every sequence, the new tokens' included (taken as 0 or Sk where outside 0 .. Sk)
 *   offsets         device, int32 [B]
 * lengths and offsets are read by the kernels: nothing synchronises, and a captured call follows them.  What lies in slots from a length on is never
 * read into a result.
 * Two tensors that one call writes have no byte in common (they may lie within one another: keys and values side by side), and nothing that is written is read
 * by the same call but where that is said.
 * Errors: INVALID_ARG (null, sizes, written tensors that share memory, or that reach into one another and are laid out differently, too small a workspace), SHAPE (H no multiple of Hkv), UNSUPPORTED (d, dtype, alignment,
 * strides, sizes), HIP.  Enqueue on hip_stream, on the current device.
 * Sizes that are taken: T and Sk below 2^27, B Hkv up to 2^24, B Hkv T up to SMHA_PACKED_MOST_ROWS, heads of new tokens' and outputs' rows, 64 rows more included, below 2 GiB;
 * in attention also B H and B H T up to 2^24, and, r being H / Hkv T rows in tiles of n = 16 (r up to 16), 32 (up to 32), 64 (up to 64) or 128, B Hkv ceil(r / n) + 4096
 * below 2^24 and B Hkv ceil(r / n) (Sk / k + 8) up to 2^30, where k is 32 for n up to 32 and 64 beyond. */
#define SMHA_PACKED_MOST_ROWS (1 << 27)

/* Bytes of a packed row. */
smha_status_t smha_packed_row(int d, int *bytes);

/* Packs new tokens' keys and values into their slots: token t of sequence b into slot offsets[b] + t (offsets NULL: lengths[b] - T + t), where that is in 0 ..
 * lengths[b] - 1; other tokens are left out, other slots as they are.
 *   K_new, V_new    device, [B][Hkv][T][d] of `dtype` (F16 or BF16); strides and alignment as in smha_sink_forward
 *   K_values, V_values  device, [B][Hkv][T][d] of `dtype`, packed as tensors are (no strides): what the tokens' rows stand for, rounded once more for BF16, zero where a
 *                   token is left out; both NULL: not wanted.  May be K_new and V_new themselves where these are packed; otherwise they reach into
 *                   none of the others, nor into each other */
smha_status_t smha_packed_write(const void *K_new, const void *V_new, void *K, void *V, void *K_values, void *V_values,
                                const int32_t *lengths, const int32_t *offsets, int B, int Hkv, int T, int Sk, int d,
                                smha_dtype_t dtype, const int64_t kn_strides[3], const int64_t vn_strides[3],
                                const int64_t k_strides[3], const int64_t v_strides[3], void *hip_stream);

/* What T slots of every sequence from slot offsets[b] (NULL: 0) on stand for; zeros where a slot is not in 0 .. lengths[b] - 1.
 *   K_out, V_out    device, [B][Hkv][T][d] of `out_dtype` (F16 and F32: the values; BF16: rounded to it); strides in elements, rows 16-byte aligned,
 *                   none over another, less than 2 GiB a head */
smha_status_t smha_packed_read(const void *K, const void *V, void *K_out, void *V_out, const int32_t *lengths, const int32_t *offsets,
                               int B, int Hkv, int T, int Sk, int d, smha_dtype_t out_dtype, const int64_t k_strides[3],
                               const int64_t v_strides[3], const int64_t ko_strides[3], const int64_t vo_strides[3],
                               void *hip_stream);

/* smha_cache_forward (without a prefix and accounts) on packed rows: attention of the last T tokens of every sequence, whose rows are in the cache, one
 * or a chunk of a prompt.  Q, O: [B][H][T][d] of `dtype`, scale, window and n_sink as there.
 * Products are formed of Q and the rows' values, both as they are (bfloat16 queries as binary16 times a power of two, by which columns below 2^-31 of a query's largest lose
 * digits); sums and exponentials are 32 bits; the probabilities are rounded to binary16 for the product with V, whatever `dtype` is: 2^-11 of themselves, and
 * 2^-32 of the row's largest below 2^-21 of it.  The result does not depend on the order in which workgroups run.  Keys before every token's window and past every token's place are never
 * read into a result; those that some token sees have to stand for something finite with every code, as rows that smha_packed_write packed from finite values do (a NaN there may reach
 * other tokens of the sequence).
 * workspace: device, 16-byte aligned, smha_packed_workspace bytes or more (0, and then NULL will do, where there are few keys); the call's
 * alone until it has run. */
smha_status_t smha_packed_workspace(int B, int H, int Hkv, int T, int Sk, int d, int window, int n_sink, size_t *need);
smha_status_t smha_packed_forward(const void *Q, const void *K, const void *V, void *O, const int32_t *lengths, int B, int H, int Hkv,
                                  int T, int Sk, int d, smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3],
                                  const int64_t v_strides[3], const int64_t o_strides[3], int window, int n_sink, float scale,
                                  void *workspace, size_t workspace_bytes, void *hip_stream);

const char *smha_status_string(smha_status_t status);

/* Symbol names of kernels, for matching profiler output (name and duration bookkeeping is left to the caller).
 * smha_call_kernel_name: the kernel that smha_forward launches for a call with this batch size, head count, head size
 * and input type ("" for arguments that it refuses), on a preparation of its own (see smha_plan_prepare).  smha_kernel_name knows no call shape: the kernel that runs where
 * the block kernel's wave form does not take its place, which depends on the call (block_form 0 only). */
const char *smha_call_kernel_name(const smha_plan_t *plan, int B, int H, int d, smha_dtype_t in_dtype,
                                  smha_kernel_t kernel);
const char *smha_kernel_name(const smha_plan_t *plan, int d, smha_dtype_t in_dtype,
                             smha_kernel_t kernel);

#ifdef __cplusplus
}
#endif
#endif /* SMHA_H */
