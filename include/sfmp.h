/*
 * sfmp.h - C ABI of the MI355X (gfx950) block-wise mixed-precision GEMM / GEMV library.
 *
 * The operation (paper: Fig. 3(c); Section 3.3 block-wise bit allocation; Section 3.4
 * Eq. 8-9 row/column reordering; Section 3.5 unified mixed-precision kernel; Appendix B
 * Eq. 11 dequantisation form):
 *
 *     Y[m, row_perm[i]] = sum_j  X[m, col_perm[j]] * ( s[j/128, i] * q[i, j] + z[j/128, i] )
 *
 * where q is the integer code matrix of the reordered weight Wt [N, K] (N output features,
 * K input features), every 128 x 128 tile of Wt carries its own bit-width b in {2,3,4}
 * (the "bitmap"), and (s, z) is one fp16 scale / additive zero-point pair per row per
 * group of 128 reordered columns (other group lengths and bf16 storage: sfmp_layout_set_quant).
 *
 * Conventions
 *   - Every function returns SFMP_OK (0) or a negative SFMP_ERR_* code and never throws.
 *   - "host" pointers are ordinary CPU memory, "device" pointers are HIP device memory on
 *     the current device.  All buffers are owned by the caller; the library allocates and
 *     frees no device memory and never synchronises the stream.
 *   - hip_stream is a hipStream_t passed as void* (NULL = the default stream).
 *   - N and K must be positive multiples of 128; M >= 1 is arbitrary.
 *
 * Packed format (what sfmp_pack writes and the kernels read)
 *   Three byte streams S2, S3, S4.  Stream S_b holds all tiles of width b in ascending
 *   (tile row, tile column) order; a tile of width b occupies exactly 2048*b bytes.
 *   A tile is 8 slabs of 256*b bytes; slab sigma holds the tile rows {8i + sigma}.  Inside a
 *   slab each of 64 lanes owns b consecutive little-endian 32-bit words: word w of lane l of
 *   slab sigma is at byte offset sigma*256*b + l*4*b + 4*w of the tile, so one load of 4*b
 *   bytes per lane of a 64-wide wavefront reads 256*b contiguous bytes, and a 16-row slab of
 *   a tile can be fetched on its own.
 *   Element (r, c) of the tile (r = row, c = column inside the tile) belongs to
 *       lane  l     = 16*((c%32)/8) + r/8
 *       slab  sigma = r%8
 *       step  kappa = c/32,  slot v = c%8,  reg = v/2,  half = v%2
 *   and its bits sit inside the lane's b words of that slab at
 *       b=4: word reg,     bits [16*half + 4*kappa, +4)
 *       b=2: word reg%2,   bits [16*half + 8*(reg/2) + 2*kappa, +2)
 *       b=3: every 16-bit half of a word holds five 3-bit fields j=0..4 at bits [3j, 3j+3) and
 *            one spare bit 15; (kappa, reg) -> (word, field):
 *                kappa 0: (0,0) (1,0) (2,0) (0,3)
 *                kappa 1: (0,1) (1,1) (2,1) (0,4)
 *                kappa 2: (0,2) (1,2) (2,2) SPARE
 *                kappa 3: (1,3) (2,3) (1,4) (2,4)
 *            SPARE: bit t of the code is the spare bit (bit 16*half + 15) of word t, t = 0,1,2.
 *   With this placement the two codes of a register (slots 2*reg, 2*reg+1) share one 32-bit
 *   mask and land inside the fp16 mantissa window of the two halves, the four registers of a
 *   k-step share one field position, and the 8 slots of a lane are exactly the 8 k-values that
 *   lane feeds to a 16x16x32 fp16 matrix instruction.
 *
 *   Block-index table (int32 words), replacing any run-time offset computation
 *   (Appendix G, "Comparison with LUT-based GEMM Family", attributes a <=3 % cost to computing block offsets at
 *   run time):
 *       [0,3)                 number of tiles of width 2, 3, 4
 *       [3, 3+nt)             tile_desc[tr*(K/128)+tc] = (slot << 2) | (b-2); slot = index of
 *                             the tile inside stream S_b
 *       3 x (N/128 + 1)       row_ptr_b for b = 2,3,4 (CSR over tile rows)
 *       count2+count3+count4  col_idx_b for b = 2,3,4 (tile column of each tile, stream order)
 */
#ifndef SFMP_H
#define SFMP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SFMP_TILE 128
#define SFMP_GROUP 128        /* default quantisation group length along K */
#define SFMP_SCALE_FP16 0     /* scales and zeros stored as IEEE fp16 */
#define SFMP_SCALE_BF16 1     /* ... as bfloat16 (the storage type of the paper's Table 1) */

#define SFMP_OK 0
#define SFMP_ERR_NULL (-1)        /* a required pointer is NULL */
#define SFMP_ERR_SHAPE (-2)       /* N or K not a positive multiple of 128, or M < 1 */
#define SFMP_ERR_BITWIDTH (-3)    /* a bitmap entry is not 2, 3 or 4 */
#define SFMP_ERR_CODE_RANGE (-4)  /* a code is >= 2^b for its tile */
#define SFMP_ERR_WORKSPACE (-5)   /* workspace missing, misaligned (256 B) or too small */
#define SFMP_ERR_HIP (-6)         /* a HIP call or kernel launch failed */
#define SFMP_ERR_PERM (-7)        /* sfmp_check_perm: not a permutation of 0..n-1 */
#define SFMP_ERR_LAYOUT (-8)      /* layout struct inconsistent with itself */
#define SFMP_ERR_ALIGN (-9)       /* a device pointer is not aligned as required (see sfmp_gemm) */
#define SFMP_ERR_TOO_LARGE (-10)  /* sfmp_gemm_static: the problem needs more scratch than the static buffer holds */

#define SFMP_LUT_TABLE_FP32 0  /* sfmp_lut_gemv: table entries held as fp32 */
#define SFMP_LUT_TABLE_FP16 1  /* ... as fp16, the 2-byte entries of Appendix F (fp32 sum of the 8 activations, rounded once) */

#define SFMP_KV_PAGE 64        /* tokens of a cache page */
#define SFMP_KV_INT8 0         /* cache codes: whole numbers -127..127, stored plus 128 */
#define SFMP_KV_FP8 1          /* ... 8-bit floating point, 4 exponent and 3 mantissa bits, no infinities (OCP E4M3) */
#define SFMP_KV_MAX_BATCH 1024 /* sequences of one sfmp_kv_reserve or sfmp_kv_reorder call */

#define SFMP_TYPE_FP16 0
#define SFMP_TYPE_BF16 1
#define SFMP_TYPE_FP32 2

#define SFMP_STATIC_SCRATCH_BYTES (16 * 1024 * 1024)  /* scratch of sfmp_gemm_static, per GPU */

/* Sizes of a packed matrix.  Filled by sfmp_pack_query / sfmp_pack; passed by the caller,
 * unchanged, to the device entry points. */
typedef struct sfmp_layout {
  int32_t N, K;                    /* rows (output features) and columns (input features) of Wt */
  int32_t tile, group;             /* 128, 128 */
  int32_t count2, count3, count4;  /* tiles of each width */
  int32_t index_words;             /* length of the block-index table in int32 words */
  int64_t bytes_s2, bytes_s3, bytes_s4, bytes_index;
  int32_t scale_format;            /* SFMP_SCALE_FP16 (default) or SFMP_SCALE_BF16 */
  int32_t reserved;                /* 0 */
} sfmp_layout_t;

/* Text for an error code (static storage, never NULL).  For SFMP_ERR_HIP the text of the last
 * HIP error seen by the calling thread is appended. */
const char* sfmp_strerror(int code);

/* Host only.  Sizes of the three streams and of the index table for a bitmap
 * (int8 [N/128, K/128], row-major, host).  Section 4.2, paragraph "Extra Metadata": one int8 per block. */
int sfmp_pack_query(const int8_t* bitmap_host, int32_t N, int32_t K, sfmp_layout_t* out);

/* Host only.  Chooses the quantisation-parameter format of a layout filled by sfmp_pack_query / sfmp_pack
 * (which set group 128, fp16): group = 64, 128, 256 or 512 columns per (scale, zero) pair, K a multiple of it
 * (Appendix G "Effect of n_b": the block width n_b is also the group size); scale_format = SFMP_SCALE_FP16 or
 * SFMP_SCALE_BF16.  The packed streams and the index table do not depend on either.  scales and zeros are then
 * [K/group, N] arrays of 16-bit values in that format.  With group 64 a 128-column tile holds two groups, which share
 * the tile's bit-width (a bit-allocation block narrower than 128 columns is not expressible: the bitmap has one entry
 * per 128 x 128 tile).  SFMP_ERR_LAYOUT for any other value. */
int sfmp_layout_set_quant(sfmp_layout_t* layout, int32_t group, int32_t scale_format);

/* Host only.  Packs codes (uint8 [N, K] row-major, reordered coordinates, host) into the three
 * streams and writes the block-index table; all four outputs are host buffers of the sizes
 * sfmp_pack_query reports (a stream of size 0 may be NULL).  Every code is checked against
 * its tile's width.  The caller uploads the buffers (each to a 16-byte aligned device
 * address).  This is the offline packing step of Section 3.5 / Appendix F ("block-major
 * layout, contiguous within each block"), in the byte format described above. */
int sfmp_pack(const uint8_t* codes_host, const int8_t* bitmap_host, int32_t N, int32_t K,
              uint8_t* s2_host, uint8_t* s3_host, uint8_t* s4_host, int32_t* index_host,
              sfmp_layout_t* out);

/* Device.  Expands the packed streams back to codes_dev (uint8 [N, K] row-major, device) with
 * the same device unpack routines the GEMM kernels use.  Asynchronous on hip_stream.
 * Debug / parity entry point: unpacked codes must equal the packer's input bit for bit. */
int sfmp_unpack(const sfmp_layout_t* layout, const void* s2_dev, const void* s3_dev, const void* s4_dev,
                const int32_t* index_dev, uint8_t* codes_dev, void* hip_stream);

/* Host only.  Bytes of device workspace sfmp_gemm needs for this layout and M
 * (256-byte granularity; never 0). */
int sfmp_gemm_workspace(const sfmp_layout_t* layout, int32_t M, int64_t* bytes);

/* Device.  Zero-fills a workspace (a small fill kernel on hip_stream, safe under graph
 * capture).  Optional: sfmp_gemm writes every workspace byte it later reads (staged or gathered
 * activations, the product before the row un-permute), so an uninitialised workspace is fine.
 * One workspace serves one stream at a time: two calls that overlap on the same workspace
 * race. */
int sfmp_workspace_init(void* workspace_dev, int64_t bytes, void* hip_stream);

/* Device.  The mixed-precision product of Fig. 3(c):
 *   X         fp16 [M, K] row-major, ORIGINAL column order.
 *   col_perm  int32 [K]; the kernel reads X[m, col_perm[j]] for reordered column j
 *             (Section 3.4: the weight's column permutation applied to the activation);
 *             NULL = identity.
 *   layout, s2, s3, s4, index   a matrix packed by sfmp_pack, uploaded unchanged.
 *   scales, zeros  16-bit [K/group, N] (group-major; group and storage type from the layout, fp16 and 128
 *             unless sfmp_layout_set_quant said otherwise): w_hat = s*q + z (Appendix B Eq. 11).
 *   bitmap    int8 [N/128, K/128] (device), the bitmap the matrix was packed with, or NULL.  It is part of the
 *             operation's statement (Section 4.2 "Extra Metadata": one int8 per block) but no kernel reads it: the
 *             block-index table that sfmp_pack derived from it carries every tile's width and position, and is
 *             the authority.  A bitmap that disagrees with the index table is not detected.
 *   row_perm  int32 [N]; output feature i of the reordered product is stored at column
 *             row_perm[i] of Y (undoing P_row of Eq. 9); NULL = leave the rows reordered.
 *   Y         fp16 [M, N] row-major; fully overwritten.  fp32 accumulation, one
 *             round-to-nearest-even conversion at the end.  The order of the fp32 sums is fixed for a given
 *             (N, K, M, group length): the same call on the same inputs gives the same bits, on any stream
 *             (no floating-point atomics anywhere).  Y may lie over X for M >= 5: the activations have then been read
 *             before the first result is stored (which may take another form of the kernel, with its own fixed order, than
 *             the call with separate buffers).  For M <= 4 X and Y must not overlap.
 *   workspace device memory of at least sfmp_gemm_workspace() bytes, 256-byte aligned; contents
 *             on entry are irrelevant, contents on return are unspecified.
 * Alignment (SFMP_ERR_ALIGN otherwise): X, col_perm, row_perm, s2, s3, s4, scales and zeros 16 bytes (the kernels
 * read them with 16-byte vector loads and direct global-to-LDS copies); index 4 bytes; Y 2 bytes for M <= 16 and
 * 16 bytes for M > 16 (whole 16-byte row segments are stored there).
 * Precision for M <= 16 (and the chunks of 16 rows): the codes go through the matrix cores as fp16 denormals, and
 * v_mfma_f32_16x16x32_f16 aligns its 32 products by nominal exponents (2^-14 for a denormal) and keeps 24 bits below the
 * largest: a product whose activation lies 2^4 or more below the largest activation of its 32 columns loses low-order
 * bits, less than |s| 2^(E-14) each (E = exponent of that largest activation) - of the order of 2^-14 of the largest
 * product of those 32 columns, above fp32 rounding and far below the fp16 rounding of the result unless the result is
 * a small difference of large terms.
 * Number range: for M <= 16 scales and zeros are widened to fp32 and never rounded.  For M > 16 on the matrix-core
 * path the dequantised weight s*q + z is formed and rounded ONCE in fp16 (bf16 parameters are converted to fp16 first,
 * which is exact inside fp16's normal range): scales, zeros and weights must lie within fp16's normal range,
 * 2^-14 <= |v| <= 65504 (or be 0), to keep full precision; below it a weight carries an absolute error of up to 2^-25,
 * above it it overflows.
 * M = 1 runs the bandwidth-bound GEMV kernel, 2 <= M <= 16 (and M = 1 with K above about 32k) the
 * same scheme with the activations staged per tile column, 16 < M <= 128 with K >= 4096 on small matrices and
 * batches (N <= 1024: M <= 128; K <= 8192: M <= 32 on any N, M <= 64 up to
 * 1536 tiles of 128 x 128, M <= 96 up to 1024 tiles; longer K: M <= 32 on N <= 4096; K <= 4096: also where the chunks
 * need no workspace and are estimated to be faster) that kernel once more, on
 * chunks of 16 rows side by side in one launch, and everything else the MFMA prefill kernels (with K
 * cut into ranges and fp32 partial products in the workspace when there would be few workgroups;
 * SFMP_ERR_SHAPE there if K > 57344, or, with a row permutation or a split K, N > 81920; the kernels for
 * M <= 16 and for the chunked form return SFMP_ERR_SHAPE if N * K >= 2^33).
 * Asynchronous on hip_stream; re-entrant and thread-safe.  The only state kept between calls is a mutex-guarded
 * record, per device, of the kernels whose LDS limit has been raised.  The permutations are not checked for
 * being bijections (out-of-range entries are the caller's error; use sfmp_check_perm). */
int sfmp_gemm(const void* X_dev, int32_t M, const int32_t* col_perm_dev, const sfmp_layout_t* layout,
              const void* s2_dev, const void* s3_dev, const void* s4_dev, const int32_t* index_dev,
              const void* scales_dev, const void* zeros_dev, const int8_t* bitmap_dev,
              const int32_t* row_perm_dev, void* Y_dev, void* workspace_dev, int64_t workspace_bytes,
              void* hip_stream);

/* Device.  sfmp_gemm for callers that cannot allocate device memory and have no workspace to pass: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  The same arguments and the same result, bit for
 * bit, as sfmp_gemm, without the workspace: the scratch memory (staged or gathered activations, the product before the
 * row un-permute, partial products of a split K) is a 256-byte aligned array of SFMP_STATIC_SCRATCH_BYTES (16 MiB) that
 * is part of the library's device code, one copy per GPU, held from the moment the library is loaded on that GPU until
 * the process ends.  The call allocates and frees nothing (no hipMalloc / hipFree, no allocating library routine); its
 * first call on a device looks the array's address up once (hipGetSymbolAddress) - make that first call outside any
 * graph capture.  SFMP_ERR_TOO_LARGE if sfmp_gemm_workspace(layout, M) exceeds SFMP_STATIC_SCRATCH_BYTES (for example
 * M = 2048 on K = 4096; every M <= 16 fits for K up to 1 Mi); other errors as sfmp_gemm.  Nothing in the scratch
 * has to start at zero: every call writes what it later reads, whatever the previous call left.  All calls on one
 * GPU share that GPU's array: calls that overlap in time on one GPU (two streams, two threads) race; order them. */
int sfmp_gemm_static(const void* X_dev, int32_t M, const int32_t* col_perm_dev, const sfmp_layout_t* layout,
                     const void* s2_dev, const void* s3_dev, const void* s4_dev, const int32_t* index_dev,
                     const void* scales_dev, const void* zeros_dev, const int8_t* bitmap_dev,
                     const int32_t* row_perm_dev, void* Y_dev, void* hip_stream);

/* One problem of a batched launch: the arguments of sfmp_gemm without M and workspace. */
typedef struct sfmp_gemv_problem {
  const void* X_dev;             /* fp16 [M, K] */
  const int32_t* col_perm_dev;   /* int32 [K] or NULL */
  const sfmp_layout_t* layout;   /* host pointer; read during the call only */
  const void* s2_dev;
  const void* s3_dev;
  const void* s4_dev;
  const int32_t* index_dev;
  const void* scales_dev;
  const void* zeros_dev;
  const int8_t* bitmap_dev;
  const int32_t* row_perm_dev;   /* int32 [N] or NULL */
  void* Y_dev;                   /* fp16 [M, N] */
} sfmp_gemv_problem_t;

/* Device.  Up to 8 independent M = 1 products (each exactly what sfmp_gemm computes, each with its
 * own weights, permutations, X and Y) in ONE kernel launch: the launch and first-touch latency that
 * bounds small decode layers is paid once for, say, the q, k and v projections of a decoder layer
 * (Section 4 measures decode at batch 1, where every projection is a GEMV).  problems_host is a host
 * array read during the call.  Needs no workspace.  SFMP_ERR_SHAPE if a problem cannot use the
 * GEMV kernel (K above about 32k) - call sfmp_gemm per problem then. */
int sfmp_gemv_batched(const sfmp_gemv_problem_t* problems_host, int32_t count, void* hip_stream);

/* The same for a small batch: up to 8 independent products with a common M, 1 <= M <= 16 (each exactly what
 * sfmp_gemm computes; X_dev of a problem is fp16 [M, K], Y_dev fp16 [M, N]; for M >= 5 a Y_dev may lie over any X_dev), in
 * one launch of the GEMM kernel plus, for M >= 2 where the kernel does not gather its activations itself, one launch of
 * the activation staging kernel.  Problems that pass the same X_dev, col_perm_dev and K
 * (q, k and v; gate and up) share one staged copy of the activations.  M = 1 is sfmp_gemv_batched.
 * One launch runs one form of the kernel, chosen for the whole batch (by its largest K and its largest share of
 * slabs per workgroup), which may not be the form a single sfmp_gemm call takes for one of its problems: the operation
 * is the same, the order of the fp32 sums and hence the last bit of an output may differ from the single call.  The
 * same batch on the same inputs gives the same bits every time.
 * sfmp_gemm_batched_workspace (host only) gives the workspace size for these problems and this M (never 0);
 * the workspace is device memory, 256-byte aligned, contents irrelevant on entry and unspecified on return.
 * SFMP_ERR_SHAPE if M is outside 1..16, if a problem would put more than 16 slabs on a workgroup (N above about
 * 65536 times its share of the grid), or if some but not all problems have group length 64 (one launch runs one of
 * the two classes; sfmp_gemv_batched likewise) - call sfmp_gemm per problem then. */
int sfmp_gemm_batched_workspace(const sfmp_gemv_problem_t* problems_host, int32_t count, int32_t M, int64_t* bytes);
int sfmp_gemm_batched(const sfmp_gemv_problem_t* problems_host, int32_t count, int32_t M, void* workspace_dev,
                      int64_t workspace_bytes, void* hip_stream);

/* Host only.  SFMP_OK if perm_host[0..n) is a permutation of 0..n-1, else SFMP_ERR_PERM. */
int sfmp_check_perm(const int32_t* perm_host, int32_t n);

/* Host only.  Folds the row permutation of one matrix into the column permutation of the next, so that the
 * first product can stay in reordered row order (row_perm_dev = NULL: no un-permute pass) and the second
 * gathers from it directly (Section 3.4: the reordering is applied to activations and undone on outputs; the
 * reorder-overhead measurement of Section 4.2 counts exactly these two reorder operations per layer):
 *   folded[j] = inverse(row_perm_prev)[col_perm_next[j]],   j in [0, n)
 * so that  Xt[:, folded[j]] = X[:, col_perm_next[j]]  whenever  Xt[:, i] = X[:, row_perm_prev[i]],  which holds
 * for Xt = f(Yt), X = f(Y) with any element-wise f between the two matrices (a per-feature weight, as in a norm,
 * has to be reordered by the caller the same way).  col_perm_next_host = NULL stands for the identity.  n is
 * the first matrix' N and the second one's K.  SFMP_ERR_PERM if either input is not a permutation.
 * folded_host may not alias the inputs. */
int sfmp_fold_perms(const int32_t* row_perm_prev_host, const int32_t* col_perm_next_host, int32_t n,
                    int32_t* folded_host);

/* ---- One-bit lookup-table GEMV on a bit-plane format (the paper's own kernel scheme) ----------------------
 * Section 3.5 and Appendix F describe the unified kernel as a one-bit lookup-table GEMM: every block is
 * decomposed into one-bit matrices (Appendix B, Eq. 10), put into +-1 form (s^ = s/2, W^_i = 2 W_i - 1,
 * z^ = z + (2^b - 1) s / 2), packed 8 input features to a byte, and multiplied through tables of the signed
 * sums of 8 activations held in on-chip memory, of which half is stored (mirror storage).  The three calls
 * below are that scheme for M = 1, as a measured alternative to sfmp_gemm (which contracts on the matrix cores):
 * the same operation Y = X[col_perm] . (s q + z)^T with the same bitmap, scale / zero arrays (fp16, group
 * length 128 only) and permutations, on its own weight format.
 *
 * Bit-plane format B1: tiles of 128 x 128 codes in row-major order of (tile row, tile column); a tile of width b
 * holds b planes, lowest bit first; a plane is 128 rows x 16 bytes (2048 bytes); bit t of byte (r, g) is bit i of
 * the code at row 128 tr + r, column 128 tc + 8 g + t.  tile_off[t], t = tr * (K/128) + tc, is the start of tile
 * t in planes (units of 2048 bytes); tile_off[ntiles] is the total, so a tile's width is tile_off[t+1] - tile_off[t].
 *
 * sfmp_lut_pack_query: sizes of the two arrays for a bitmap [N/128, K/128] (host).  SFMP_ERR_SHAPE,
 * SFMP_ERR_BITWIDTH as for sfmp_pack_query.
 * sfmp_lut_pack: codes [N, K] uint8 (host, row-major, reordered coordinates) -> planes_host (plane_bytes bytes),
 * tile_off_host (table_words uint32), both caller-allocated; SFMP_ERR_CODE_RANGE if a code does not fit its tile.
 * sfmp_lut_gemv_workspace / sfmp_lut_gemv: device pointers throughout; X fp16 [K], col_perm int32 [K] or NULL,
 * planes and tile_off as packed (uploaded unchanged), scales / zeros fp16 [K/128, N], row_perm int32 [N] or NULL,
 * Y fp16 [N] fully overwritten; workspace of at least the queried bytes, 256-byte aligned, contents irrelevant
 * on entry and unspecified on return (fp32 partial sums of the K ranges).  table_format: SFMP_LUT_TABLE_FP32, or
 * SFMP_LUT_TABLE_FP16 for the 2-byte table entries of Appendix F (each entry = the fp32 signed sum of its 8
 * activations rounded once to fp16: a relative error of up to 2^-11 per looked-up value; SFMP_ERR_LAYOUT for any other
 * value).  Accumulation in fp32 either way, one round-to-nearest-even conversion at the end; results repeat bit for
 * bit.  Asynchronous on hip_stream; two launches; no global state.  Errors as for sfmp_gemm. */
int sfmp_lut_pack_query(const int8_t* bitmap_host, int32_t N, int32_t K, int64_t* plane_bytes, int64_t* table_words);
int sfmp_lut_pack(const uint8_t* codes_host, const int8_t* bitmap_host, int32_t N, int32_t K, uint8_t* planes_host,
                  uint32_t* tile_off_host);
int sfmp_lut_gemv_workspace(int32_t N, int32_t K, int64_t* bytes);
int sfmp_lut_gemv(const void* X_dev, const int32_t* col_perm_dev, int32_t N, int32_t K, const void* planes_dev,
                  const uint32_t* tile_off_dev, const void* scales_dev, const void* zeros_dev,
                  const int32_t* row_perm_dev, void* Y_dev, int32_t table_format, void* workspace_dev,
                  int64_t workspace_bytes, void* hip_stream);

/* ---- 8-bit paged key/value cache, its attention, its pages --------------------------------------------------------
 * What a decoder needs between its q|k|v projections and its o projection.  Keys and values of all sequences of a GPU
 * live in one pool of pages of SFMP_KV_PAGE = 64 tokens, in 8 bits, with one fp32 scale for each page, head and of K and
 * V; a table gives the pages of every sequence.
 *
 * Pool (device, owned by the caller):
 *   codes   uint8 [layers][pages][kv_heads][2][64 * head_dim].  The first of the two blocks holds the keys as
 *           [token][dim], the second the values TRANSPOSED, as [dim][token]: read 16 bytes per lane, both are operands of
 *           the matrix instructions as they lie, without a transposition.
 *   scales  fp32 [layers][pages][kv_heads][2]
 *   An element is code * scale.  SFMP_KV_INT8: code = byte - 128, scale = m / 127 where m is the largest magnitude of the
 *   block (one page, head, K or V).  SFMP_KV_FP8: scale = 2^e with the smallest e such that m <= 448 * 2^e.  Rounding to
 *   nearest even.  A block whose largest magnitude is below 2^-100 is held as zeros with scale 0.  A block that is given
 *   an infinity or a NaN gets the scale NaN: every element of it reads as NaN until its page is given to other tokens.
 * Tables (device, owned by the caller):
 *   page_table int32 [sequences][table_pages]; lengths int32 [sequences], tokens of each; refs int32 [pages], sequences
 *   that hold a page (0 = free).  Sequence i holds exactly the first ceil(lengths[i] / 64) pages of its row.  An empty
 *   pool has lengths and refs of 0; the page table need not be initialised.
 * The order of a step: sfmp_kv_reserve (once for all layers: room for the new tokens, lengths grow), then for each layer
 * sfmp_kv_append and sfmp_kv_attention on the new rows, which are THE LAST rows of their sequences.
 * The kernels bound every index that they read from tables: an entry outside its range is read as page 0 or as an empty
 * sequence, never out of bounds; what they then compute is unspecified.
 * All calls are asynchronous on hip_stream, allocate nothing and keep nothing. */
typedef struct sfmp_kv_layout {
  int32_t pages, kv_heads;
  int32_t head_dim;                /* 64, 128 or 256 */
  int32_t format;                  /* SFMP_KV_INT8 or SFMP_KV_FP8 */
  int32_t layers;                  /* layers that share the page table */
  int32_t reserved;                /* 0 */
  int64_t page_bytes;              /* codes of one page of one layer */
  int64_t codes_bytes, scales_bytes;
} sfmp_kv_layout_t;

typedef struct sfmp_kv_tables {
  int32_t* page_table_dev;
  int32_t* lengths_dev;
  int32_t* refs_dev;
  int32_t sequences, table_pages;
} sfmp_kv_tables_t;

/* Rows of a call: batch entry b is sequence slots[b] (slots NULL: sequence b) and owns rows row_start[b] ..
 * row_start[b+1]-1 of the row-major arguments (row_start NULL: row b).  Both are device arrays. */
typedef struct sfmp_kv_batch {
  const int32_t* slots_dev;
  const int32_t* row_start_dev;    /* [batch + 1], ascending from 0 */
  int32_t batch;
  int32_t rows;                    /* rows of the arguments, row_start[batch] */
  int32_t max_rows;                /* at least the most rows of one entry; 1 if row_start is NULL */
  int32_t reserved;                /* 0 */
} sfmp_kv_batch_t;

/* Host only.  Fills a layout; SFMP_ERR_SHAPE (pages, kv_heads, layers < 1, kv_heads > 1024, head_dim not 64, 128 or
 * 256), SFMP_ERR_LAYOUT (format). */
int sfmp_kv_query(int32_t pages, int32_t kv_heads, int32_t head_dim, int32_t format, int32_t layers,
                  sfmp_kv_layout_t* out);

/* Device.  Quantises keys and values of new tokens into layer `layer`.  K, V: 16-bit (dtype SFMP_TYPE_FP16 or
 * SFMP_TYPE_BF16), row r at K + r * k_stride elements, [kv_heads][head_dim] inside a row; 16-byte aligned, strides
 * multiples of 8 (a slice of a fused q|k|v result can be passed as it is).  The n rows of an entry are the last n tokens
 * of its sequence (rows that would lie before the first token are left out), and the pages that they go to have to be held by that sequence alone
 * (sfmp_kv_reserve sees to it).  Where a page already holds earlier tokens of the sequence, its scale grows if the new
 * ones need it, and the earlier codes are requantised: code * old / new scale, rounded to nearest even (exact for SFMP_KV_FP8 but for
 * subnormal results).  The scale of a page whose first token is among the new rows is made from the new rows alone; its
 * slots past the last token are zeroed. */
int sfmp_kv_append(const sfmp_kv_layout_t* layout, int32_t layer, void* codes_dev, float* scales_dev,
                   const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const void* K_dev, const void* V_dev,
                   int32_t dtype, int64_t k_stride, int64_t v_stride, void* hip_stream);

/* Device.  Reads cached tokens back: rows of entry b are the tokens first_dev[b], first_dev[b] + 1, ... of its sequence.
 * K, V: [rows][kv_heads][head_dim], row strides in elements, dtype SFMP_TYPE_FP16, _BF16 or _FP32; code * scale rounded once.  Tokens past
 * the end of a sequence read as 0. */
int sfmp_kv_gather(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev,
                   const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const int32_t* first_dev, void* K_dev,
                   void* V_dev, int32_t dtype, int64_t k_stride, int64_t v_stride, void* hip_stream);

/* Device.  Attention of new rows over their sequences' cached tokens (theirs among them):
 *   row i of the n rows of an entry of length t stands at position p = t - n + i and sees the tokens j <= p, with
 *   window > 0 those with j > p - window;
 *   O[row, head] = sum_j w_j V_j / sum_j w_j,  w_j = exp(scale * <Q[row, head], K_j>),  K and V of head / (q_heads/kv_heads).
 * Q: 16-bit (dtype), row r at Q + r * q_stride, [q_heads][head_dim] inside a row, q_heads a multiple of kv_heads; O
 * likewise with o_stride; both 16-byte aligned, strides multiples of 8.  lse: NULL, or fp32 [rows][q_heads], the natural
 * logarithm of the sum of w.  A row that sees no token (p < 0, an empty sequence) gets O = 0, lse = -infinity.  Scores,
 * softmax statistics and sums are held in fp32; products are taken on the matrix cores from exact fp16 values of the
 * codes and of Q (bf16: each row scaled by a power of two); the softmax weights are rounded to fp16 before the product
 * with V, relative to the largest of their row in the page (2^-11 of itself, for weights under 2^-28 of that largest one 2^-39 of
 * it), which adds to a result less error than its own rounding to fp16.  max_tokens: at least the longest
 * sequence of the batch; tokens past it are not read.  The same call on the same inputs gives the same bits; a sequence's
 * result may differ in its last bits with the batch it is in (the work is cut by the whole batch).
 * SFMP_ERR_SHAPE (beside the bounds above: table_pages > 2^20, rows > 2^30): q_heads (no multiple of kv_heads, or above 65536), strides,
 * batch > 65535, max_tokens < 1 or above 2^26, window < 0, scale not finite or not positive,
 * max_rows * q_heads / kv_heads > 2^30, or batch * kv_heads * ceil(max_tokens / 64) * ceil(max_rows * q_heads / kv_heads / 16) >= 2^31.  SFMP_ERR_WORKSPACE as for sfmp_gemm; the
 * workspace's contents are irrelevant on entry.  Weights stand relative to a score that the largest exceeds by less than a factor of 2^16 while they are
 * added up: |V| times the tokens seen has to stay below 2^111.  sfmp_kv_attention_workspace: bytes that are enough for every call with this layout and
 * q_heads, and with no more batch entries, rows, max_rows and max_tokens than these, with any window. */
int sfmp_kv_attention_workspace(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t q_heads,
                                int32_t max_rows, int32_t max_tokens, int64_t* bytes);
int sfmp_kv_attention(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev,
                      const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const void* Q_dev, int32_t q_heads,
                      int32_t dtype, int64_t q_stride, int32_t max_tokens, int32_t window, float scale, void* O_dev,
                      int64_t o_stride, float* lse_dev, void* workspace_dev, int64_t workspace_bytes, void* hip_stream);

/* Device.  The same with first tokens that stay visible behind the window: a row at position p sees the tokens j <= p with
 * j > p - window or j < sinks (window 0: all tokens j <= p, whatever `sinks`).  The pages that lie between are not read, so that
 * a call takes the time of its window and first pages, however long the sequence is.  They stay held: no call gives back pages from the middle of a
 * sequence, so that it takes the memory of all its tokens and ends at 64 * table_pages of them; a stream that goes on is started again, its first
 * and last tokens appended to an empty sequence.  Positions count from the sequence's first token; keys keep the rotation that they were appended
 * with.  Everything else, errors and workspace (sfmp_kv_attention_workspace) too, as sfmp_kv_attention; SFMP_ERR_SHAPE if sinks < 0. */
int sfmp_kv_attention_sinks(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev,
                            const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const void* Q_dev, int32_t q_heads,
                            int32_t dtype, int64_t q_stride, int32_t max_tokens, int32_t window, int32_t sinks, float scale,
                            void* O_dev, int64_t o_stride, float* lse_dev, void* workspace_dev, int64_t workspace_bytes,
                            void* hip_stream);

/* Device.  Attention of a batch whose sequences share their first pages, group by group (samples or beams of a prompt, questions about a
 * document, requests behind one instruction: what sfmp_kv_fork makes): the shared pages are read once for all rows of a group instead of once
 * for each sequence.
 *
 * Group g is the batch entries group_start[g] .. group_start[g+1]-1 (int32 [groups + 1], ascending; entries outside of all groups attend for
 * themselves).  sfmp_kv_share, called once for all layers when the step's tokens have been reserved, finds the pages that the sequences of each
 * group hold in common before they differ - all of its sequences: one that is empty, shorter than the others or of another prompt (a beam that
 * sfmp_kv_reorder has left empty) limits what its whole group shares, and is better left outside of it - and divides the work; sfmp_kv_attention_shared then computes what sfmp_kv_attention_sinks does
 * (window 0: sfmp_kv_attention), with the same O, lse, errors and numerics but for the order of its sums.  The same call on the same
 * inputs gives the same bits.
 *   prefix_dev: NULL, or int32 [groups], the tokens of these pages (a multiple of 64; of a group of one sequence all its full pages; 0 for an
 *   empty group).
 *   plan_dev: written by sfmp_kv_share, read by sfmp_kv_attention_shared; 256-byte aligned.  It holds for calls with the same batch, groups, q_heads,
 *   max_tokens, window, sinks and pool layout until lengths, tables, slots, row or group starts change.  A plan that was made
 *   with other numbers than the call's is not used: O and lse stay as they were.  One with the numbers of the call but of other contents
 *   gives unspecified results.
 * Where there is nothing to gain (nearly as many groups as sequences, more than 64 rows of a sequence and key head, short contexts) or more to plan than 32 bits
 * hold (about 2^29 pages times key heads and tiles of rows), the call runs as
 * sfmp_kv_attention_sinks, and sfmp_kv_share only finds what prefix_dev asks for.
 * Errors as sfmp_kv_attention_sinks; SFMP_ERR_SHAPE for groups < 0 or above 65535, SFMP_ERR_WORKSPACE for a plan that is missing, not aligned or too
 * small too.  sfmp_kv_share_plan, sfmp_kv_attention_shared_workspace: bytes of plan and workspace that are enough for every call with this
 * layout and q_heads, and with no more batch entries, rows, groups, max_rows and max_tokens than these. */
int sfmp_kv_share_plan(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t groups, int32_t q_heads, int32_t max_rows,
                       int32_t max_tokens, int64_t* bytes);
int sfmp_kv_share(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch,
                  const int32_t* group_start_dev, int32_t groups, int32_t q_heads, int32_t max_tokens, int32_t window,
                  int32_t sinks, int32_t* prefix_dev, void* plan_dev, int64_t plan_bytes, void* hip_stream);
int sfmp_kv_attention_shared_workspace(const sfmp_kv_layout_t* layout, int32_t batch, int32_t rows, int32_t groups,
                                       int32_t q_heads, int32_t max_rows, int32_t max_tokens, int64_t* bytes);
int sfmp_kv_attention_shared(const sfmp_kv_layout_t* layout, int32_t layer, const void* codes_dev, const float* scales_dev,
                             const sfmp_kv_tables_t* tables, const sfmp_kv_batch_t* batch, const int32_t* group_start_dev,
                             int32_t groups, const void* Q_dev, int32_t q_heads, int32_t dtype, int64_t q_stride,
                             int32_t max_tokens, int32_t window, int32_t sinks, float scale, void* O_dev, int64_t o_stride,
                             float* lse_dev, const void* plan_dev, int64_t plan_bytes, void* workspace_dev,
                             int64_t workspace_bytes, void* hip_stream);

/* Device.  Page management without the host: no call reads anything back, so a decode loop with all of them can be
 * captured in a graph.  n sequences per call, each at most once; the arrays are int32 [n] on the device.
 *
 * sfmp_kv_reserve: makes room for counts[i] more tokens (counts NULL: one) of sequence slots[i] and adds them to its
 * length.  In the order of i, each sequence gets first a copy of its last page in all layers, if that page is partly
 * filled and still held by another sequence too (copy on write: the last of its holders keeps it), then the pages that
 * the new tokens need; new pages are the free ones of lowest number.  status_dev[0] = 0, or, with nothing changed at
 * all, the number of pages that were missing, or -1 if a slot is out of range, a count negative or a row of the page
 * table too short.  n <= SFMP_KV_MAX_BATCH.
 * sfmp_kv_fork: children[i] becomes a copy of parents[i] that holds the same pages (several may share a parent).  A
 * child must be empty (length 0) and no sequence may be both a parent and a child.
 * sfmp_kv_reorder: sequence slots[i] becomes what sequence slots[parents[i]] was before the call: it holds the same pages (several may have one
 * parent; a sequence that is nobody's parent is gone, and the pages that it alone held are free).  parents[i] outside 0 .. n-1: it becomes
 * empty.  What a beam search does with its sequences after sfmp_beam_select.  n <= SFMP_KV_MAX_BATCH; more sequences (sfmp_beam_select takes 65535
 * rows) go in several calls of whole requests, each with its parents less the number of its first row.
 * sfmp_kv_free: sequence slots[i] keeps its first keep[i] tokens (keep NULL: none) and gives back the other pages.
 * sfmp_kv_compact: moves the live pages with numbers >= n_live, n_live being the number of live pages, in ascending order into the free pages
 * below it, in all layers, and renumbers page table and refs: afterwards the pages n_live .. pages-1 are free.
 * status_dev[0] = n_live.
 * sfmp_kv_pages_workspace: bytes of workspace for sfmp_kv_reserve and sfmp_kv_compact (256-byte aligned, contents
 * irrelevant on entry). */
int sfmp_kv_pages_workspace(const sfmp_kv_layout_t* layout, int64_t* bytes);
int sfmp_kv_reserve(const sfmp_kv_layout_t* layout, void* codes_dev, float* scales_dev, const sfmp_kv_tables_t* tables,
                    const int32_t* slots_dev, const int32_t* counts_dev, int32_t n, int32_t* status_dev,
                    void* workspace_dev, int64_t workspace_bytes, void* hip_stream);
int sfmp_kv_fork(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* parents_dev,
                 const int32_t* children_dev, int32_t n, void* hip_stream);
int sfmp_kv_reorder(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* slots_dev,
                    const int32_t* parents_dev, int32_t n, void* hip_stream);
int sfmp_kv_free(const sfmp_kv_layout_t* layout, const sfmp_kv_tables_t* tables, const int32_t* slots_dev,
                 const int32_t* keep_dev, int32_t n, void* hip_stream);
int sfmp_kv_compact(const sfmp_kv_layout_t* layout, void* codes_dev, float* scales_dev, const sfmp_kv_tables_t* tables,
                    int32_t* status_dev, void* workspace_dev, int64_t workspace_bytes, void* hip_stream);

/* ---- Choice of the next token --------------------------------------------------------------------------------------
 * Device.  One token for every row of logits (dtype SFMP_TYPE_FP16, _BF16 or _FP32; row r at logits + r * stride
 * elements, vocab of them), from the caller's random number uniform[r] in [0, 1).  With m the row's largest logit and T
 * its temperature, token i weighs w_i = exp((l_i - m) / T), held as a whole number of 2^-31 (a token below 2^-32 of the
 * most probable one is never chosen).  Tokens are ordered by falling logit, equal ones by rising number, and kept as long as they are among
 *   the first top_k (top_k <= 0: all), of these
 *   the shortest prefix that holds at least top_p of their weight (top_p >= 1: all), and
 *   those with (l_i - m) / T >= ln min_p (min_p <= 0: all; the most probable token always stays).
 * The token is the first of the order whose running sum of weights exceeds uniform * (sum of the kept ones).  T <= 0
 * takes the first token of the order.  NaN logits count as -infinity; a row without a logit above -infinity gives -1
 * and the log-probability -infinity.  Sums of weights are whole numbers: the result does not depend on how the row was cut.
 * temperature, top_k, top_p, min_p: fp32 / int32 / fp32 / fp32 [rows], each may be NULL (1, all, all, all).  tokens: int32
 * [rows].  logprobs: NULL, or fp32 [rows], (l_token - m) / T less ln of the sum of all w of the
 * row.  With w in whole units, and tokens below 2^-32 of the most probable one left out, that sum is off by at most vocab * 2^-32, and so is
 * the log-probability: 3e-5 for 131072 tokens, which can be much of the value where one token has nearly all the weight.  With T <= 0 the
 * tokens that share the largest logit weigh 1 each and the others nothing: 0, or where n tokens share it -ln n (the first is chosen all the same).
 * SFMP_ERR_SHAPE: rows < 0 or above 65535, vocab < 1 or above 2^24, stride < vocab.  Alignment: logits to their element size.
 * sfmp_sample_workspace: bytes that are enough for every call of no more rows and no larger vocabulary. */
int sfmp_sample_workspace(int32_t rows, int32_t vocab, int64_t* bytes);
int sfmp_sample(const void* logits_dev, int32_t dtype, int32_t rows, int32_t vocab, int64_t stride,
                const float* temperature_dev, const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev,
                const float* uniform_dev, int32_t* tokens_dev, float* logprobs_dev, void* workspace_dev,
                int64_t workspace_bytes, void* hip_stream);

/* Device.  One step of a beam search.  Request r has the rows r * beams .. r * beams + beams - 1 of logits (dtype SFMP_TYPE_FP16, _BF16 or _FP32; row i
 * at logits + i * stride elements, vocab of them) and of scores (fp32, the sums of log-probabilities so far).  Token t continues row i with the value
 *     scores[i] + (l_t - m) - ln sum_j exp(l_j - m),   m the row's largest logit,
 * and ranks by weights[i] times it (weights NULL: 1; 1 / length to compare beams of different lengths: positive, finite).  A row with ended[i]
 * not 0 (ended NULL: none) has one continuation: end_token, with the value scores[i].  The `choices` continuations of a request that rank
 * highest, of equal ones those of the lower row and then of the lower token, are written in that order: next_scores fp32, parents int32 (the row of
 * logits; what sfmp_kv_reorder takes where choices = beams) and tokens int32, each [requests][choices].
 * NaN logits count as -infinity, +infinity as the largest number of fp32; tokens of -infinity and rows whose score is -infinity or NaN (or that have
 * no logit above -infinity) have no continuation.  Where a request has fewer than `choices`, the rest is -infinity, -1, -1.  (A request that starts
 * from one prompt has the scores 0, -infinity, -infinity, ...)
 * Values are held and compared in 64 bits and rounded once.  Of the sum of exponentials the row's largest `choices` terms are made in 64 bits, the
 * others in 32: one whose logit lies d below the largest enters the sum with an error of at most 2^-24 (10 + 4 d) of itself, mostly far less (with
 * d above 87 it may be left out).  Continuations of different beams whose values lie closer together than that, in proportion to what these other
 * terms weigh (up to 2^-20 where all tokens are alike), may change places.  Rows of equal logits have equal values, whatever their alignment.
 * The same call on the same inputs gives the same bits.  Results do not overlap inputs.
 * SFMP_ERR_SHAPE: requests < 0, beams outside 1 .. 32, requests * beams > 65535, choices outside 1 .. 64, vocab outside 1 .. 2^24, stride < vocab,
 * with ended an end_token outside the vocabulary.  Alignment: logits to their element size.  The workspace is 256-byte aligned, its contents
 * irrelevant on entry; sfmp_beam_select_workspace: bytes that are enough for every call of no more requests, beams, tokens and choices. */
int sfmp_beam_select_workspace(int32_t requests, int32_t beams, int32_t vocab, int32_t choices, int64_t* bytes);
int sfmp_beam_select(const void* logits_dev, int32_t dtype, int32_t requests, int32_t beams, int32_t vocab, int64_t stride,
                     const float* scores_dev, const float* weights_dev, const int32_t* ended_dev, int32_t end_token, int32_t choices,
                     float* next_scores_dev, int32_t* parents_dev, int32_t* tokens_dev, void* workspace_dev,
                     int64_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SFMP_H */
