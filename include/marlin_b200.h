/*
 * marlin_b200 -- W4A16 linear layer for NVIDIA B200 (sm_100a), C ABI.
 *
 *     C[M x N] (fp16) = A[M x K] (fp16) . dequant(Wq[K x N] int4, fp16 scales),  fp32 accumulation
 *     dequant:  W[k][n] = (Q[k][n] - 8) * S[k / G][n],  Q in 0..15
 *
 * The operation is the mixed-precision layer of the MARLIN paper (arxiv 2408.11743), Section 3.4
 * "Kernel Design": A in fp16, B a K x N INT4 matrix, symmetrically quantised, with one fp16 scale per
 * output column or per G consecutive weights of a column (ceil(K/G) * N scales).  The 2:4 variant is
 * Section 4 ("The Sparse-MARLIN Kernel"): groups of four along K, two values kept, 2-bit positions.
 *
 * General rules
 *   - Every pointer named *device* is a CUDA device pointer owned by the caller, 16-byte aligned,
 *     valid on the current device until the work queued on `stream` has finished.  Host pointers
 *     are said to be host pointers.  Buffers of one call must not overlap.
 *   - Calls are asynchronous on `stream`; nothing synchronises, nothing is allocated, nothing throws.
 *     Every function that can fail returns a marlin_status; 0 is success.
 *   - There is no CPU path and no other-architecture path: on a device that is not compute
 *     capability 10.x the calls return MARLIN_ERR_ARCH.
 *   - Shapes: K % 128 == 0, K <= 2^20, N % 64 == 0, N <= 65536, M >= 1 (any number of rows: a call splits
 *     them over as many launches as it needs).  group_size is a multiple of 128 that divides K, or K itself
 *     (also written -1): one scale per column; on layers whose N is a multiple of 256 also 64 or 32 (Section 2.3,
 *     group quantization with smaller groups; other values return MARLIN_ERR_GROUP).
 *   - The packed device layout is opaque (the design notes of this repository describe it); only marlin_pack* writes it and
 *     only marlin_unpack* / marlin_gemm* read it.
 */
#ifndef MARLIN_B200_H_
#define MARLIN_B200_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define MARLIN_API __attribute__((visibility("default")))
#else
#define MARLIN_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MARLIN_OK = 0,
  MARLIN_ERR_NULL = 1,           /* a required pointer is NULL                                  */
  MARLIN_ERR_SHAPE = 2,          /* M, K or N out of range or not a multiple of the tile sizes  */
  MARLIN_ERR_GROUP = 3,          /* group_size not supported for this K                         */
  MARLIN_ERR_ALIGN = 4,          /* a device pointer is not 16-byte aligned                     */
  MARLIN_ERR_WORKSPACE = 5,      /* workspace smaller than marlin_workspace_bytes()             */
  MARLIN_ERR_ARCH = 6,           /* current device is not sm_100                                */
  MARLIN_ERR_CUDA = 7,           /* a CUDA runtime call or the launch failed                    */
  MARLIN_ERR_DEVICE_TIMEOUT = 8, /* a bounded wait inside a kernel expired (see marlin_read_status) */
  MARLIN_ERR_CACHE = 9           /* a length or a page number points outside of the cache: kernels report it through
                                    marlin_read_status, and leave out what it would have reached */
} marlin_status;

/* A CUDA stream handle (cudaStream_t) passed as an opaque pointer; NULL is the default stream. */
typedef void* marlin_stream;

MARLIN_API const char* marlin_status_string(int status);

/* ---- sizes (host arithmetic only; valid without a GPU) ------------------------------------- */

/* Bytes of the packed weight buffer: K*N/2 dense; K*N/4 when sparse24 != 0.  0 on a bad shape. */
MARLIN_API size_t marlin_packed_weight_bytes(int K, int N, int sparse24);
/* Bytes of the packed scale buffer: 2 * (K/G) * N.  0 on a bad shape or group size. */
MARLIN_API size_t marlin_packed_scale_bytes(int K, int N, int group_size);
/* Bytes of the packed 2:4 metadata buffer: K*N/8 (2 bits per kept value). */
MARLIN_API size_t marlin_packed_meta_bytes(int K, int N);
/* Bytes of the workspace marlin_gemm* needs for any M <= max_M on this K x N layer.
 * The workspace holds a status word, arrival counters and slots for the fp32 partial tiles
 * of the fix-up (the global reduction of Section 3.4 "Striped Partitioning"): at least 5.2 MB, and two slots of
 * 256 columns x 32, 64 or 128 rows per CTA that a batch of max_M rows can use (at most 42 MB).
 * The caller zeroes it ONCE after allocation (cudaMemset); every call leaves the counters zero and writes the slots
 * before it reads them (what they hold between calls is not specified).
 * One workspace must not be used by two calls that can run at the same time.  It may serve calls on
 * different layers, formats and batch sizes one after the other (one stream, or ordered by events) if it
 * has the largest of their sizes: the parts lie at the same offsets for every call. */
MARLIN_API size_t marlin_workspace_bytes(int max_M, int K, int N);

/* ---- offline quantiser (Section 3.5 (a): group scales picked by a search over group-wise clipping
 *      thresholds; here without calibration data: round to nearest, least squared weight error) ------ */

/* fp16 weights -> canonical 4-bit codes and fp16 group scales, the inputs of marlin_pack.
 *   W             device, fp16 [K][N] row-major, finite values
 *   q_kpacked     device, out, uint32 [K/8][N]: nibble j of word (kb, n) = code of row 8*kb + j, codes 0..15 = q
 *   scales        device, out, fp16 [K/G][N]
 *   n_grid, n_candidates   1 <= n_candidates <= n_grid: candidate t = 0 .. n_candidates-1 clips the group's range
 *                 to r_t = 1 - t / n_grid of its largest magnitude a (n_candidates = 1: plain round to nearest)
 * Per group of G rows of a column: s_t = fp16(2 a r_t / 15) (never zero: at least the smallest positive fp16),
 * q_i = clamp(round_half_even(w_i / s_t), -8, 7) + 8, and the candidate with the least sum of squared errors
 * (w_i - (q_i - 8) s_t)^2 wins, the first one on ties.  All of it in fp32 with a fixed order of operations (see
 * csrc/quantize.cu), so the outputs are reproducible bit for bit.  Shapes and group sizes as for marlin_pack;
 * pointers 16-byte aligned; errors are returned before anything is queued. */
MARLIN_API int marlin_quantize_rtn(const void* W, uint32_t* q_kpacked, void* scales, int K, int N, int group_size,
                        int n_grid, int n_candidates, marlin_stream stream);

/* ---- offline re-layout (Section 3.4 "Maximizing Loading Bandwidth", "Dequantization and Tensor
 *      Cores": weights are static, so they are reshuffled once into the order the kernel streams) -- */

/* Dense pack.
 *   q_kpacked  device, uint32 [K/8][N]: canonical codes, nibble j of word (kb, n) = Q[8*kb + j][n]
 *   scales     device, fp16   [K/G][N] row-major
 *   w_packed   device, out, marlin_packed_weight_bytes(K, N, 0) bytes
 *   s_packed   device, out, marlin_packed_scale_bytes(K, N, G) bytes
 * Integer-only permutation; unpack(pack(x)) == x bit for bit. */
MARLIN_API int marlin_pack(const uint32_t* q_kpacked, const void* scales, void* w_packed, void* s_packed,
                int K, int N, int group_size, marlin_stream stream);

/* Inverse of marlin_pack: writes the canonical forms back. */
MARLIN_API int marlin_unpack(const void* w_packed, const void* s_packed, uint32_t* q_kpacked, void* scales,
                  int K, int N, int group_size, marlin_stream stream);

/* Zero points for layers quantised asymmetrically, W = (q - z) * s with one integer z in 0..15 per scale group
 * (Section 2.3 "uniform quantization": a zero point and a scale per group; the integer form is the one of the
 * activation-aware format the paper names in Section 6).  Codes and scales go through marlin_pack as usual.
 *   zeros      device, uint8 [K/G][N] row-major, values 0..15
 *   z_packed   device, out, marlin_packed_scale_bytes(K, N, G) bytes (fp16 values in the order of the packed scales)
 * Shapes and group sizes as for marlin_pack. */
MARLIN_API int marlin_pack_zeros(const uint8_t* zeros, void* z_packed, int K, int N, int group_size, marlin_stream stream);
MARLIN_API int marlin_unpack_zeros(const void* z_packed, uint8_t* zeros, int K, int N, int group_size, marlin_stream stream);

/* ---- the layer (Section 3.4, all paragraphs: weight streaming, dequantisation, tensor-core
 *      product, striped partition with global reduction) ----------------------------------------- */

/* C = A . dequant(W).
 *   A          device, fp16 [M][K] row-major
 *   w_packed, s_packed   device, from marlin_pack with the same K, N, group_size
 *   C          device, out, fp16 [M][N] row-major, every element written
 *   workspace  device, at least marlin_workspace_bytes(M, K, N) bytes, zeroed once by the caller
 * Accumulation is fp32 (also across stripes) and the result is rounded to fp16 once (nearest even).  The
 * weights reach the tensor cores as exact integers q - 8 (warp-level kernel, up to 16 rows: scales applied to
 * the fp32 sums per group; tcgen05 kernel where there is one scale per column or N is not a multiple of 256: scales
 * applied to fp32 sums too) or as fp16((q - 8) * s) (tcgen05 kernel otherwise: one more rounding of 2^-11 per
 * weight, as in the paper's kernel).
 * Up to 16 rows the warp-level kernel runs, from 17 rows (from nine on layers of more than 2^26 weights with one scale
 * per column) a tcgen05 kernel.  That one takes all rows in one launch: above
 * 128 rows the layer is replicated in the numbering of the work units, once per slab of up to 128 rows (Section 3.4,
 * last paragraph), and the stripes of the CTAs run over (column tile, slab, k-block), so the weights come from
 * DRAM once and from the L2 after that.  Groups of 64 or 32 rows run on it at every batch size.
 * Partial sums are added in a fixed order everywhere: the same inputs give the same bits on every call.
 * Errors: argument checks return before anything is queued.  A kernel whose bounded waits expire
 * sets the workspace status word; read it with marlin_read_status. */
MARLIN_API int marlin_gemm(const void* A, const void* w_packed, const void* s_packed, void* C,
                int M, int K, int N, int group_size,
                void* workspace, size_t workspace_bytes, marlin_stream stream);


/* ---- the gated MLP of a decoder layer as a chain of two launches (Section 5.1 names the per-kernel overheads on
 *      real layer shapes; fusing the activation removes one launch and the round trip of the wide intermediate) -- */

/* Gate and up projections of one MLP side by side, in the column order the fused epilogue expects: output column
 * n = 16 b + r holds gate channel 8 b + r for r < 8 and up channel 8 b + r - 8 otherwise.
 *   q_gate, q_up   device, uint32 [K/8][I] canonical codes;   s_gate, s_up   device, fp16 [K/G][I]
 *   q_out          device, out, uint32 [K/8][2 I];            s_out          device, out, fp16 [K/G][2 I]
 * Feed q_out, s_out to marlin_pack with N = 2 I.  I % 32 == 0. */
MARLIN_API int marlin_interleave_gate_up(const uint32_t* q_gate, const void* s_gate, const uint32_t* q_up, const void* s_up,
                              uint32_t* q_out, void* s_out, int K, int I, int group_size, marlin_stream stream);

/* marlin_gemm on such a layer (N = 2 I columns) with the activation fused into the epilogue:
 *   H[m][c] = fp16( silu(g) * u ),  g = fp16(A . W)[m][gate channel c],  u = fp16(A . W)[m][up channel c],
 * silu(g) = g / (1 + exp(-g)) in fp32.  H is device, out, fp16 [M][N/2] row-major.  Everything else as marlin_gemm
 * (the product is rounded to fp16 before the activation, as it would be if H were computed from a stored C). */
MARLIN_API int marlin_gemm_swiglu(const void* A, const void* w_packed, const void* s_packed, void* H, int M, int K, int N,
                       int group_size, void* workspace, size_t workspace_bytes, marlin_stream stream);

/* C = (silu(A . W_gate) * (A . W_up)) . W_down: marlin_gemm_swiglu into H (device scratch, fp16 [M][I]), then
 * marlin_gemm of H with the down projection (I x N).  One workspace serves both launches (they run one after the
 * other on `stream`): at least max(marlin_workspace_bytes(M, K, 2 I), marlin_workspace_bytes(M, I, N)) bytes. */
MARLIN_API int marlin_mlp_swiglu(const void* A, const void* w_gate_up, const void* s_gate_up, const void* w_down,
                      const void* s_down, void* H, void* C, int M, int K, int I, int N, int group_size,
                      void* workspace, size_t workspace_bytes, marlin_stream stream);

/* ---- 8-bit weights (Section 6 names other formats the approach extends to): W = (q - 128) * s, q in 0..255 ------ */

/* q8: device, uint8 [K][N] row-major codes; scales as for marlin_pack.  w_packed: marlin_packed_weight_bytes_w8(K, N)
 * = K * N bytes.  N % 256 == 0 (these layers run on the tcgen05 kernel at every batch size).  Integer-only
 * permutation; marlin_unpack_w8 is its inverse bit for bit. */
MARLIN_API size_t marlin_packed_weight_bytes_w8(int K, int N);
MARLIN_API int marlin_pack_w8(const uint8_t* q8, const void* scales, void* w_packed, void* s_packed, int K, int N,
                   int group_size, marlin_stream stream);
MARLIN_API int marlin_unpack_w8(const void* w_packed, const void* s_packed, uint8_t* q8, void* scales, int K, int N,
                     int group_size, marlin_stream stream);
/* C = A . W as marlin_gemm; the conversion places a code byte under the exponent of 1024 and subtracts 1152 (the
 * 8-bit form of the exponent trick of Section 3.4 "Dequantization and Tensor Cores"), scales in the loop. */
MARLIN_API int marlin_gemm_w8(const void* A, const void* w_packed, const void* s_packed, void* C, int M, int K, int N,
                   int group_size, void* workspace, size_t workspace_bytes, marlin_stream stream);

/* The layer with zero points: C = A . W, W[k][n] = (q[k][n] - z[k/G][n]) * s[k/G][n].  Arguments as marlin_gemm, plus
 * z_packed from marlin_pack_zeros.  Up to 16 rows the
 * warp-level kernel runs: the weights enter the MMAs as for the symmetric layer and one more MMA per 16 rows of k,
 * with an all-ones weight operand, gives sum_k a[k][m] per group, so that the group closes with
 * s * (sum_k a (q - 8) + (8 - z) sum_k a).  Above, the tcgen05 kernel, where the zero point replaces the constant 8
 * inside the conversion (the subtrahend of the exponent trick of Section 3.4 "Dequantization and Tensor Cores"
 * becomes 1024 + z): no extra instruction per weight.  workspace: marlin_workspace_bytes(M, K, N). */
MARLIN_API int marlin_gemm_zp(const void* A, const void* w_packed, const void* s_packed, const void* z_packed, void* C,
                   int M, int K, int N, int group_size, void* workspace, size_t workspace_bytes,
                   marlin_stream stream);

/* The same layer for callers that cannot allocate device memory or carry a workspace pointer
 * around: for example a plug-in that runs inside another framework's pre-captured execution plan,
 * or a constrained runtime where cudaMalloc is forbidden after start-up.  (The paper has no
 * counterpart; this is a convenience of this library.)
 *
 * Works like marlin_gemm, but the fix-up workspace is a fixed array inside the library's device
 * image (about 5 MB, held by every GPU that loads the library until the process exits), so only
 * M <= MARLIN_STATIC_WS_MAX_M is accepted; larger M returns MARLIN_ERR_SHAPE.  The call allocates
 * nothing: no cudaMalloc, no cudaFree, no library routine that allocates.
 *
 * The first call on each device looks up the device address of that array (with that device
 * current) and remembers it; make this first call outside any stream capture.  Every call clears
 * the arrival counters of the array on `stream` before the kernels run (the array keeps whatever
 * the previous call left), and all calls on one device share the one array: two such calls that
 * can overlap on the GPU (two streams, or two host threads) race with each other and must be
 * serialised by the caller.
 * Errors: the argument checks of marlin_gemm, made before anything is queued; MARLIN_ERR_CUDA if
 * the address lookup or the clearing fails.  The array's status word is private to the library:
 * a bounded wait that expires inside a kernel of this entry point is NOT reported to the caller
 * (use marlin_gemm with a workspace of your own and marlin_read_status where that matters). */
#define MARLIN_STATIC_WS_MAX_M 16
MARLIN_API int marlin_gemm_static_ws(const void* A, const void* w_packed, const void* s_packed, void* C,
                                     int M, int K, int N, int group_size, marlin_stream stream);

/* ---- 2:4 structured-sparse variant (Section 4: values structure + metadata indices) ------------ */

/* Pack the compressed form.
 *   qc_kpacked device, uint32 [K/16][N]: kept codes Qc[K/2][N], nibble j of word (r, n) = Qc[8r+j][n]
 *   idx        device, uint8  [K/2][N]: position 0..3 of kept value t inside group t/2 of four rows
 *              along K; idx[2u][n] < idx[2u+1][n]
 *   scales     device, fp16 [K/G][N], groups over the ORIGINAL K
 *   outputs    w_packed (K*N/4 bytes), meta_packed (K*N/8 bytes), s_packed (2*(K/G)*N bytes) */
MARLIN_API int marlin_pack_sparse24(const uint32_t* qc_kpacked, const uint8_t* idx, const void* scales,
                         void* w_packed, void* meta_packed, void* s_packed,
                         int K, int N, int group_size, marlin_stream stream);

MARLIN_API int marlin_unpack_sparse24(const void* w_packed, const void* meta_packed, const void* s_packed,
                           uint32_t* qc_kpacked, uint8_t* idx, void* scales,
                           int K, int N, int group_size, marlin_stream stream);

/* C = A . dequant(expand(W)) with the pruned positions contributing zero.  Layers whose N is a multiple of 256
 * run on the sparse tcgen05 instruction (tcgen05.mma.sp) at every batch size, all rows in one launch (slabs of
 * rows as in marlin_gemm), reading the compressed weights from DRAM once; other N on the warp-level sparse
 * MMA in slabs of 16 rows. */
MARLIN_API int marlin_gemm_sparse24(const void* A, const void* w_packed, const void* meta_packed,
                         const void* s_packed, void* C, int M, int K, int N, int group_size,
                         void* workspace, size_t workspace_bytes, marlin_stream stream);

/* ---- the paged key-value cache: the part of a decoder layer between the qkv layer and the output layer -----------
 *
 * Section 5.2 of the paper measures these layers inside a serving engine; there the tokens that a sequence has so far
 * are kept as keys and values in pages of a fixed number of tokens, handed out in any order. */

#define MARLIN_KV_FP16 0  /* cache elements are fp16 */
#define MARLIN_KV_E4M3 1  /* cache elements are 8-bit floats (4 exponent and 3 mantissa bits, largest 448), and stand for
                             their value times k_scale[head] or v_scale[head] */

/* A cache and its tables (a host structure of device pointers; the library keeps none of it after a call).
 * Element d of head h of the token at position p of sequence b lies in k (and in v) at
 *   table[b * table_stride + p / page_size] * stride[0] + h * stride[1] + (p % page_size) * stride[2] + d
 * so [pages][heads][page_size][head_dim] and [pages][page_size][heads][head_dim] are both of this form.  Strides count
 * elements and are multiples of 16 bytes; k and v (16-byte aligned, or NULL nowhere) have the same ones.  No two of
 * these places may overlap. */
typedef struct {
  void* k;                 /* device                                                                            */
  void* v;                 /* device                                                                            */
  int64_t stride[3];       /* elements between pages, heads and tokens                                          */
  const int32_t* table;    /* device, [sequences][max_pages]: page numbers; entries behind a sequence's last page
                              are not read                                                                      */
  int64_t table_stride;    /* entries between sequences, >= max_pages                                           */
  const int32_t* lengths;  /* device, [sequences]: tokens of each sequence, the new ones of the call included   */
  const float* k_scale;    /* device, [kv_heads], or NULL (1); 8-bit caches only                                */
  const float* v_scale;
  int pages;               /* pages in k and v                                                                  */
  int max_pages;           /* entries of a row of `table`                                                       */
  int sequences;
  int kv_heads;
  int head_dim;            /* a multiple of 16, at most 256                                                     */
  int page_size;           /* tokens, a power of two                                                            */
  int format;              /* MARLIN_KV_FP16 or MARLIN_KV_E4M3                                                  */
} marlin_kv_cache;

/* The new tokens of a call: rows starts[b] .. starts[b + 1] - 1 of the inputs belong to sequence b, in the order of their
 * positions, of which the last is lengths[b] - 1; `starts` is device, int32 [sequences + 1], not descending, its values
 * in 0 .. tokens.  NULL: one token per sequence (tokens == sequences), row b for sequence b.  Rows in front of starts[0]
 * and behind starts[sequences] belong to nobody: neither the cache nor their rows of the outputs are written.  A token whose position
 * would be negative (a sequence with fewer tokens than rows, for example an empty one of a padded batch) is not put
 * into the cache; its rows of the outputs are zeros.
 * A sequence whose length lies outside of 0 .. max_pages * page_size (or 2^30, if that is less) has no positions at all: its new
 * tokens are not put into the cache, nothing is read for them, and their rows of the outputs are zeros.  A page number outside
 * of 0 .. pages - 1 is a page that is not there (nothing is written to it, attention reads zeros for it).  Both set the status
 * word to MARLIN_ERR_CACHE. */

/* Bytes of workspace of the three calls below on heads of head_dim elements (0: not supported; host arithmetic only).
 * The workspace is that of marlin_workspace_bytes and under the same contract: zeroed once, the counters zero again
 * after every call, one call at a time; one buffer of the largest size serves these calls and the layers. */
MARLIN_API size_t marlin_attention_workspace_bytes(int head_dim);

/* Puts the keys and values of new tokens into the cache and rotates queries and keys by their positions.
 *   q, k, v    device, fp16: heads of one token side by side, q_heads (or kv_heads) * head_dim values, tokens q_stride,
 *              k_stride, v_stride elements apart (multiples of 8): three column ranges of the output of one qkv layer,
 *              or three tensors.  q may be NULL (and q_heads 0): only the cache is written.
 *   q_out      device, out, fp16 [tokens][q_heads * head_dim]; NULL where q is
 *   inv_freq   device, fp32 [rotary_dim / 2]: radians per position of each pair, or NULL: no rotation (then q must be NULL)
 *   rotary_dim a multiple of 16, at most head_dim: the first rotary_dim elements of a head are rotated, in pairs
 *              (j, j + rotary_dim / 2), or (2 j, 2 j + 1) where `interleaved` is set:
 *                (a, c) -> (a cos t - c sin t, c cos t + a sin t),  t = position * inv_freq[j]
 * Angles are formed in 64 bits and reduced by whole turns before sine and cosine are taken in fp32; the rotation is fp32
 * and the result is rounded once (to nearest even; to e4m3 after division by the scale, saturating at 448, NaN kept). */
MARLIN_API int marlin_kv_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                     void* q_out, const marlin_kv_cache* cache, const int32_t* starts, int tokens, int q_heads,
                     const float* inv_freq, int rotary_dim, int interleaved,
                     void* workspace, size_t workspace_bytes, marlin_stream stream);

/* Attention of new tokens over the cache, which holds them already (marlin_kv_append).
 *   q          device, fp16, q_heads * head_dim values per token, tokens q_stride elements apart (a multiple of 8); query
 *              head h reads key head h / (q_heads / kv_heads), q_heads a multiple of kv_heads
 *   scale      factor of the logits, usually 1 / sqrt(head_dim)
 *   window     0, or the number of positions that a token sees, its own included (a sliding window)
 *   out        device, out, fp16 [tokens][q_heads * head_dim]
 * out = sum_j w_j v_j, w = softmax over the positions j <= p, j > p - window of scale * q . k_j, p the token's position;
 * zeros where there is none.  Values at other positions never reach a result, whatever they are (infinities, NaN).
 * One launch: the tiles of 32 to 128 keys of all sequences and key heads are numbered through and cut into about equal ranges,
 * one per CTA (the stripes of Section 3.4 "Striped Partitioning"); parts of a sequence are joined by the CTA that comes
 * last, in the order of the keys, so that the same inputs give the same bits on every call.  Sums and the softmax are fp32;
 * a weight is rounded to fp16 before it is multiplied with a value: by at most 2^-11 of it, or 2^-32 of the largest weight of its
 * row if that is more.  One below that counts as 0 there (n such keys are missing from the result by up to n 2^-32 of the weights,
 * and an infinite value under such a weight gives NaN).  A call of
 * 2^32 tiles or more (an item counts for two to four beside its own; 40 s of work with heads of 128 elements) is refused
 * on the device (MARLIN_ERR_CACHE, nothing is written).
 * Any number of tokens per sequence is right; it is made for one and the few of speculative decoding (bound by reading the cache).
 * With many of them, rows are taken in blocks of 64, and every block goes over all tiles between the first token's window and the
 * end of the sequence, also those that its own rows do not see: a prompt costs about twice the products it needs, and
 * with a window as much as without one.  (A prompt of 2048 tokens, 64 heads over 8 of 128 elements: 0.6 ms.) */
MARLIN_API int marlin_attention_decode(const void* q, int64_t q_stride, const marlin_kv_cache* cache, const int32_t* starts,
                            int tokens, int q_heads, float scale, int window, void* out,
                            void* workspace, size_t workspace_bytes, marlin_stream stream);

/* The attention half of a decoder layer as a chain of four launches (marlin_mlp_swiglu is the other half): QKV = A . W_qkv,
 * marlin_kv_append of its columns (q_heads, then kv_heads keys, then kv_heads values), marlin_attention_decode, C = O . W_o.
 *   A       device, fp16 [M][K], M tokens;  W_qkv: K x (q_heads + 2 kv_heads) * head_dim, W_o: q_heads * head_dim x N
 *   QKV, Q, O   device scratch, fp16 [M][(q_heads + 2 kv_heads) * head_dim], [M][q_heads * head_dim] twice.  Q may be NULL
 *           where inv_freq is.  Rows of O that belong to no sequence are not written, and go through W_o as they are.
 *   workspace   the largest of marlin_workspace_bytes of both layers and marlin_attention_workspace_bytes.
 * All arguments are checked before anything is queued. */
MARLIN_API int marlin_attention_block(const void* A, const void* w_qkv, const void* s_qkv, const void* w_o, const void* s_o,
                           void* QKV, void* Q, void* O, void* C, const marlin_kv_cache* cache, const int32_t* starts,
                           int M, int K, int q_heads, int N, int group_size, const float* inv_freq, int rotary_dim,
                           int interleaved, float scale, int window,
                           void* workspace, size_t workspace_bytes, marlin_stream stream);

/* ---- the same cache in 8 bits with a scale for each block of tokens, and with first tokens that stay visible -------- */

#define MARLIN_KV_INT8 2  /* `format` of a cache of the calls below that is given scales by block: codes in two's complement */

/* Scales of an 8-bit cache (MARLIN_KV_E4M3 or MARLIN_KV_INT8; its own k_scale and v_scale are NULL then): a code of head h of the token
 * at position p stands for its value times
 *   k[page * stride[0] + h * stride[1] + (p % page_size) / block_size * stride[2]]       (page: its page of the table; v alike)
 * Strides count floats.  block_size is a power of two, at most page_size and 128.  No two scales share a place. */
typedef struct {
  float* k;           /* device */
  float* v;           /* device */
  int64_t stride[3];  /* floats between pages, heads and blocks */
  int block_size;     /* tokens */
} marlin_kv_scales;

/* marlin_kv_append into such a cache, whose scales are made on the way: nothing has to be measured beforehand.  With L the largest code (127;
 * 448 in e4m3) and a the largest magnitude of the new elements of a head in a block, after the rotation, that is finite:
 *   a block whose first token is among the new ones gets the scale s = a / L, whatever it held before (in fp32, a times the number nearest to 1 / L);
 *   one that has tokens already keeps its scale if a / L <= s, otherwise s is doubled until that is so, and the codes of its earlier tokens
 *   are divided by the same power of two and rounded to nearest even (so a code loses at most a step of the block's last scale, however often
 *   that grew; nothing in e4m3 except where it becomes subnormal).  A scale that is not finite and above 0 stands for codes of 0, and for
 *   no scale: the block gets s = a / L, and the codes of its earlier tokens become 0, those of NaN too.
 *   codes are the nearest (even) of x * (1 / s) in fp32; an infinity becomes the largest code, a NaN stays one in e4m3 and is 0 in two's
 *   complement.  Where a is 0 and the block has no scale yet, s is 0 and all codes are 0, also those of infinities; a NaN stays one in e4m3.
 * Tokens that are taken back later (marlin_kv_reserve) leave the scale as they made it, and the codes of the tokens in front of them in its coarser steps.
 * Sines and cosines are off by at most 2^-20 (2^-22 in marlin_kv_append, whose rotated queries can have other last bits).  Everything else as
 * there.  The same inputs give the same bits on every call; a prompt in two calls can give other ones than in one. */
MARLIN_API int marlin_kv_append_scaled(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            void* q_out, const marlin_kv_cache* cache, const marlin_kv_scales* scales, const int32_t* starts, int tokens,
                            int q_heads, const float* inv_freq, int rotary_dim, int interleaved,
                            void* workspace, size_t workspace_bytes, marlin_stream stream);

/* marlin_attention_decode over any cache of this header (scales NULL: fp16, or e4m3 with scales by key head), where a token at position p sees
 * besides the `window` last positions the first `sinks` ones: j <= p and (j > p - window or j < sinks).  (sinks mean nothing without
 * a window.)  Results, errors and limits as there, with three differences:
 *   with scales by block the weights are rounded to fp16 together with the scales of their values, so a product w_j s_j is off by at most
 *   2^-11 of it, or 2^-31 of the largest weight of its row times the largest scale that it meets, if that is more;
 *   blocks of rows go only over tiles that some of their rows can see, so that a prompt with a window costs what the window holds;
 *   a scale that is not finite reaches the rows that see its tokens, and no others.
 * Many tokens a sequence over fp16 and up to 128 elements have a kernel of their own, here only: a prompt of 2048 tokens, 64 heads over 8 of 128 elements,
 * 136 us (marlin_attention_decode: 0.6 ms).  Whether a call takes it goes by the mean of its tokens a sequence; sequences with one token each beside a
 * prompt are right, but each of their key heads then costs a block of 256 rows that one CTA goes through alone. */
MARLIN_API int marlin_attention_sinks(const void* q, int64_t q_stride, const marlin_kv_cache* cache, const marlin_kv_scales* scales,
                           const int32_t* starts, int tokens, int q_heads, float scale, int window, int sinks, void* out,
                           void* workspace, size_t workspace_bytes, marlin_stream stream);

/* marlin_attention_block with marlin_kv_append_scaled (where scales are given) and marlin_attention_sinks in the middle. */
MARLIN_API int marlin_attention_block_sinks(const void* A, const void* w_qkv, const void* s_qkv, const void* w_o, const void* s_o,
                                 void* QKV, void* Q, void* O, void* C, const marlin_kv_cache* cache, const marlin_kv_scales* scales,
                                 const int32_t* starts, int M, int K, int q_heads, int N, int group_size, const float* inv_freq,
                                 int rotary_dim, int interleaved, float scale, int window, int sinks,
                                 void* workspace, size_t workspace_bytes, marlin_stream stream);

/* ---- page tables from lengths ------------------------------------------------------------------------------------- */

/* The pages of a cache as marlin_kv_reserve keeps them (a host structure of device pointers; what they point to is read and written). */
typedef struct {
  int32_t* table;       /* device, [sequences][max_pages]: page numbers of each sequence, as in marlin_kv_cache */
  int64_t table_stride;
  int32_t* lengths;     /* device, [sequences]: tokens of each sequence */
  int32_t* free_pages;  /* device, [capacity]: numbers of pages that nobody has; the last of the first free_count[0] is handed out first */
  int32_t* free_count;  /* device, [1] */
  int capacity;         /* of free_pages: as many as there are pages */
  int max_pages;
  int sequences;
  int page_size;        /* tokens, a power of two */
} marlin_kv_pages;

/* Makes room for the new tokens of a step, and takes back what sequences do not need any more.  Sequence b with lengths[b] tokens keeps the first
 * min(keep[b], lengths[b]) of them and gets counts[b] new ones behind these; lengths[b] becomes the sum.  (Drafted tokens that were not
 * accepted: keep is less than the length.  A sequence that ends: keep and count 0.  The scale of a block that drafts have made larger stays, see
 * marlin_kv_append_scaled.)
 *   counts     device, int32 [sequences], or NULL: one each;   keep   device, int32 [sequences], or NULL: all
 *   tokens     rows of the step: at least the sum of the counts (0: none).  2^30 tokens and 2^30 sequences are the most.
 *   starts     device, out, int32 [sequences + 1], or NULL: starts[b] = counts[0] + .. + counts[b - 1] (2^31 - 1 if that is less; negative
 *              counts are none), what the calls above take
 *   slots      device, out, int64 [tokens], or NULL: table[b][p / page_size] * page_size + p % page_size for the token at position p
 *   positions  device, out, int32 [tokens], or NULL: p.  Both are -1 in rows behind the last token and in those of refused sequences.
 * Pages are taken from the top of the stack, in the order of the sequences and of their positions; entries of the table behind the
 * last page are not touched.  Pages that are not needed any more go back on the stack in the order in which the same pages
 * would be taken again: a step that is taken back leaves stack and lengths as they were.  They are handed out from the next call on.
 * A sequence is refused, and left as it was, when fewer pages are free than it and the sequences in front of it need (sequences that need
 * none are served all the same), when its row of the table is too short, its count negative or its rows lie behind `tokens`.  Its length
 * becomes -1 - length: the calls above leave it out and report it, and the next call here takes it for the length again.  (Only the
 * last three reasons set the status word to MARLIN_ERR_CACHE.)
 * workspace: at least 8192 bytes under the contract of marlin_workspace_bytes.  One launch; nothing is read on the host. */
MARLIN_API int marlin_kv_reserve(const marlin_kv_pages* pages, const int32_t* counts, const int32_t* keep, int tokens, int32_t* starts,
                      int64_t* slots, int32_t* positions, void* workspace, size_t workspace_bytes, marlin_stream stream);

/* Synchronises `stream`, then returns the device-side status word of `workspace`
 * (MARLIN_OK, MARLIN_ERR_DEVICE_TIMEOUT if a kernel gave up a bounded wait, or MARLIN_ERR_CACHE), or
 * MARLIN_ERR_CUDA if the stream reports an error.  The status word is sticky until the
 * workspace is zeroed again.  Where there have been both, it is MARLIN_ERR_DEVICE_TIMEOUT: results of that call and the counters
 * are not to be relied on, while MARLIN_ERR_CACHE says that some tokens were left out and all else is right. */
MARLIN_API int marlin_read_status(const void* workspace, marlin_stream stream);

/* ---- host-side planning, exposed for inspection and tests (no GPU needed) ----------------------- */

/* The partition of Section 3.4 "Striped Partitioning", adapted to this shape, for the warp-level kernel:
 * the (column tile, 128-row k-block) units of the weight matrix are numbered column tile by column tile,
 * top to bottom, and worker i of `workers` owns units [bounds[i], bounds[i+1]).  Two forms: where the
 * column tiles divide the SMs well, every tile is cut into the same number of equal k-ranges, one per
 * worker (no stripe crosses a tile boundary); otherwise the units are cut into `workers` even stripes,
 * the paper's form.  Fills n_tile (columns per tile: 64, 128 or 256), workers (<= sm_count) and
 * bounds[0..workers] (host pointers; `cap` entries available in bounds).
 * This is the base form.  A launch may take another: fewer CTAs, which leave SMs to the next launch, or pairs of
 * workers with several column tiles, where its cost model finds that faster.
 * Returns MARLIN_ERR_SHAPE if cap is too small or the shape is invalid. */
MARLIN_API int marlin_plan_stripes(int M, int K, int N, int sm_count, int* n_tile, int* workers,
                        int64_t* bounds, int cap);

#ifdef __cplusplus
}
#endif
#endif /* MARLIN_B200_H_ */
