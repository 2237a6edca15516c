/*
 * hufflm.h - C ABI of the Huff-LLM bf16 weight codec and its fused
 * decode-GEMV for AMD gfx950 (MI355X).
 *
 * Method: Huff-LLM (arXiv 2502.00922). A bf16 weight is split 1-4-4-7
 * (Sec. 5.1): sign and 7 mantissa bits are kept raw; the 8 exponent bits are
 * two 4-bit symbols, each coded with a per-matrix Huffman code (Sec. 3.1,
 * Sec. 5.1). Compression runs once, offline, on the CPU (Sec. 3.1). Weights
 * stay compressed in memory and are decoded only where they are multiplied
 * (Sec. 1 contributions, Sec. 3.2): here inside y = W x, so that HBM carries
 * only compressed bytes.
 *
 * ---------------------------------------------------------------------------
 * HLF1 container (all integers little-endian)
 * ---------------------------------------------------------------------------
 * W is row-major [rows][cols]; weight i = r*cols + c.
 * Fields of a weight w: s = w>>15, eh = (w>>11)&15, el = (w>>7)&15, m = w&127.
 *
 * Codebooks, one per field per matrix: histogram of the field over the whole
 * matrix; Huffman code lengths from a binary heap keyed (weight, kind, id),
 * kind 0 = leaf with id = symbol, kind 1 = internal node with id = creation
 * order, the two smallest keys merged first; if the longest code exceeds lmax
 * the lengths are replaced by package-merge lengths (items sorted by
 * (weight, symbol); lmax-1 rounds of pairing consecutive items and stable
 * merging with the leaves by (weight, kind); the first 2(n-1) items of the
 * last list are taken; length = occurrences). A field with one present
 * symbol has length 0 and emits no bits. With a joint limit pair_max (see
 * hl_build_codebook) the two fields' limits are a and min(lmax, pair_max - a)
 * for the a of least total code length. Code values are canonical (RFC 1951
 * Sec. 3.2.2 assignment).
 *
 * Tiling: segment (r, cs) is W[r][cs*S .. cs*S+S) (S divides cols, S % 8 == 0,
 * 8 <= S <= 512, L = cols/S segments per row). A group is GR rows x GC
 * consecutive column segments, GR*GC = 64 (GR = group_rows, a power of two,
 * with GC dividing L): row block rb is rows GR*rb .. GR*rb+G-1 (G = GR, or
 * fewer in the last block), column block cb is segments cb*GC .. cb*GC+GC-1,
 * and group g = rb*(L/GC) + cb. Its N = G*GC segments are numbered
 * mu = j*G + i for row offset i < G and segment offset j < GC; a 64-wide
 * wavefront decodes one group, one segment per lane. Segments are numbered in
 * group order: group g starts at segment GR*rb*L + cb*GC*G.
 *
 * Stream: for each weight of a segment in order, code(el) then code(eh),
 * each emitted most-significant bit first; the stream is packed least
 * significant bit first (bit k is bit k%8 of byte k/8). Segment mu of a group
 * occupies stored(mu) = base + seg_len[mu] bits: its codes, then zero bits up
 * to that length. base is the least code-bit count among the group's
 * segments, or the greatest minus 255 when they span more than 255 bits (the
 * shorter segments are then padded to base), so that every seg_len fits one
 * byte. The segments of a group are concatenated in mu order; each group
 * stream starts on a 16-byte boundary and is zero-padded to a multiple of 128
 * bits. (The paper's decoder reads one stream serially, Sec. 3.2, and needs
 * no lengths; here every segment is decoded from its own start.)
 *
 * Layout (sections start at 64-byte boundaries, zero padding between):
 *   0      header (128 bytes, below)
 *   off_seg_bits  uint8 seg_len[n_seg]      stored bits of each segment over
 *                                           its group's base
 *   off_grp_off   uint32 grp_meta[2n_grp+1] group g: [2g] stream start in
 *                                           16-byte units from off_stream,
 *                                           [2g+1] base; [2n_grp] the end
 *   off_stream    group streams
 *   off_raw       uint8 raw[n]: (s<<7)|m; group g starts at S times its first
 *                 segment number; weight t of segment mu is at ((t/8)*N + mu)*8
 *                 + t%8 within the group
 *   total_bytes = off_raw + n
 * Header: u32 magic 0x31464C48 ('HLF1'), u16 version 2, u8 lmax, u8 flags,
 *   u64 rows, u64 cols, u32 seg_len, u32 group_rows (GR), u64 n_seg,
 *   u64 n_grp, u64 off_seg_bits, u64 off_grp_off, u64 off_stream,
 *   u64 off_raw, u64 total_bytes, u32 max_grp_units, u8 eh_nsym, u8 el_nsym,
 *   u8 eh_single, u8 el_single, u8 eh_len[16], u8 el_len[16].
 *
 * flags 0 is the split format above. flags 1 is the whole-exponent format:
 * the exponent byte e = (w>>7)&255 is one symbol of a single per-matrix code
 * over 256 symbols (the same Huffman, package-merge and canonical rules, with
 * lmax in [8, 13]), and the stream holds code(e) for each weight of a segment
 * in order, most-significant bit first. Its 256 code lengths (u8, indexed by
 * e) follow the header at byte 128, so off_seg_bits = 384. Header bytes
 * 92..93 hold the u16 count of present exponent values, byte 94 the value
 * when it is the only one (else 0), bytes 95..127 are zero. Everything else
 * (tiling, padding, offsets, raw plane) is as in the split format. The split
 * follows the paper's split-size analysis (Sec. 3.1): an 8-bit symbol is
 * costly for a single-cycle CAM match, not for a table lookup in local memory.
 *
 * flags 2 is the float16 format, the paper's {1,5,5,5} split (Sec. 3.1,
 * Sec. 3.2): a float16 weight w is sign s = w>>15 (kept raw), exponent
 * e = (w>>10)&31, mantissa-high mh = (w>>5)&31 and mantissa-low ml = w&31;
 * e, mh and ml each have a per-matrix code over 32 symbols (the same rules,
 * lmax in [5, 12]). The stream holds code(ml), code(e), code(mh) for each
 * weight of a segment in order, each most-significant bit first. A 128-byte
 * section after the header holds three records (e, mh, ml) of u8 nsym,
 * u8 single, u8 len[32], then zeros; off_seg_bits = 256; header bytes 92..127
 * are zero. The raw plane holds only signs: byte k*(S/8) + t/8, bit t%8 is the
 * sign of weight t of the segment numbered k in group order, and
 * total_bytes = off_raw + n/8.
 *
 * ---------------------------------------------------------------------------
 * Conventions of the ABI
 * ---------------------------------------------------------------------------
 * Pointers named *_dev are device (HBM) pointers; all others are host. The
 * caller owns every buffer; the library allocates no device memory and keeps
 * no state across calls. `stream` is a hipStream_t (NULL = default stream).
 * Launch functions are asynchronous: they validate arguments on the host,
 * enqueue kernels and return; HL_EHIP reports a failed launch. Corruption
 * that only the device could see is not reported: kernels clamp every read
 * to the container, so a damaged stream gives wrong weights, never a fault.
 * No function throws; all are reentrant.
 */
#ifndef HUFFLM_H
#define HUFFLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HL_OK = 0,
  HL_EINVAL = 1,        /* bad argument (null pointer, size, range) */
  HL_ENOMEM = 2,        /* output buffer too small / host allocation failed */
  HL_ECORRUPT = 3,      /* container fails validation */
  HL_EUNSUPPORTED = 4,  /* valid request this build does not handle */
  HL_EHIP = 5           /* HIP runtime error */
} hl_status;

/* HL_E4M3: 8 bits (4 of exponent, 3 of mantissa, no infinities), only where a
 * function names it. */
typedef enum { HL_F32 = 0, HL_BF16 = 1, HL_F16 = 2, HL_E4M3 = 3 } hl_dtype;

#define HL_MAGIC 0x31464C48u
#define HL_VERSION 2u
#define HL_HEADER_BYTES 128u
#define HL_GROUP_SEGS 64u
#define HL_MAX_BATCH 16u
#define HL_LUT_BYTES 49440u   /* decode tables of the largest format (float16) */
#define HL_LEN8_BYTES 256u    /* whole-exponent code lengths after the header */
#define HL_LMAX8_MIN 8u
#define HL_LMAX8_MAX 13u
#define HL_CB16_BYTES 128u    /* float16 code tables after the header */
#define HL_LMAX16_MIN 5u
#define HL_LMAX16_MAX 12u
#define HL_PAIR_MAX 11u       /* the fused kernel's table window: pairs of codes up to it take the fast form */
#define HL_NORM_MAX_HIDDEN 32768u   /* columns of hl_rms_norm */
#define HL_ATTENTION_MAX_DIM 256u   /* columns of a head in hl_prefix_attention */
#define HL_NOALLOC_SCRATCH_BYTES (4u << 20)  /* scratch of hl_decode_gemv_noalloc, per GPU */

typedef enum { HL_FORMAT_SPLIT = 0, HL_FORMAT_WHOLE_EXPONENT = 1, HL_FORMAT_FP16 = 2 } hl_format;

typedef struct {
  uint8_t nsym;     /* symbols present in the field (1..16) */
  uint8_t single;   /* the symbol when nsym == 1, else 0 */
  uint8_t len[16];  /* code length per symbol; 0 = absent (or the only one) */
} hl_field_code;

typedef struct {
  uint32_t lmax;    /* code-length limit used to build the lengths, 4..15 */
  hl_field_code eh; /* exponent bits 7..4 */
  hl_field_code el; /* exponent bits 3..0 */
} hl_codebook;

/* Whole-exponent code (format 1). */
typedef struct {
  uint32_t lmax;      /* code-length limit used to build the lengths, 8..13 */
  uint16_t nsym;      /* exponent values present (1..256) */
  uint8_t single;     /* the value when nsym == 1, else 0 */
  uint8_t reserved;   /* 0 */
  uint8_t len[256];   /* code length per exponent value; 0 = absent (or the only one) */
} hl_codebook8;

/* One 5-bit field of the float16 format. */
typedef struct {
  uint8_t nsym;     /* symbols present (1..32) */
  uint8_t single;   /* the symbol when nsym == 1, else 0 */
  uint8_t len[32];  /* code length per symbol; 0 = absent (or the only one) */
} hl_field_code5;

/* Float16 codes (format 2). */
typedef struct {
  uint32_t lmax;       /* code-length limit used to build the lengths, 5..12 */
  hl_field_code5 e;    /* exponent, bits 14..10 */
  hl_field_code5 mh;   /* mantissa bits 9..5 */
  hl_field_code5 ml;   /* mantissa bits 4..0 */
} hl_codebook16;

/* Non-owning view of one container resident in device memory. */
typedef struct {
  const uint8_t* blob_dev;   /* whole container */
  uint32_t* lut_dev;         /* HL_LUT_BYTES, filled by hl_tensor_prepare */
  uint64_t rows, cols, n_seg, n_grp, total_bytes;
  uint64_t off_seg_bits, off_grp_off, off_stream, off_raw;
  uint32_t seg_len, grp_rows, lmax, max_grp_units;
  uint32_t max_seg_bits;     /* the longest stored segment (base + seg_len) */
  uint32_t format;           /* hl_format: which of cb / cb8 / cb16 is in use (the others are zero) */
  hl_codebook cb;
  hl_codebook8 cb8;
  hl_codebook16 cb16;
} hl_tensor;

/* Text of a status code (static storage). */
const char* hl_status_str(hl_status s);

/* Segment length the encoder uses for `cols` when asked for 0: among the
 * multiples of 8 in [8, 128] that divide cols with cols/S a multiple of 4
 * (16-row groups), the one nearest to 64 by ratio, the larger on a tie; if
 * there is none, among the multiples of 8 in [8, 512] that divide cols, the
 * one nearest to 128; 0 if there is none. */
uint32_t hl_default_seg_len(uint64_t cols);

/* Per-matrix codebooks of the two exponent fields (Sec. 5.1) from n bf16
 * bit patterns. Each code is limited to lmax bits, lmax in [4, 15] (12
 * matches the maximum code length the paper reports, Sec. 5.2). With
 * pair_max > 0 the longest eh code plus the longest el code is also at most
 * pair_max bits, so that one window of pair_max bits holds every weight's two
 * codes (the decoder's window match of Sec. 3.2 applied to the pair one
 * table lookup decodes): among the splits a + (pair_max - a) of the limit,
 * a = 0 .. lmax, the codes of least total length (each the length-limited
 * optimum for its limit), the smallest a on a tie. 11 is the fused kernel's
 * table window (HL_PAIR_MAX); 0 = no joint limit. Errors: HL_EINVAL for
 * n == 0, null pointers, lmax out of range, pair_max above 30 or too small
 * for the alphabets. */
hl_status hl_build_codebook(const uint16_t* w_bf16, size_t n, uint32_t lmax, uint32_t pair_max,
                            hl_codebook* out);

/* Group rows the encoder uses when asked for 0: 16 (16 rows x 4 segments)
 * when 4 divides the segments per row, else 32, else 64. */
uint32_t hl_default_grp_rows(uint64_t cols, uint32_t seg_len);

/* Encode W [rows][cols] (bf16 bit patterns, host) into an HLF1 container
 * (Sec. 3.1: once, offline, on the CPU). seg_len 0 selects
 * hl_default_seg_len(cols); grp_rows 0 selects hl_default_grp_rows. With
 * out == NULL, *out_bytes receives the exact size; otherwise *out_bytes is the
 * capacity of `out` on entry and the size written on return (HL_ENOMEM if too
 * small). nthreads 0 = the CPUs of the calling process's affinity mask (at most 64); the
 * output does not depend on nthreads.
 * Errors: HL_EINVAL (shape, seg_len, grp_rows, a weight whose field has no
 * code in `cb`). */
hl_status hl_encode(const uint16_t* w_bf16, uint64_t rows, uint64_t cols,
                    const hl_codebook* cb, uint32_t seg_len, uint32_t grp_rows,
                    uint32_t nthreads, void* out, size_t* out_bytes);

/* Whole-exponent code (format 1) of n bf16 bit patterns: one code over the
 * 256 exponent values (the 8-bit symbols of the split-size analysis,
 * Sec. 3.1), built by the same rules as hl_build_codebook. lmax in [8, 13]
 * (the decode table's 13-bit window then matches every code in one lookup).
 * Errors: HL_EINVAL for n == 0, null pointers or lmax out of range. */
hl_status hl_build_codebook8(const uint16_t* w_bf16, size_t n, uint32_t lmax,
                             hl_codebook8* out);

/* Encode W into an HLF1 container of the whole-exponent format (flags 1).
 * Arguments, size query and errors as hl_encode. */
hl_status hl_encode8(const uint16_t* w_bf16, uint64_t rows, uint64_t cols,
                     const hl_codebook8* cb, uint32_t seg_len, uint32_t grp_rows,
                     uint32_t nthreads, void* out, size_t* out_bytes);

/* Float16 codes (format 2, the paper's {1,5,5,5} split, Sec. 3.1) of n
 * float16 bit patterns: one code per 5-bit field, built by the same rules as
 * hl_build_codebook. lmax in [5, 12]. Errors: HL_EINVAL for n == 0, null
 * pointers or lmax out of range. */
hl_status hl_build_codebook16(const uint16_t* w_f16, size_t n, uint32_t lmax,
                              hl_codebook16* out);

/* Encode a float16 matrix W [rows][cols] into an HLF1 container of the
 * float16 format (flags 2). Arguments, size query and errors as hl_encode. */
hl_status hl_encode16(const uint16_t* w_f16, uint64_t rows, uint64_t cols,
                      const hl_codebook16* cb, uint32_t seg_len, uint32_t grp_rows,
                      uint32_t nthreads, void* out, size_t* out_bytes);

/* Full structural check of a container held in host memory: header, section
 * offsets, codebooks (Kraft sum exactly 1, lengths <= lmax), per-group
 * stream sizes against the stored segment lengths (base + seg_len, each at
 * most S times the longest code of a weight). O(n_seg). Returns HL_OK or
 * HL_ECORRUPT. */
hl_status hl_validate(const void* blob_host, size_t blob_bytes);

/* Build a device view of a container copied to `blob_dev` (blob_bytes long)
 * from its host copy `blob_host` (the same bytes), which is fully validated
 * (as hl_validate, O(n_seg)): the compressed weights stay resident in device
 * memory in this form and are never expanded there (Sec. 1 contributions:
 * weights kept compressed in memory, decompressed only to be multiplied).
 * lut_dev must point to HL_LUT_BYTES of device memory that the view uses
 * from now on. blob_dev and lut_dev must be 16-byte aligned (the kernels
 * copy both in 16-byte pieces). Errors: HL_EINVAL (also for a misaligned
 * pointer), HL_ECORRUPT. */
hl_status hl_tensor_view(const void* blob_dev, const void* blob_host,
                         size_t blob_bytes, uint32_t* lut_dev, hl_tensor* out);

/* Fill t->lut_dev on the device: the joint decode table of the two codes for
 * a 13-bit window (the decoder's L_max-bit window match of Sec. 3.2) and the
 * per-length canonical tables used for pairs longer than the window. In the
 * whole-exponent format the table decodes the one exponent code (never
 * longer than the window) and the per-length tables are zero. */
hl_status hl_tensor_prepare(const hl_tensor* t, void* stream);

/* Device buffers of the calls below (x, decoded weights, workspaces, plain
 * bf16 weights) are read or written in 16-byte pieces and must be 16-byte
 * aligned (any hipMalloc or torch allocation is); float32 outputs must be
 * 4-byte aligned. A misaligned pointer gives HL_EINVAL. */

/* Decode the whole matrix to bf16 bit patterns (float16 for the float16
 * format), out_dev[rows*cols] (row-major): the decoder of Sec. 3.2 (window
 * match, symbol, pointer advance by the code length, concatenation with the
 * raw sign and mantissa) without the product; the layer-wise full
 * decompression the paper contrasts with its own (Sec. 1, Sec. 2.1).
 * Bit-exact with the encoder's input. Errors: HL_EINVAL (also for a
 * misaligned out_dev). */
hl_status hl_decode(const hl_tensor* t, uint16_t* out_dev, void* stream);

/* Bytes of device workspace hl_decode_gemv may use for `t` at this batch
 * (arrival counters, the tiled activations of larger batches and the
 * cross-block partial sums; 0 when it uses none and on bad arguments). */
size_t hl_gemv_workspace_bytes(const hl_tensor* t, uint32_t batch);

/* y[b][r] = sum_k W[r][k] * x[b][k] for b < batch, decoding W on the fly in
 * registers (Sec. 3.2: weights are decompressed only to be multiplied).
 * x_dev: [batch][cols] float32 or bf16; y_dev: [batch][rows] float32 (fully
 * written). fp32 accumulation; every output is summed in a fixed order, so
 * results do not vary between runs. batch in [1, 16].
 * workspace_dev: hl_gemv_workspace_bytes(t, batch) bytes, zero-filled by the
 * caller once before first use; each call leaves it ready for the next, of
 * any batch and on any matrix it is large enough for. Calls
 * that may run concurrently need separate workspaces. With NULL (or too
 * small) the product is still computed, with less parallelism for matrices
 * with few rows. Errors: HL_EINVAL (also for misaligned x, y or workspace). */
hl_status hl_decode_gemv(const hl_tensor* t, const void* x_dev, hl_dtype x_dtype,
                         uint32_t batch, float* y_dev, void* workspace_dev,
                         size_t workspace_bytes, void* stream);

/* hl_decode_gemv without a caller workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, serving loops that
 * forbid allocation): the tiled activations, partial sums and arrival counters
 * go to a scratch array (HL_NOALLOC_SCRATCH_BYTES and 4 KB) that the library holds on each GPU it
 * runs on until the process ends (its address is looked up on the first call
 * on a GPU). No device memory is allocated or freed. The arrival counters a
 * split product uses are zeroed by a small kernel on `stream` before it (no
 * memset). Every call on one GPU shares that GPU's scratch: calls that overlap
 * on one GPU (other streams, other host threads) race and give wrong results.
 * Arguments and results as hl_decode_gemv; the same kernels run, so outputs
 * equal hl_decode_gemv's bit for bit. Errors: those of hl_decode_gemv, and
 * HL_EUNSUPPORTED when the product would need more than
 * HL_NOALLOC_SCRATCH_BYTES of scratch. */
hl_status hl_decode_gemv_noalloc(const hl_tensor* t, const void* x_dev, hl_dtype x_dtype,
                                 uint32_t batch, float* y_dev, void* stream);

/* The products of up to 4 matrices that share x, y_devs[m][b][r] =
 * sum_k W_m[r][k] * x[b][k] (a decode step's q, k and v projections, or its
 * gate and up projections), as hl_decode_gemv computes each. ts[m]: views
 * with the same number of columns. When every matrix is in a bf16 format with
 * 16-row groups and segments of 64 weights, x is bf16 and the
 * matrices have at least one row block per CU together, one launch decodes
 * them all: its blocks are divided among the matrices in proportion to their
 * row blocks, so the launch and first-load latency of small matrices is paid
 * once. Otherwise the matrices are multiplied one after another with
 * hl_decode_gemv. workspace_dev: at least the largest
 * hl_gemv_workspace_bytes(ts[m], batch), under hl_decode_gemv's rules.
 * Errors: HL_EINVAL (also for matrices with different column counts), and
 * those of hl_decode_gemv. */
hl_status hl_decode_gemv_multi(const hl_tensor* const* ts, uint32_t count, const void* x_dev,
                               hl_dtype x_dtype, uint32_t batch, float* const* y_devs,
                               void* workspace_dev, size_t workspace_bytes, void* stream);

/* Bytes of device workspace hl_decode_gemm needs for `tokens` activation rows:
 * up to 64 tokens the partial sums of up to one range per column block of
 * four segments (on the persistent kernel's matrices, up to 64 tokens, only
 * the tiled activations use it), beyond that the decoded weights
 * (rows * cols * 2); 0 for tensors it does not take. */
size_t hl_gemm_workspace_bytes(const hl_tensor* t, uint32_t tokens);

/* Prefill product Y[n][r] = sum_k W[r][k] * X[n][k] for n < tokens (many
 * activation rows; the paper's prompts of tens of tokens, Sec. 4). Up to 64
 * tokens on matrices with at least one 16-row block per compute unit, the
 * persistent fused decode-GEMV multiplies each decoded 8-weight step with
 * one, two or four 16-token tiles (the activations first copied to the
 * workspace in chunks of 16 rows per tile; four tiles for S = 64 and stream
 * columns of 16 words or more); otherwise, up to 64 tokens, each 16-row x 4-segment
 * weight tile is decoded once per chunk of up to 128 tokens and multiplied
 * with all of them on the matrix cores (Sec. 3.2: weights decompressed only
 * to be multiplied). Beyond that, where the product is compute-bound (Sec. 5),
 * the matrix is decoded once into the workspace (hl_decode) and multiplied by
 * hipBLASLt; where that has no algorithm without a workspace of its own (few
 * output tiles and long sums), by the fused kernel, or, with segments too long
 * for it, by hl_gemv_bf16 in batches of 16 tokens. Every output of the fused
 * kernels is summed in a fixed order. x_dev: [tokens][cols] bf16; y_dev: [tokens][rows] float32 (fully
 * written); fp32 accumulation. bf16 formats (split or whole exponent) with
 * 16-row groups and S = 32 or 64; others give HL_EUNSUPPORTED.
 * workspace_dev: hl_gemm_workspace_bytes(t, tokens) bytes (no initial
 * contents needed); calls that may run concurrently need separate
 * workspaces. Errors: HL_EINVAL (also for a missing or short workspace). */
hl_status hl_decode_gemm(const hl_tensor* t, const void* x_dev, hl_dtype x_dtype, uint32_t tokens,
                         float* y_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Uncompressed comparator: the same product from plain bf16 W [rows][cols]
 * in device memory. */
hl_status hl_gemv_bf16(const uint16_t* w_dev, uint64_t rows, uint64_t cols,
                       const void* x_dev, hl_dtype x_dtype, uint32_t batch,
                       float* y_dev, void* stream);

/* ---------------------------------------------------------------------------
 * Between the products of a decoder layer: norm, attention and its cache.
 * The paper's layers (Sec. 2.1) are their products; these operators are what a
 * decode step over compressed weights needs besides. They take and give plain
 * tensors, in the activation types of the products above.
 * ------------------------------------------------------------------------- */

/* RMS norm with the residual's addition, of `tokens` rows of `hidden` columns
 * (row-major, contiguous):
 *   t = x + residual,  sum = t,  out = t / sqrt(mean(t^2) + eps) * weight.
 * x, residual, weight: float32, bf16 or float16, each its own type; t is held
 * in float32, and `sum` (of residual's type) is its only rounding: the norm is
 * of the unrounded sum. residual_dev NULL: t = x, and sum_dev is not written
 * (r_dtype is ignored). sum_dev may be residual_dev, and x_dev or residual_dev
 * may be out_dev where the two have one type.
 * out_dtype: float32, bf16, float16, or HL_E4M3 with float32 scales: the
 * columns of a group share scale = max|out| / 448 (1 where that is below the
 * least normal float32, as for a group of zeros), and out holds out / scale
 * (the float32 quotient) rounded to nearest, ties to even. group: 32, 64 or 128
 * columns (dividing hidden; scale_dev [tokens][hidden/group]), or 0 for the whole
 * row (scale_dev [tokens][1]). For other out types group must be 0 and scale_dev
 * is ignored.
 * A NaN in a row makes the row's out NaN.
 * Pointers are aligned to their elements, with a group to 16 bytes; hidden may
 * be any number. Errors: HL_EINVAL (also for a misaligned pointer),
 * HL_EUNSUPPORTED for hidden above HL_NORM_MAX_HIDDEN and for more rows than a
 * launch takes (2^23 of 4096 columns). */
hl_status hl_rms_norm(const void* x_dev, hl_dtype x_dtype, const void* residual_dev, hl_dtype r_dtype,
                      const void* weight_dev, hl_dtype w_dtype, uint64_t tokens, uint64_t hidden, float eps,
                      void* sum_dev, void* out_dev, hl_dtype out_dtype, uint32_t group, float* scale_dev,
                      void* stream);

/* Keys and values [sequence][token][key head][column] in device memory, by
 * strides in elements (of 16 bits): any order of the first three, columns next
 * to each other. Pointers 16-byte aligned, strides multiples of 8. */
typedef struct {
  const void* k_dev;
  const void* v_dev;
  uint64_t tokens;   /* capacity of a sequence (of a prefix: its length); 0: there is none */
  uint64_t k_seq, k_token, k_head;
  uint64_t v_seq, v_token, v_head;
} hl_kv;

/* An attention call's shape: `batch` sequences with `queries` new tokens each,
 * `heads` query heads of `dim` columns, heads / kv_heads of which share a key
 * head (heads % kv_heads == 0; dim a multiple of 8, at most
 * HL_ATTENTION_MAX_DIM). */
typedef struct {
  hl_dtype dtype;    /* of q, keys, values and out: HL_BF16 or HL_F16 */
  uint32_t batch, queries, heads, kv_heads, dim;
  float scale;       /* of the scores (1/sqrt(dim) as a rule) */
  hl_kv prefix;      /* shared by all sequences: its k_seq and v_seq are ignored */
  hl_kv own;         /* each sequence's own, at the first lens[b] tokens of its capacity */
} hl_attention;

/* Bytes of device workspace hl_prefix_attention needs on the current GPU, never
 * 0 but on bad arguments. */
size_t hl_attention_workspace_bytes(const hl_attention* attention, int with_weights);

/* Attention of each sequence's new tokens over a prefix that all sequences
 * share and over its own cache, which already holds the new tokens' keys and
 * values at its end. The prefix is read once for the whole batch.
 *   s_j = scale * q . k_j,  out = sum_j p_j v_j,  p = softmax(s)
 * over all keys of the prefix and, for token i of `queries`, the own keys
 * j < lens[b] - (queries - 1 - i). A token that sees no key (or only scores of
 * minus infinity) has out = 0 and lse = minus infinity. Keys and values that a
 * token does not see do not affect it, whatever they hold; an infinite or NaN
 * value that it sees leaves its column of out infinite or NaN, however small the
 * weight.
 * q_dev, out_dev: [batch][queries][heads][dim]. lens_dev: int32 [batch], read
 * on the device (a length above own.tokens counts as own.tokens, a negative
 * one as 0); NULL only where own.tokens == 0. lse_dev (or NULL): float32
 * [batch][queries][heads], log(sum_j exp(s_j)).
 * weight_out_dev (or NULL): float32 [batch][kv_heads][own.tokens], what
 * eviction goes by (own.tokens is not 0 then): weight_in_dev (NULL: zeros; may
 * be the same buffer) plus,
 * for every own key, the sum of its p over the call's tokens and the heads
 * that share it. It holds a float32 score for each (row, own key) in the
 * workspace, so it is meant for few new tokens.
 * Scores, softmax statistics and sums are float32; p is rounded to the 16-bit
 * type for the second product. Every sum has a fixed order.
 * workspace_dev: hl_attention_workspace_bytes (16-byte aligned, no initial
 * contents needed); calls that may run concurrently need separate ones.
 * Errors: HL_EINVAL (also for a missing or short workspace), HL_EUNSUPPORTED
 * for dim above HL_ATTENTION_MAX_DIM and sizes past the kernels' 32-bit
 * counts. */
hl_status hl_prefix_attention(const hl_attention* attention, const void* q_dev, const int32_t* lens_dev,
                              void* out_dev, float* lse_dev, const float* weight_in_dev, float* weight_out_dev,
                              void* workspace_dev, size_t workspace_bytes, void* stream);

/* Eviction from a cache by accumulated attention weight: of every sequence and
 * key head at most `keep` tokens stay, moved in their order to the first slots
 * of another cache. With n = lens[b] (bounded as in hl_prefix_attention): all
 * tokens where n <= keep; else the newest `recent` (recent <= keep) and, of
 * the others, the keep - recent of greatest weight; of equal ones the lowest
 * slot, NaN below every number.
 * from, to: caches of `batch` sequences, kv_heads and dim (a multiple of 8),
 * that do not overlap; to->tokens >= keep. weight_dev: float32
 * [batch][kv_heads][from->tokens]. Written: the first `keep` tokens of `to`
 * (zeros past the kept ones), weight_out_dev float32 and slots_dev int32
 * [batch][kv_heads][keep] (the kept tokens' weights and their slots in `from`;
 * 0 and -1 past them), lens_out_dev int32 [batch] (min(n, keep)). Any 16-bit
 * type. Errors: HL_EINVAL, HL_EUNSUPPORTED for sizes past 32-bit counts. */
hl_status hl_cache_evict(const hl_kv* from, const hl_kv* to, uint32_t batch, uint32_t kv_heads, uint32_t dim,
                         const float* weight_dev, const int32_t* lens_dev, uint64_t keep, uint64_t recent,
                         float* weight_out_dev, int32_t* slots_dev, int32_t* lens_out_dev, void* stream);

/* ---------------------------------------------------------------------------
 * A cache in 4 bits, and what else a decode step takes in 4 bits or ends in.
 * ------------------------------------------------------------------------- */

/* Bytes of a row of a 4-bit cache: `dim` columns of one token and key head, in
 * G = dim / 32 groups of neighbouring columns that share a scale and a base,
 *   value = base + scale * (code - 8),  code 0 .. 15:
 *   16 * G bytes of codes: byte n * G + g has the codes of columns 32g + 2n (its
 *   low half) and 32g + 2n + 1, n = 0 .. 15;
 *   G pairs (scale, base), each bf16, the scale first;
 *   zeros up to a multiple of 16 bytes.
 * 0 where dim is not a multiple of 32, or above HL_ATTENTION_MAX_DIM. */
size_t hl_cache4_row_bytes(uint32_t dim);

/* Caches of such rows are hl_kv like those in 16 bits, with strides in units of
 * 16 bits (multiples of 8), so hl_cache_evict moves them too (as rows of
 * hl_cache4_row_bytes(dim) / 2 columns). */

/* Rounds new tokens' keys and values to 4-bit rows. from: [sequence][token][key
 * head][column] of bf16 or float16, from->tokens new ones a sequence. They go to
 * the slots that end at the sequence's length, lens[b] - from->tokens + i for
 * token i (lens_dev NULL: to slots 0 .. from->tokens - 1); those without a slot in
 * the cache are left out, and other slots are not written.
 * Of 32 columns from lo to hi:
 *   base = (7 lo + 8 hi) / 15, scale = max((hi - base) / 7, (base - lo) / 8),
 * computed in float32 (a rounding each operation) and rounded to bf16, and code - 8
 * is the whole number of -8 .. 7 nearest to (x - base) / scale, ties to even (0
 * where scale is 0). Columns among which one is an infinity or a NaN, or whose base
 * or scale would not be finite, become NaN, all 32. Errors: HL_EINVAL,
 * HL_EUNSUPPORTED for dim above HL_ATTENTION_MAX_DIM and sizes past 32-bit counts. */
hl_status hl_cache_write4(const hl_kv* from, hl_dtype dtype, const hl_kv* cache, uint32_t batch, uint32_t kv_heads,
                          uint32_t dim, const int32_t* lens_dev, void* stream);

/* The values that 4-bit rows stand for, to out [batch][tokens][heads][dim] of
 * float32, bf16 or float16: base + scale * (code - 8) in float32, rounded once
 * more for 16 bits. Strides in bytes, multiples of 16; both pointers 16-byte
 * aligned. Errors as hl_cache_write4. */
hl_status hl_cache_read4(const void* rows_dev, uint64_t seq_stride, uint64_t token_stride, uint64_t head_stride,
                         uint32_t batch, uint64_t tokens, uint32_t heads, uint32_t dim, void* out_dev, hl_dtype dtype,
                         void* stream);

/* hl_prefix_attention over a prefix and own caches of 4-bit rows; its workspace.
 * `dtype` is q's and out's; dim is a multiple of 32. What rows stand for enters the
 * sums unrounded; p and p * scale are rounded to bf16 for the second product, to two
 * bf16 pieces where out is float16. A column group of a token that a row sees is NaN
 * in out where its scale or base is; of tokens that it does not see, rows may hold
 * anything. Any strides are taken; rows are shorter than a line of memory, so long
 * caches are read faster where a key head's tokens lie next to each other. Everything
 * else, weights and errors among it, as hl_prefix_attention. */
size_t hl_attention4_workspace_bytes(const hl_attention* attention, int with_weights);
hl_status hl_prefix_attention4(const hl_attention* attention, const void* q_dev, const int32_t* lens_dev,
                               void* out_dev, float* lse_dev, const float* weight_in_dev, float* weight_out_dev,
                               void* workspace_dev, size_t workspace_bytes, void* stream);

/* The product of a layer whose weights are kept in 4 bits,
 *   y[b][r] = sum_k x[b][k] * (base + scale * (code[r][k] - 8)),
 * for b < batch, batch in [1, HL_MAX_BATCH]. codes_dev: [rows][cols / 2], the
 * code of an even column in the low half of a byte, of the next one in the high
 * half. scales_dev, bases_dev: bf16 or float16 [rows][cols / group], one for each
 * `group` neighbouring columns: 32, 64 or 128, dividing cols; bases_dev NULL: all 0.
 * x_dev: [batch][cols] bf16 or float16; y_dev: [batch][rows] float32 (fully
 * written). The codes (as 16 + code, less 24) multiply x exactly and sums are float32,
 * in a fixed order; scales and bases multiply a group's sums in float32. A row with an
 * infinite or NaN scale or base has no finite y, nor has a row of x with an infinity or
 * a NaN (NaN, too, where the definition is infinite); x above 2^115 may have none,
 * where 55 times the sum of a group's |x| is not finite. codes_dev and x_dev are 16-byte aligned, the
 * others 4-byte. Errors: HL_EINVAL (also for a misaligned pointer),
 * HL_EUNSUPPORTED for cols of 2^24 and above and rows past 32-bit counts. */
hl_status hl_gemv4(const uint8_t* codes_dev, const void* scales_dev, const void* bases_dev, hl_dtype scale_dtype,
                   uint64_t rows, uint64_t cols, uint32_t group, const void* x_dev, hl_dtype x_dtype, uint32_t batch,
                   float* y_dev, void* stream);

/* How a row's token is drawn; each setting for all rows, or, where its pointer is
 * not NULL, of each row in device memory (float32 or int32 [rows]). */
typedef struct {
  const float* temperature_dev;
  const int32_t* top_k_dev;
  const float* top_p_dev;
  const float* min_p_dev;
  float temperature; /* not above 0: the greatest logit's token */
  int32_t top_k;     /* below 1, or vocab and above: all */
  float top_p;       /* 1 and above: all */
  float min_p;       /* 0 and below: all */
} hl_sampling;

/* A token of each row of logits: with w_i = exp((l_i - max l) / temperature) and
 * the tokens in the order of falling logits, of equal ones the lowest index first,
 *   of these the first top_k are kept;
 *   of these the first ones up to that at which the sum of w reaches top_p of the
 *   sum over all that top_k kept;
 *   of these the ones with w >= min_p (at least the first token);
 * the token is the lowest index i at which the sum of the kept w over 0 .. i is above
 * u times their total, u = uniforms[row] in [0, 1) (0 for a lower one or a NaN; for 1
 * and above the last kept token). Tokens whose w is below 2^-40 are never drawn and
 * count nowhere. A row is many times slower where top_k or top_p ends among more than
 * 2048 logits of a thousandth of the distance that weighs (equal ones). logprobs: log
 * of the token's w over the kept total. A logit that is NaN counts as minus infinity;
 * where the greatest is plus infinity, those that are have w = 1 and the others 0. A
 * row with nothing above minus infinity has token -1 and logprob minus infinity. Each
 * w is held to 2^-43 of the greatest (not of itself), and sums of what is held are
 * exact: a sum over n tokens is off by n * 2^-43 of the greatest at most. The token is
 * that of exact numbers but where u times the total (top_p times it) is within n *
 * 2^-42 of where another token begins. logits_dev: [rows][vocab] float32, bf16 or
 * float16, rows row_stride elements apart, aligned to their elements. tokens_dev
 * int32, logprobs_dev float32 [rows]. workspace_dev: hl_sample_workspace_bytes
 * (16-byte aligned, no initial contents needed; 0 on bad arguments; 15 to 31 KB a row
 * and 10 for each 2048 to 16384 of its logits, 174 MB at most: further rows go after
 * each other); calls that may run concurrently need separate ones. Errors: HL_EINVAL
 * (also for a missing or short workspace), HL_EUNSUPPORTED for vocab of 2^20 and above
 * and more than 65535 rows. */
size_t hl_sample_workspace_bytes(uint32_t rows, uint64_t vocab);
hl_status hl_sample(const hl_sampling* sampling, const void* logits_dev, hl_dtype dtype, uint64_t row_stride,
                    uint32_t rows, uint64_t vocab, const float* uniforms_dev, int32_t* tokens_dev, float* logprobs_dev,
                    void* workspace_dev, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HUFFLM_H */
