/*
 * ozk — FP64 GEMM emulated on NVIDIA B200 FP4 tensor cores by Ozaki scheme II on
 * base-13 E2M1 limbs, and bit-exact INT8 GEMM on the same limbs.
 *
 * C ABI.  Every matrix pointer is a DEVICE pointer owned by the caller; matrices are
 * column-major (element (r,c) at ptr[r + c*ld]).  `stream` is a cudaStream_t passed as
 * void* (NULL = the legacy default stream).  Compute calls enqueue work on `stream` and
 * return without synchronising; they allocate no memory.  All scratch lives in ONE
 * caller-owned device workspace registered with ozk_set_workspace(); calls that share
 * the workspace must be ordered by the caller (same stream, or events).
 *
 * Errors.  Argument errors are returned synchronously and enqueue nothing.
 * Data-dependent conditions (a NaN/Inf input, a bounded device wait that expired) are
 * recorded in a status word inside the workspace and reported by
 * ozk_get_async_status(), which synchronises the stream.  After OZK_ERR_NONFINITE or
 * OZK_ERR_DEVICE_TIMEOUT the output matrix is unspecified.
 */
#ifndef OZK_H_
#define OZK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int ozk_status;
enum {
  OZK_OK = 0,
  OZK_ERR_INVALID_ARG = -1,    /* null pointer, negative size, ld too small, bad alignment */
  OZK_ERR_UNSUPPORTED = -2,    /* num_moduli out of range, K beyond an exactness bound, device is not sm_100 */
  OZK_ERR_WORKSPACE = -3,      /* no workspace registered, or it is too small for this call */
  OZK_ERR_CUDA = -4,           /* a CUDA runtime/driver call failed (launch, tensor-map encode) */
  OZK_ERR_NONFINITE = -5,      /* asynchronous: an input element is NaN or Inf */
  OZK_ERR_DEVICE_TIMEOUT = -6  /* asynchronous: a bounded wait inside a kernel gave up */
};

enum { OZK_MIN_MODULI = 2, OZK_MAX_MODULI = 27, OZK_DEFAULT_MODULI = 19 };
/* Longest k range of one limb-GEMM launch, and the largest K ozk_dgemm accepts (16 ranges). */
enum { OZK_CHUNK_K = 131072, OZK_MAX_K = 2097152 };

/* ---------------------------------------------------------------------------------------
 * Constants of the method (host-side, no GPU needed).
 * ------------------------------------------------------------------------------------- */

/* Section 5.1: the first `num_moduli` moduli chosen greedily in descending order from 169,
 * pairwise coprime, 169 the only multiple of 13, every residue class representable by two
 * limbs c0 + 13 c1 with c0, c1 in S = {0,+-1,+-2,+-3,+-4,+-6,+-8,+-12}.  The first 19 are the
 * list printed in the paper; 20..27 continue the same rule.  Writes num_moduli ints to
 * `out` (host memory); returns num_moduli, or OZK_ERR_INVALID_ARG. */
int ozk_get_moduli(int num_moduli, int* out);

/* Eq. 3 read for a general integer width: the largest c <= 53 with 2*K*2^(2c) < P, P the
 * product of the first num_moduli moduli.  Inputs are converted to integers of at most c
 * bits (Section 4.2).  Returns c >= 1, or OZK_ERR_UNSUPPORTED when no c >= 1 exists, or
 * OZK_ERR_INVALID_ARG. */
int ozk_capacity_bits(int64_t K, int num_moduli);

/* Section 5.2: the CRT constants for the first num_moduli moduli as little-endian 32-bit
 * words, 6 words each: P into P_words[6], w_l = (P/m_l) * ((P/m_l)^-1 mod m_l) into
 * weights[6*l .. 6*l+5] (host memory).  Returns OZK_OK or OZK_ERR_INVALID_ARG. */
ozk_status ozk_get_crt_constants(int num_moduli, uint32_t* P_words, uint32_t* weights);

const char* ozk_status_string(ozk_status status);
const char* ozk_version(void);

/* ---------------------------------------------------------------------------------------
 * Workspace.
 * ------------------------------------------------------------------------------------- */

/* Bytes of device workspace ozk_dgemm(M,N,K,...,num_moduli) needs: status block, limb-pair
 * tables, shifts s (rows of A) and t (columns of B), 2*num_moduli E2M1 limb planes per
 * operand padded to 128 rows x 256 k, and num_moduli residue matrices of one byte per
 * element of the padded C.  For 0 < K <= 1792 with N padding to a multiple of 256 the A side
 * holds two more planes per modulus (the limbs of 13 a mod m, see the two-accumulator form
 * under ozk_stage_residue_gemm); with the Karatsuba variant on, one sum-limb plane per Karatsuba
 * modulus and operand.  The size is therefore not monotonic in K (K = 1792 needs more than K = 2048): a caller that
 * reuses one workspace for several shapes registers the largest of their sizes.  Returns 0 on invalid arguments. */
size_t ozk_dgemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int num_moduli);

/* Bytes of device workspace ozk_igemm_i8(M,N,K,...) needs (3 limb planes per operand). */
size_t ozk_igemm_i8_workspace_bytes(int64_t M, int64_t N, int64_t K);

/* Registers the caller-owned device buffer used by all later compute calls of this
 * process.  `dev_ptr` must be 256-byte aligned (any cudaMalloc / PyTorch allocation is).
 * The library never frees it.  Passing NULL unregisters. */
ozk_status ozk_set_workspace(void* dev_ptr, size_t bytes);

/* Synchronises `stream`, then reads and clears the status word in the workspace.
 * Returns OZK_OK, OZK_ERR_NONFINITE, OZK_ERR_DEVICE_TIMEOUT, OZK_ERR_WORKSPACE or OZK_ERR_CUDA. */
ozk_status ozk_get_async_status(void* stream);

/* ---------------------------------------------------------------------------------------
 * The hot path.
 * ------------------------------------------------------------------------------------- */

/* Emulated DGEMM, C = A*B with every C_ij the exact product of the integer-converted
 * inputs rounded once (Sections 4.2, 5; Fig. 3): shared-exponent conversion of the rows
 * of A and columns of B to integers of ozk_capacity_bits(K, num_moduli) bits, residues
 * mod each modulus as two base-13 E2M1 limbs, four FP4 limb products per modulus on the
 * tensor cores with the residue composed in the epilogue, single-pass integer CRT,
 * inverse scaling, one round-to-nearest-even.
 *   A: M x K, lda >= max(1,M).  B: K x N, ldb >= max(1,K).  C: M x N, ldc >= max(1,M), overwritten.
 *   num_moduli in [OZK_MIN_MODULI, OZK_MAX_MODULI]; 19 keeps all 53 bits for K <= 76549.
 *   One limb-GEMM launch covers at most 131072 values of k (FP32 accumulators stay exact
 *   integers: 128*K <= 2^24 with limbs |c| <= 8; Lemma 3 bounds K by 58254 for limbs up to 12).
 *   EXTENSION, not in the paper (which never splits K): a longer K is cut into such ranges, one
 *   limb-GEMM launch each, and the residues of the ranges are added modulo each modulus (the
 *   residue of a sum is the sum of the residues), up to OZK_MAX_K.  The capacity of
 *   ozk_capacity_bits(K, ...) always refers to the whole K.  M, N, K = 0 are allowed (K = 0
 *   gives C = 0).  M and N are otherwise limited only by the workspace.
 *   The library keeps per-device launch state keyed by the device ordinal, so one process may
 *   use several devices (each call acts on the current device, to which `stream` and all
 *   pointers must belong); the registered workspace and the stage timing are one per process,
 *   and calls from several host threads must be serialised by the caller.
 * Returns OZK_OK once the work is enqueued.  The call only enqueues kernels and memsets on
 * `stream` (no allocation, no synchronisation), so after one eager call, which sets the
 * kernels' attributes, it may be captured into a CUDA graph and replayed. */
ozk_status ozk_dgemm(int64_t M, int64_t N, int64_t K,
                     const double* A, int64_t lda,
                     const double* B, int64_t ldb,
                     double* C, int64_t ldc,
                     int num_moduli, void* stream);

/* EXTENSION, not in the paper: ozk_dgemm with the 53-bit cap on the converted integers
 * (Section 4.2) lifted to max_bits, 1 <= max_bits <= OZK_MAX_EXTENDED_BITS.  Every step is the
 * paper's; only the width is c = min(max_bits, largest c with 2 K 2^(2c) < P) (Eq. 3), so
 * with more than 19 moduli the row / column maximum converts without rounding and smaller
 * entries keep up to max_bits - 53 more bits below it (converted integers are held in 64-bit
 * words).  max_bits = 53 is ozk_dgemm itself.  Same arguments, workspace
 * (ozk_dgemm_workspace_bytes), layout, asynchrony and error behaviour as ozk_dgemm;
 * max_bits out of range -> OZK_ERR_INVALID_ARG.  ozk_capacity_bits_ext returns the width used. */
enum { OZK_MAX_EXTENDED_BITS = 62 };
int ozk_capacity_bits_ext(int64_t K, int num_moduli, int max_bits);
ozk_status ozk_dgemm_ext(int64_t M, int64_t N, int64_t K,
                         const double* A, int64_t lda,
                         const double* B, int64_t ldb,
                         double* C, int64_t ldc,
                         int num_moduli, int max_bits, void* stream);

/* Bit-exact INT8 x INT8 -> INT32 GEMM on FP4 tensor cores (Section 3, last paragraph;
 * Eq. 1 with p = q = 3): every int8 becomes three greedy base-13 limbs, nine limb
 * products are accumulated in five groups i+j = g and combined as sum_g 13^g G_g.
 *   A: M x K int8, B: K x N int8, C: M x N int32, column-major as above.
 *   K <= 87381 (three products of magnitude <= 64 share an FP32 accumulator:
 *   192*K <= 2^24); the int32 result is exact for K <= 131071 anyway. */
ozk_status ozk_igemm_i8(int64_t M, int64_t N, int64_t K,
                        const int8_t* A, int64_t lda,
                        const int8_t* B, int64_t ldb,
                        int32_t* C, int64_t ldc, void* stream);

/* ozk_dgemm for matrices in HOST memory (pinned memory for full speed): same result, same
 * arguments, but A, B and C are host pointers.  C is produced in blocks of 2048 x 2048 (larger
 * when a dimension exceeds 131072); the host-to-device copies of the column blocks of B and the
 * row blocks of A (sent alternately), the three stages, and the device-to-host copies of the
 * finished blocks of C run on three streams and overlap: a block of C is computed as soon as
 * its row block and its column block have arrived (the paper times device-resident data only,
 * Section 6.1).  The call returns once everything is enqueued; `stream` completes when C has
 * arrived in host memory.  The workspace holds the limb planes of A and B, one block of
 * residues, and two staging blocks each for A, B and C.  The first call creates two internal
 * streams and a pool of events.  K <= OZK_CHUNK_K here (OZK_ERR_UNSUPPORTED beyond). */
size_t ozk_dgemm_host_workspace_bytes(int64_t M, int64_t N, int64_t K, int num_moduli);
ozk_status ozk_dgemm_host(int64_t M, int64_t N, int64_t K,
                          const double* A, int64_t lda,
                          const double* B, int64_t ldb,
                          double* C, int64_t ldc,
                          int num_moduli, void* stream);

/* Emulated DGEMM by Ozaki scheme I on the same limbs (Section 4; Fig. 2; Eq. 1; Lemma 2): the
 * integer-converted inputs (c = 53 bits, Section 4.2) are decomposed into p = q = 15 greedy base-13
 * E2M1 limbs, the limb products are aggregated along the anti-diagonals i + j = g, weighted by 13^g
 * in multiword integers, scaled back and rounded once.  The result equals ozk_dgemm with 19 moduli
 * bit for bit (both are the exact product of the same converted integers rounded once, Section 7.1).
 * Arguments and layout as ozk_dgemm.  K <= 87381 (three products of magnitude <= 64 share an FP32
 * accumulator).  Workspace: 15 + 16 limb planes and 20 int64 block values per element of C. */
size_t ozk_dgemm_oz1_workspace_bytes(int64_t M, int64_t N, int64_t K);
ozk_status ozk_dgemm_oz1(int64_t M, int64_t N, int64_t K,
                         const double* A, int64_t lda,
                         const double* B, int64_t ldb,
                         double* C, int64_t ldc, void* stream);

/* ---------------------------------------------------------------------------------------
 * Staged entry points: the same kernels one stage at a time, used by the parity tests.
 * They use the registered workspace exactly as ozk_dgemm does.
 * ------------------------------------------------------------------------------------- */

/* Stage 1 (Section 4.2 + Section 5.1): exponent scan, integer conversion, residues,
 * limb planes.  Optional device outputs (NULL to skip):
 *   s_out[M], t_out[N]          the shifts s_i, t_j (int32)
 *   At_out[M*K], Bt_out[K*N]    the converted integers, column-major with ld = M and K (int64)
 * The limb planes stay in the workspace; ozk_stage_read_planes() copies them out. */
ozk_status ozk_stage_preprocess(int64_t M, int64_t N, int64_t K,
                                const double* A, int64_t lda, const double* B, int64_t ldb,
                                int num_moduli, int32_t* s_out, int32_t* t_out,
                                int64_t* At_out, int64_t* Bt_out, void* stream);

/* Decodes limb plane (modulus index l, limb 0|1) of operand 'A' or 'B' from the workspace
 * into doubled-E2M1 integers (int8, values in S): out[r + k*rows], r < rows (M for 'A',
 * N for 'B'), k < K.  Valid after ozk_stage_preprocess / ozk_dgemm on the same sizes.
 * limb = 2 reads the sum-limb plane of a Karatsuba modulus (variant on, see ozk_stage_set_karatsuba).
 * limb = 3 | 4 (operand 'A' only, sizes that take the two-accumulator form) reads limb 0 | 1 of
 * (13 a) mod m_l, the planes that form multiplies by the high limbs of B. */
ozk_status ozk_stage_read_planes(char operand, int64_t M, int64_t N, int64_t K, int num_moduli,
                                 int l, int limb, int8_t* out, void* stream);

/* Stage 2 (Section 5.1, Section 6.4): the limb GEMM with residue composition, on the
 * planes in the workspace.  residues_out (optional, device): num_moduli matrices of
 * M x N bytes, column-major with ld = M, r_l = (A~ B~) mod m_l in [0, m_l).
 * Two forms of the same residues (bit for bit).  Regular: b = b0 + 13 b1, a = a0 + 13 a1,
 * three accumulators a0 b0, a0 b1 + a1 b0, a1 b1 per tile of C.  Two-accumulator form, taken
 * for 0 < K <= 1792 when N pads to a multiple of 256: a b = b0 beta + b1 gamma (mod m) with
 * beta = a mod m and gamma = 13 a mod m, both as limb pairs, so that only the accumulators
 * b0 beta_0 + b1 gamma_0 and b0 beta_1 + b1 gamma_1 exist and two tiles of C fit tensor memory
 * at once: the read-back of one overlaps the products of the next (faster at short K, level
 * with the regular form at K = 2048 and slower beyond, because the A side moves twice the planes).  OZK_GEMM_GAMMA=0 in the
 * environment keeps the regular form at every K (measurement aid, read once per process). */
ozk_status ozk_stage_residue_gemm(int64_t M, int64_t N, int64_t K, int num_moduli,
                                  uint8_t* residues_out, void* stream);

/* Stage 3 (Section 5.2 + Section 4.2): direct CRT, symmetric representative, inverse
 * scaling, one rounding.  residues_in (optional, device; same layout as residues_out): if
 * given together with s_in[M], t_in[N], the stage runs on them instead of the workspace
 * contents.  x_out (optional, device): the reconstructed integer of every element as
 * 6 little-endian 32-bit words, two's complement, element (i,j) at x_out[6*(i + j*M)]. */
ozk_status ozk_stage_crt(int64_t M, int64_t N, int64_t K, int num_moduli,
                         const uint8_t* residues_in, const int32_t* s_in, const int32_t* t_in,
                         double* C, int64_t ldc, uint32_t* x_out, void* stream);

/* The paper has no counterpart to this entry point.  It is for callers that cannot allocate
 * device memory and so cannot provide the workspace the calls above need: code running under a
 * framework whose allocator owns all device memory and forbids raw cudaMalloc (which synchronises
 * the device), plug-ins inside latency-critical loops, processes that have no free memory left.
 * It computes what stage 1 computes first, the row shifts s_i = c - 1 - e_i of A
 * (c = ozk_capacity_bits(K, num_moduli), Section 4.2), and keeps its only scratch, one 64-bit
 * maximum per row, in a fixed array inside the library image: OZK_NOALLOC_MAX_ROWS rows,
 * 512 KiB, resident on every GPU that loads the library until the process exits.  This call and
 * everything it calls neither allocate nor free memory; the array itself is set up by the CUDA
 * driver when it loads the library's device code, which with lazy loading can be as late as the
 * first call on a device: make that call at start-up (a process with no free device memory gets
 * OZK_ERR_CUDA from it), as advised for stream capture below.  `stream` must belong to the
 * current device.
 *   A: M x K column-major FP64 (device), lda >= M.  s_out: M int32 (device).  An all-zero row
 *   gets 0; a row containing NaN or Inf gets INT32_MIN (there is no status word to report it).
 *   M > OZK_NOALLOC_MAX_ROWS, or K beyond the limits of ozk_dgemm -> OZK_ERR_UNSUPPORTED.
 * The first call on each device looks up the device address of the array (with that device
 * current); make that first call before starting any stream capture.  Every call uses the same
 * array and finds the previous call's contents in it: the rows it needs are cleared on `stream`
 * first, and two calls whose work overlaps on the GPU (different streams, no ordering) race. */
enum { OZK_NOALLOC_MAX_ROWS = 65536 };
ozk_status ozk_row_shifts_noalloc(int64_t M, int64_t K, const double* A, int64_t lda, int num_moduli,
                                  int32_t* s_out, void* stream);

/* Measurement aid (the paper times its stages with CUDA events, Section 6.1): when enabled,
 * ozk_dgemm records four CUDA events on its stream, before stage 1 and after each of the three
 * stages.  Enabling creates the events (a host-side allocation; do it outside timed regions).
 * ozk_stage_timing_read() synchronises on those events and writes the milliseconds of
 * preprocessing, limb GEMM and reconstruction to ms3[0..2] (host), averaged over the ozk_dgemm
 * calls made since enabling or since the previous read (the most recent 64 of them), so that a
 * timed loop need not synchronise between its calls.  No call since then -> OZK_ERR_INVALID_ARG. */
ozk_status ozk_stage_timing_enable(int enable);
ozk_status ozk_stage_timing_read(float* ms3);

/* Variant switch (process-wide, off by default): partial Karatsuba for the moduli whose residue classes all
 * have a limb pair (c0, c1) with c0 + c1 again a doubled E2M1 value: 83, 73, 71, 67, 61, 59, 53 among the
 * first 19 (Section 5.1, last paragraph; Section 6.4).  When on, the encoder writes a third plane of sum limbs
 * for those moduli and the CTA-pair limb GEMM forms a0 b0, a1 b1 and (a0 + a1)(b0 + b1) instead of the four
 * products (68 instead of 75 products at 19 moduli); the residues, hence C, are the same bit for bit.  Sum
 * limbs reach 12, so a limb-GEMM launch covers at most 65536 values of k (144 K <= 2^24, Lemma 3).  The
 * workspace grows by the sum-limb planes: query ozk_dgemm_workspace_bytes after switching.  The paper found
 * the variant slower under kernel fusion; so does this build (measurements in profiles/). */
ozk_status ozk_stage_set_karatsuba(int enable);

/* Measurement aid: while stage timing is enabled, the thread that issues the tensor-core
 * instructions of the limb GEMM's first CTA pair counts its clocks (clock64): clk3[0] the whole
 * kernel, clk3[1] waiting for tensor memory to be drained by the epilogue, clk3[2] waiting for
 * operand stages from the TMA producer; the rest it spent issuing.  Reads the counters the most
 * recent limb-GEMM launch left in the workspace (synchronise its stream first); host pointer. */
ozk_status ozk_stage_gemm_cycles(long long* clk3);

/* One tcgen05.mma.kind::mxf4.block_scale instruction sequence on caller-supplied packed
 * E2M1 operands, used to pin the hardware byte formats (nibble order, E2M1 codes, UE8M0
 * scale byte, FP32 accumulator exactness): D[128 x 128] (FP32, row-major, device) =
 * scale^2 * sum_k P[r,k] Q[c,k], P and Q being 128 x K nibbles, K-contiguous, two per byte,
 * K a multiple of 256.  scale_byte is the UE8M0 byte given to every block of both operands. */
ozk_status ozk_stage_mma_probe(const uint8_t* P, const uint8_t* Q, int64_t K, int scale_byte,
                               float* D, void* stream);

/* Test aid for the bounded waits (every wait on a barrier or counter inside the kernels gives up after two
 * seconds, records OZK_ERR_DEVICE_TIMEOUT in the status word and lets the kernel free its tensor memory
 * and return): launches the probe kernel above on zero operands held in the workspace with a barrier
 * that expects 16 bytes nobody sends, so that its wait runs out.  Afterwards ozk_get_async_status
 * returns OZK_ERR_DEVICE_TIMEOUT once and the context and the library remain usable.  Needs a
 * registered workspace of at least 192 KiB. */
ozk_status ozk_stage_wait_probe(void* stream);

/* ---------------------------------------------------------------------------------------
 * 8-bit operands: quantisation, the block-scaled product, AdamW.  Not in the paper: the forms in
 * which a model's layers are multiplied and updated on the same tensor cores.
 *
 * Unlike the calls above, matrices here are ROW-MAJOR (element (r,c) at ptr[r*ld + c], strides in
 * elements), as activations and weights are stored.  Codes are E4M3 bytes (sign, 4 exponent bits of
 * bias 7, 3 fraction bits; 0x7F and 0xFF are NaN, there is no infinity, the largest value is 448).
 * Every 128 elements along the axis that a product sums over share one scale.  Scales are UE8M0
 * bytes c standing for 2^(c-127), c <= 254, unless a call says float.  A power-of-two scale makes
 * x / scale exact, so a code is the one rounding of its element.
 *
 * Scale layouts ("lines" are the rows of the operand, or its columns, whichever the product does
 * not sum over; block b covers elements 128 b .. 128 b + 127 of the summed axis):
 *   LINES   one scale per line and block: byte ((b / 4) * lines + line) * 4 + b % 4, i.e. 32-bit words of four
 *           blocks, [ceil(blocks/4)][lines]; ozk_fp8_line_scale_bytes() bytes, 4-byte aligned.  Bytes of the last
 *           word beyond the last block are not read by the product and written as 127 by the quantiser.
 *   TILES   one scale per 128 x 128 tile of the matrix as stored: byte (r / 128) * ceil(cols / 128) + c / 128.
 *   LINES_F32, TILES_F32   32-bit floats, row-major [lines][blocks] and [ceil(rows/128)][ceil(cols/128)].
 * ------------------------------------------------------------------------------------- */
enum { OZK_F32 = 0, OZK_BF16 = 1 };
enum { OZK_SCALE_LINES = 0, OZK_SCALE_TILES = 1, OZK_SCALE_LINES_F32 = 2, OZK_SCALE_TILES_F32 = 3 };

/* Bytes of the LINES scales of an operand with this many lines and summed elements (0 on invalid arguments). */
size_t ozk_fp8_line_scale_bytes(int64_t lines, int64_t k);

/* Quantises X (rows x cols, OZK_F32 or OZK_BF16, ldx >= cols) with one scale per 1 x 128 block of a row
 * (row_codes, row_scales: for products that sum over the columns; lines = rows), or per 128 x 1 block of a
 * column (col_codes, col_scales: for products that sum over the rows, such as a weight gradient, which sums
 * over the tokens; lines = cols), or both in one pass over X.  A pair that is not wanted is NULL, NULL.
 *   scale = 2^max(-127, ceil(log2(amax / 448))) with amax the largest finite magnitude of the block (scale 1 for a block
 *   of zeros); code = E4M3(x / scale), to nearest even; NaN and infinities become NaN and do not enter amax.
 * Codes have leading dimensions row_ld, col_ld >= cols, multiples of 16, and 16-byte aligned bases; columns beyond
 * `cols` are not written.  rows, cols = 0 are allowed. */
ozk_status ozk_fp8_quantize_lines(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx,
                                  uint8_t* row_codes, int64_t row_ld, uint8_t* row_scales,
                                  uint8_t* col_codes, int64_t col_ld, uint8_t* col_scales, void* stream);

/* The same with one scale per 128 x 128 tile (TILES): weights, which products sum over either way. */
ozk_status ozk_fp8_quantize_tiles(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx,
                                  uint8_t* codes, int64_t ld, uint8_t* scales, void* stream);

/* One operand of ozk_fp8_gemm.  contract_rows = 0: stored [lines][K], the product sums over the stored columns;
 * 1: stored [K][lines], it sums over the stored rows (no transposed copy is made or needed).
 * codes 16-byte aligned, ld a multiple of 16, at least the stored columns. */
typedef struct {
  const uint8_t* codes;
  int64_t ld;
  const void* scales;
  int scale_kind;      /* OZK_SCALE_* */
  int contract_rows;
} ozk_fp8_operand;

/* C[m,n] = sum_k A(m,k) B(n,k) on the scaled values, FP32 accumulation, C row-major M x N (OZK_F32 or OZK_BF16,
 * ldc >= N), rounded once; accumulate = 1 (OZK_F32 only) adds the product to C instead.
 *   UE8M0 scales (LINES or TILES on either operand): the tensor cores apply them.  Float scales: A is
 *   LINES_F32 and B TILES_F32, both contract_rows = 0.  Other combinations return OZK_ERR_UNSUPPORTED.  A float scale of A times
 *   one of B is formed in FP32 before it meets a block's sum: the two should stay within 2^-126 .. 2^127 together.  (The quantiser writes
 *   UE8M0 scales; float scales are for operands that come with them.)
 *   A forward product y = x w^T has A = x (LINES), B = w (TILES); its input gradient dy w has A = dy (LINES), B = w
 *   with contract_rows = 1; its weight gradient dy^T x has A = dy, B = x, both LINES with contract_rows = 1.
 *   FP32 results: sums over more than 8192 are formed in ranges of at most 8192 that are added in FP32 in order,
 *   because the tensor cores truncate when they accumulate.  Results do not depend on timing.
 *   M, N, K = 0 are allowed (K = 0: C = 0, or unchanged with accumulate).  M, N, K < 2^31.  What lies between the rows of C is not touched.
 * workspace: device memory of ozk_fp8_gemm_workspace_bytes() (one size for all shapes), 256-byte aligned, whose first
 * kibibyte has been cleared once (cudaMemset); NULL takes the registered one.  A call may be several launches that pass sums
 * through it: calls that share one must be made one after the other on one stream (by one host thread at a time), and a graph that
 * captured calls must not run beside others with the same workspace.  A bounded device wait that expired is recorded at its start, see
 * ozk_get_workspace_status().
 * The call only enqueues kernels and, after one eager call, may be captured into a CUDA graph. */
size_t ozk_fp8_gemm_workspace_bytes(void);
ozk_status ozk_fp8_gemm(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B,
                        void* C, int c_type, int64_t ldc, int accumulate,
                        void* workspace, size_t workspace_bytes, void* stream);

/* The same with the two parts of the workspace apart.  status: a kibibyte, cleared once, 256-byte aligned; calls on any stream may
 * share it.  scratch: memory for the sums of this call alone, 256-byte aligned, until it has run; most products need none (NULL, 0).
 * One that needs more than scratch_bytes returns OZK_ERR_WORKSPACE and enqueues nothing; ozk_fp8_gemm_plan() says how much. */
ozk_status ozk_fp8_gemm_scratch(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B,
                                void* C, int c_type, int64_t ldc, int accumulate,
                                void* status, void* scratch, size_t scratch_bytes, void* stream);

/* How a product runs on a GPU with `sms` multiprocessors (0: the current device): pairs = 1 if pairs of CTAs form the tiles, 0 for
 * clusters along K; the tiles' extents and number; the ranges of K that a tile is split into; the scratch that is needed.
 * Needs no GPU if sms is given. */
typedef struct {
  int pairs, tile_rows, tile_cols, splits;
  int64_t tiles;
  size_t scratch_bytes;
} ozk_fp8_plan;
ozk_status ozk_fp8_gemm_plan(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, int c_type, int sms,
                             ozk_fp8_plan* plan);

/* ozk_get_async_status() for a workspace that was passed to a call rather than registered. */
ozk_status ozk_get_workspace_status(void* workspace, void* stream);

/* ---------------------------------------------------------------------------------------
 * Around the 8-bit products: the norm that writes their operands, and products grouped by expert.
 * ------------------------------------------------------------------------------------- */

/* RMS norm of x (rows x cols) with the residual stream r (of x_type, or OZK_F32) added first:
 *   h = x + r, rounded to the stream's type and written to total (the updated stream);  s = 1 / sqrt(mean(h^2) + eps);  y = h s w
 * residual NULL: h = x, and total is not used.  total may be the residual (same ld), or x where the types agree: the stream is updated in place.
 * The norm is of h as it is stored.  weight: cols numbers.  FP32 arithmetic; the order of a sum follows from the sizes, the types, how far the rows' places and strides
 * let elements be read together, and the GPU's multiprocessors: the same call repeats its bits, one on rows at other places may differ in the last ones.
 *   root       optional, rows floats: s, which the backward pass reads (wanted where col_codes are)
 *   y          optional, rows x cols: y without quantisation, not in the place of h
 *   row_codes, row_scales / col_codes, col_scales   optional: y by 1 x 128 / 128 x 1 blocks, as by ozk_fp8_quantize_lines
 * A sum of squares beyond FP32 (a mean square above 3.4e38 / cols) counts as infinite: s = 0, y = 0.  Squares below FP32 count as 0, which shows where eps is 0.  A NaN or an infinity in a row makes NaN of the row's y (0 of what is finite beside an infinity).
 * cols <= 32768.  rows, cols = 0 are allowed. */
typedef struct {
  int64_t rows, cols;
  const void* x;             /* x_type */
  int64_t ldx;
  const void* residual;      /* residual_type, or NULL */
  int64_t ldr;
  void* total;               /* residual_type: h */
  int64_t ldt;
  const void* weight;        /* weight_type */
  float* root;
  void* y;                   /* x_type */
  int64_t ldy;
  uint8_t* row_codes;
  int64_t row_ld;
  uint8_t* row_scales;
  uint8_t* col_codes;
  int64_t col_ld;
  uint8_t* col_scales;
  double eps;
  int x_type, residual_type, weight_type;
} ozk_rms_norm_args;
ozk_status ozk_rms_norm(const ozk_rms_norm_args* args, void* stream);

/* Its gradients.  dy: gradient of y; total, root: what the forward pass normed (x, where there was no residual) and its s; dtotal: optional
 * gradient of h from elsewhere.
 *   g = dy w;  dx = dh + s (g - h s mean(g h s)), the gradient of x and of r alike;  dweight = sum over the rows of dy h s (FP32, optional)
 * dx may be dtotal.  scratch: ozk_rms_norm_backward_scratch_bytes(), 16-byte aligned, for this call alone; not needed without dweight. */
size_t ozk_rms_norm_backward_scratch_bytes(int64_t rows, int64_t cols);
typedef struct {
  int64_t rows, cols;
  const void* dy;            /* dy_type */
  int64_t lddy;
  const void* total;         /* total_type */
  int64_t ldt;
  const float* root;
  const void* weight;        /* weight_type */
  const void* dtotal;        /* total_type, or NULL */
  int64_t lddt;
  void* dx;                  /* total_type */
  int64_t lddx;
  float* dweight;            /* or NULL */
  void* scratch;
  size_t scratch_bytes;
  int dy_type, total_type, weight_type;
} ozk_rms_norm_backward_args;
ozk_status ozk_rms_norm_backward(const ozk_rms_norm_backward_args* args, void* stream);

/* Segments: rows lie in the order of the experts they belong to; expert e has rows offsets[e] .. offsets[e+1] - 1 (offsets: experts + 1 numbers in
 * device memory, ascending from offsets[0] >= 0 to offsets[experts] <= rows).  Segments may be empty; rows before the first and behind the last
 * belong to nobody.  Offsets that fall or leave the rows are read as the nearest that do not.  experts <= 1024 in products.
 * 128 x ozk_fp8_segment_blocks() is below 2^31 in ozk_fp8_quantize_segments and ozk_fp8_segment_gemm (OZK_ERR_UNSUPPORTED). */

/* The operand of a product that sums over the rows of each expert: blocks of 128 rows that begin with each segment.  Block b of the segments has
 * rows 128 b .. 128 b + 127 of col_codes, with zeros behind the end of a segment, and scales as LINES (lines = cols, k = 128 x
 * ozk_fp8_segment_blocks()); blocks that no segment takes are left as they were.  row_codes, row_scales: optional, the rows of the segments
 * as by ozk_fp8_quantize_lines; other rows are left as they were. */
int64_t ozk_fp8_segment_blocks(int64_t rows, int64_t experts);   /* floor((rows + 127 min(experts, rows)) / 128): enough for any offsets */
ozk_status ozk_fp8_quantize_segments(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, const int32_t* offsets, int64_t segments,
                                     uint8_t* row_codes, int64_t row_ld, uint8_t* row_scales,
                                     uint8_t* col_codes, int64_t col_ld, uint8_t* col_scales, void* stream);

/* ozk_fp8_quantize_tiles of `experts` matrices x_step elements apart; their codes lie `step` bytes apart (a multiple of 16), their
 * scales one after another. */
ozk_status ozk_fp8_quantize_experts(int64_t experts, int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, int64_t x_step,
                                    uint8_t* codes, int64_t ld, int64_t step, uint8_t* scales, void* stream);

/* The experts' weights, as ozk_fp8_quantize_experts writes them.  contract_rows as in ozk_fp8_operand. */
typedef struct {
  const uint8_t* codes;
  int64_t ld, stride;     /* from row to row, from expert to expert */
  const uint8_t* scales;
  int contract_rows;
} ozk_fp8_experts;

/* C[t,n] = sum_k X(t,k) W_e(n,k) for the rows t of each expert e (X: rows x K, LINES, contract_rows = 0; C: rows x N), as ozk_fp8_gemm with that
 * expert's weights; input gradients have W's contract_rows = 1.  Rows of C outside the segments are left as they were, or cleared with
 * clear_rest = 1.  status: as for ozk_fp8_gemm_scratch.  No other memory is used.  rows < 2^31 - 65536 (OZK_ERR_UNSUPPORTED). */
ozk_status ozk_fp8_grouped_gemm(int64_t rows, int64_t N, int64_t K, const ozk_fp8_operand* X, const ozk_fp8_experts* W, int64_t experts,
                                const int32_t* offsets, void* C, int c_type, int64_t ldc, int clear_rest, void* status, void* stream);

/* C_e[m,n] = sum over the rows t of expert e of A(t,m) B(t,n), for every expert (weight gradients): C is [experts][M][N], `stride` elements
 * from expert to expert.  A, B: by ozk_fp8_quantize_segments with the same offsets (contract_rows = 1, LINES).  An expert without rows gets
 * zeros, or with accumulate (OZK_F32 only, adds to C) keeps what it has. */
ozk_status ozk_fp8_segment_gemm(int64_t experts, int64_t M, int64_t N, int64_t rows, const ozk_fp8_operand* A, const ozk_fp8_operand* B,
                                const int32_t* offsets, void* C, int c_type, int64_t ldc, int64_t stride, int accumulate, void* status,
                                void* stream);

/* One tensor of an AdamW step: n elements, contiguous.  Element i of the optimiser's block b has i / 128 = b.
 *   32-bit states: m, v are floats.  8-bit states: m holds E4M3 codes of the first moment and v E4M3 codes of the
 *   ROOT r = sqrt(v) of the second (its 17.8 binades below a block's largest entry are 35 of v), m_scale and v_scale one
 *   UE8M0 byte per block of 128. */
typedef struct {
  void* param;         /* options.param_type, updated */
  const void* grad;    /* options.grad_type */
  void* m;
  void* v;
  uint8_t* m_scale;    /* 8-bit states only, else NULL */
  uint8_t* v_scale;
  void* copy;          /* optional BF16 copy of an FP32 param, written */
  int64_t n;
} ozk_adamw_tensor;

typedef struct {
  int param_type, grad_type;   /* OZK_F32 or OZK_BF16 */
  int state_bits;              /* 32 or 8 */
  int stochastic;              /* 1: 8-bit roots and BF16 params are rounded up or down by a hash of (seed, tensor, element) */
  uint32_t seed;
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;                /* 1 for the first step */
  const float* grad_scale;     /* optional device scalar: gradients are multiplied by it (clipping, loss scale) */
  const int* skip;             /* optional device flag: nonzero leaves everything unchanged (overflow in the gradients) */
} ozk_adamw_options;

/* One AdamW step over `count` tensors (host array) in one launch per 448 of them, all FP32 arithmetic:
 *   g' = g grad_scale;  m' = beta1 m + (1 - beta1) g';  v' = beta2 v + (1 - beta2) g'^2;  r = sqrt(v')
 *   p' = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m' / (r / sqrt(1 - beta2^step) + eps)
 * 8-bit states are then rounded to their block's scale as by the quantiser: m' to nearest, r to nearest or, with
 * `stochastic`, up or down (a root that changes by less than half a unit per step would never change otherwise);
 * a root that is not zero is stored as at least 2^-9 of its scale, so that m / (r + eps) stays bounded.  The hash is
 * mix(i mod 2^32 ^ mix(index of the tensor + 1) ^ mix(seed)), mix(x): x ^= x>>16, x *= 0x7feb352d, x ^= x>>15, x *= 0x846ca68b,
 * x ^= x>>16 (Chris Wellons' lowbias32, 2018); the root uses its upper 16 bits, a BF16 parameter the lower 16.
 * Second moments below 2^-126 have the root zero.  Non-finite gradients give non-finite (8-bit: NaN) values in their own
 * element only.  No tensor may overlap another. */
ozk_status ozk_adamw_step(const ozk_adamw_tensor* tensors, int64_t count, const ozk_adamw_options* options, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OZK_H_ */
