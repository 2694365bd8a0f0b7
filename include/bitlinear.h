/*
 * bitlinear.h - C-ABI of the BitLinear W1.58A8 hot path for AMD MI355X (gfx950).
 *
 * The operation is the BitLinear layer of BitNet b1.58 (technical report,
 * Section 2 "Architecture": absmean ternary weights, per-token absmax int8
 * activations; Section 5.1 "GPU Inference": four ternary values stored per
 * 8-bit integer, unpacked just before the integer matrix product).
 *
 * The report gives these steps in words only.  The arithmetic below is the
 * reading this library fixes; every fp32 step is ONE IEEE-754 binary32
 * round-to-nearest-even operation, in the order written, with no fused
 * multiply-add contraction.
 *
 *   weight scale   beta = fp32( (sum_{n,k} |W[n][k]|) / (N*K) )      (sum and
 *                  division carried in fp64, one final rounding to fp32)
 *   ternarize      d = beta + 1e-5f ; t = rint(W[n][k] / d) (ties to even);
 *                  Wt[n][k] = clamp(t, -1, +1)  in {-1, 0, +1}
 *   code           c = Wt + 1  in {0, 1, 2}        (3 is never produced)
 *   activation     x~ = fp32(bf16 X[m][k]) ; gamma = max_k |x~| ;
 *   quantizer      g = max(gamma, 1e-5f) ; inv = 127.0f / g ;
 *                  q[m][k] = clamp(rint(x~ * inv), -127, 127)  (ties to even);
 *                  scale[m] = g / 127.0f ; rowsum[m] = sum_k q[m][k]  (int32)
 *   contraction    acc[m][n] = sum_k q[m][k] * Wt[n][k]      (exact, int32)
 *   rescale        y[m][n] = (float)acc[m][n] * (beta * scale[m])
 *
 * PACKED LAYOUTS.  2 bits per weight.  Rows are padded: Kp = bl_padded_k(K) (K rounded up to
 * a multiple of 64) weights per row and Np = N rounded up to a multiple of 4 rows; every field
 * outside the N x K matrix holds code 1 (weight 0).  A packed matrix is Np*Kp/4 bytes
 * (= N*K/4 when K % 64 == 0 and N % 4 == 0).
 *   BL_LAYOUT_ROWMAJOR (0): byte index b = n*(Kp/4) + k/4 ; weight k occupies
 *     bits [2*(k%4), 2*(k%4)+1] of byte b (lowest bits = lowest k).
 *   BL_LAYOUT_K16 (1): same byte count and the same 4-byte word per group of
 *     16 consecutive k of a row, but inside the word the two index digits are
 *     swapped: with i = k % 16, weight k occupies bits [2*(i/4), 2*(i/4)+1] of
 *     byte n*(Kp/4) + (k/16)*4 + i%4.  (So `(word >> 2s) & 0x03030303` yields the
 *     codes of k = 4s..4s+3 as four bytes in natural order: the kernels' native
 *     form.  Layout 0 is supported by permuting the activation bytes instead.)
 *   BL_LAYOUT_TRIT5 (2): five weights per byte, 1.6 bits per weight (the density behind the
 *     memory footprint of Table 1; the 2-bit forms above are the ones Section 5.1 describes).
 *     Rows of Kq = K rounded up to a multiple of 80 weights (Kq/5 bytes, a whole number of
 *     16-byte loads), Np rows, code 1 outside the matrix: Np*Kq/5 bytes.  Inside a row, the 4-byte
 *     word g covers k = 20g .. 20g+19; its byte j holds the codes c_i of k = 20g + 4i + j,
 *     i = 0..4, as b = ceil(v * 256 / 243) with v = sum_i c_i * 3^(4-i) (so that c_0 = (3b) >> 8,
 *     and the same step on the low byte of 3b yields c_1, and so on: no table, no division).
 *     Accepted by bl_pack_ternary, bl_unpack_ternary, bl_packed_bytes and bl_stack_build (the
 *     bandwidth-bound M = 1 decode, where bytes are time); BL_ERR_LAYOUT elsewhere.
 *   BL_LAYOUT_KMAJOR (3): the transposed matrix, one row per input feature k (K rows, no padding
 *     of K), each row the 2-bit codes of n = 0 .. Nq-1, Nq = N rounded up to a multiple of 64, packed
 *     like layout 0 along n (byte index k*(Nq/4) + n/4, bits [2*(n%4), 2*(n%4)+1]), code 1 behind
 *     column N: K*Nq/4 bytes.  For activations that are mostly zero (Section 2 takes squared ReLU
 *     for the sparsity it gives the input of the down projection): the rows of zero activations
 *     are never read.  N <= 3072.  Accepted by bl_pack_ternary, bl_unpack_ternary,
 *     bl_packed_bytes and bl_stack_build; BL_ERR_LAYOUT elsewhere.
 * QUANTISED ACTIVATIONS are int8 [M][Kp]: leading dimension Kp, zeros in columns K..Kp-1 (what
 * bl_quant_act_int8 writes), so that a padded weight meets a zero.  Outputs are [M][N].
 *
 * CONVENTIONS.  Every pointer is a DEVICE pointer owned by the caller unless a
 * comment says "host".  The library allocates and frees nothing; all work is
 * enqueued on the caller's stream `s` (a hipStream_t passed as void*; NULL is
 * the null stream) and no call synchronises.  Argument errors are found on the
 * host before any HIP call and reported as a status code (no exceptions, no
 * global error state; the only process-wide state is the test hook below).  Preconditions on
 * every matrix: 1 <= N, K <= 2^24; `packed` and `q` 16-byte aligned; otherwise
 * BL_ERR_SHAPE / BL_ERR_ALIGN.  Entry points that read bf16 or fp32 activations inside a
 * product kernel (fused producers, epilogues, bl_stack_* with X) need K % 64 == 0 and say so;
 * a ragged K goes through bl_quant_act_int8 and the int8 inputs of the products.
 * Non-finite inputs have no defined result, but what they spoil is bounded: an activation row and
 * its outputs (a NaN is passed over by gamma and quantises to -127, the other values of the row as
 * without it; an infinity makes the scale infinite), or the packed matrix (its beta).
 * There is no bias argument (the report removes all biases, Section 2).
 */
#ifndef BITLINEAR_H
#define BITLINEAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BL_OK            = 0,
    BL_ERR_NULL      = 1,  /* a required pointer is NULL                        */
    BL_ERR_SHAPE     = 2,  /* M/N/K out of range or not a permitted multiple    */
    BL_ERR_LAYOUT    = 3,  /* unknown layout id / layout not valid for shape    */
    BL_ERR_ALIGN     = 4,  /* pointer not aligned as required                   */
    BL_ERR_VALUE     = 5,  /* unknown in_kind / op id                           */
    BL_ERR_HIP       = 6,  /* a HIP runtime call or kernel launch failed        */
    BL_ERR_WORKSPACE = 7   /* workspace required but NULL                       */
} bl_status;

typedef void* bl_stream;   /* hipStream_t */

enum { BL_LAYOUT_ROWMAJOR = 0, BL_LAYOUT_K16 = 1, BL_LAYOUT_TRIT5 = 2, BL_LAYOUT_KMAJOR = 3 };
enum { BL_IN_FP32_LATENT = 0, BL_IN_INT8_TERNARY = 1 };
enum { BL_OP_PACK = 0, BL_OP_QUANT = 1, BL_OP_GEMV = 2, BL_OP_GEMM = 3 };

/* Library version (major*10000 + minor*100 + patch) and a static string
 * naming a status code.  Host-only, no GPU needed. */
int         bl_version(void);
const char* bl_status_str(int status);

/* Bytes of a packed N x K matrix (Np*Kp/4 for every layout, see PACKED LAYOUTS); 0 if the
 * shape or layout is not permitted.  Host-only.  (Section 5.1: 4 values per byte.) */
size_t bl_packed_bytes(int64_t N, int64_t K, int layout);

/* Kp: K rounded up to a multiple of 64, the row length of packed weights and the leading
 * dimension of quantised activations; 0 if K is out of range.  Host-only. */
int64_t bl_padded_k(int64_t K);

/* Bytes of device scratch the given op needs for the given shape (may be 0).
 * The workspace is caller-allocated, 256-byte aligned, and may be reused by
 * later calls on the same stream.  Host-only. */
size_t bl_workspace_bytes(int op, int64_t M, int64_t N, int64_t K);

/* Weight quantisation and packing (Section 2, "Weight Quantization": absmean
 * to ternary; Section 5.1: packing).  Offline step, not on the timed path.
 *   W        device, in_kind 0: fp32 [N][K] row-major latent weights (beta is
 *            computed and written); in_kind 1: int8 [N][K] values in {-1,0,1}
 *            (beta is read, not written).
 *   packed   device out, bl_packed_bytes(N,K,layout) bytes.
 *   beta     device, 1 float.
 *   workspace device, bl_workspace_bytes(BL_OP_PACK, 0, N, K) bytes.
 * Enqueues two kernels (partial |W| sums in fp64; their fixed-order sum inside
 * ternarize+pack), or three where W is large (an estimate of beta from a sample; the sums and
 * every code that does not depend on the rest; the other codes).  The fp64 sum order is fixed for
 * a shape and layout, so beta is reproducible. */
bl_status bl_pack_ternary(const void* W, int in_kind, int64_t N, int64_t K, int layout,
                          uint8_t* packed, float* beta, void* workspace, bl_stream s);

/* Inverse of the packing, for round-trip tests: writes Wt int8 [N][K] row-major
 * in {-1,0,1} and sets *bad (device int32, zeroed by this call) to the number
 * of 2-bit fields holding the invalid code 3 (those decode to +2). */
bl_status bl_unpack_ternary(const uint8_t* packed, int64_t N, int64_t K, int layout,
                            int8_t* Wt, int32_t* bad, bl_stream s);

/* Per-token absmax int8 activation quantisation (Section 2, "Activation
 * Quantization").
 *   X      device bf16 [M][K] row-major (raw 16-bit patterns), 16-byte aligned
 *          (2-byte aligned is enough when K % 64 != 0).
 *   q      device out int8 [M][Kp], zeros in the padding;
 *   scale  device out fp32 [M] (= max(gamma,1e-5)/127);
 *   rowsum device out int32 [M], may be NULL.          M >= 1. */
bl_status bl_quant_act_int8(const uint16_t* X, int64_t M, int64_t K,
                            int8_t* q, float* scale, int32_t* rowsum, bl_stream s);

/* W1.58A8 product for decode batches, 1 <= M <= 64 (Section 5.1).  Streams the
 * packed weights once per call.
 *   packed/beta/layout  as written by bl_pack_ternary.
 *   q      device int8 [M][Kp];  scale device fp32 [M] (needed only if y != NULL).
 *   rowsum device int32 [M] or NULL (this call derives what it needs from q).
 *   acc    device out int32 [M][N] or NULL;  y device out fp32 [M][N] or NULL;
 *          at least one of the two must be non-NULL.
 *   workspace needed only when K > 8192 and rowsum is NULL (such rows go through the
 *          prefill kernel, which then computes the row sums there:
 *          bl_workspace_bytes(BL_OP_GEMV, M, N, K) bytes; BL_ERR_WORKSPACE if NULL);
 *          otherwise unused and may be NULL. */
bl_status bl_gemv_w158a8(const uint8_t* packed, const float* beta, int layout,
                         const int8_t* q, const float* scale, const int32_t* rowsum,
                         int64_t M, int64_t N, int64_t K,
                         int32_t* acc, float* y, void* workspace, bl_stream s);

/* W1.58A8 product for prefill, any M >= 1 (Section 5.1): packed tiles are
 * unpacked to int8 on chip and contracted on the int8 matrix cores.  Same
 * arguments as bl_gemv_w158a8.  If rowsum is NULL the call computes the row
 * sums itself into `workspace` (bl_workspace_bytes(BL_OP_GEMM, M, N, K) bytes,
 * then required). */
bl_status bl_gemm_w158a8(const uint8_t* packed, const float* beta, int layout,
                         const int8_t* q, const float* scale, const int32_t* rowsum,
                         int64_t M, int64_t N, int64_t K,
                         int32_t* acc, float* y, void* workspace, bl_stream s);

/* Fused BitLinear for decode, 1 <= M <= 16, K <= 8192, K % 64 == 0, M*(K+16) <= 96 KiB: the per-token absmax
 * int8 quantiser (Section 2) runs inside the product kernel (Section 5.1), so
 * one launch takes bf16 activations to fp32 outputs.  Same arithmetic, bit for
 * bit, as bl_quant_act_int8 followed by bl_gemv_w158a8.
 *   X         device bf16 [M][K].
 *   acc / y   device out [M][N], either may be NULL (not both).
 *   q_out     device out int8 [M][K] or NULL: the quantised activations;
 *   scale_out device out fp32 [M] or NULL: max(absmax,1e-5)/127 per token. */
bl_status bl_bitlinear_decode(const uint8_t* packed, const float* beta, int layout,
                              const uint16_t* X, int64_t M, int64_t N, int64_t K,
                              int32_t* acc, float* y, int8_t* q_out, float* scale_out, bl_stream s);

/* Fused producer: the elementwise step that yields the bf16 input X[m][k] of a
 * BitLinear, evaluated inside the kernel that quantises it (no bf16 tensor in
 * HBM).  Each kind is exact elementwise fp32 work, then round-to-nearest-even
 * narrowing to bf16; the quantiser then runs on those bf16 values as usual.
 *   BL_PROD_BF16       X = in0 (bf16 [M][K]).
 *   BL_PROD_F32        X = bf16(in0)                      in0 fp32 [M][K].
 *   BL_PROD_ATTN_V     context-length-1 attention over a fused QKV row
 *                      in0 fp32 [M][(n_q+2*n_kv)*head_dim] = [Q | K | V]:
 *                      X[m][h*head_dim+d] = bf16(V[m][h/(n_q/n_kv)][d]); K = n_q*head_dim.
 *   BL_PROD_RESIDUAL   t = in0 + in1 (fp32 [M][K] each), X = bf16(t); if aux_out
 *                      is given, t is also stored there (fp32 [M][K]).
 *   BL_PROD_RELU2_GATE in0 fp32 [M][2K] = [g | u]: X = bf16((max(g,0)*max(g,0))*u)
 *                      (the squared-ReLU gated FFN activation, Section 2).
 * norm != 0 adds the sub-layer normalisation in front of the quantiser (Section 2,
 * "Normalization"; the report names the scheme but gives no formula, so this is the
 * bias-free RMS form): with t[k] the fp32 value of the kind above BEFORE narrowing,
 *   ss = sum_k t[k]^2 with exact fp64 squares and an fp64 sum (relative error of the sum
 *        far below 1e-12; the order inside a kernel is fixed, so a result is reproducible),
 *   r = fp32(1 / sqrt(ss/K + eps)) in fp64,   X[k] = bf16((t[k]*r)*gain[k])
 * (gain NULL: no second multiply).  Every later step is a single rounded IEEE operation; r can
 * depend on the summation order only when 1/sqrt(ss/K+eps) lies within ~1e-12 (relative) of
 * an fp32 rounding midpoint.  BL_PROD_RESIDUAL still stores the
 * un-normalised sum in aux_out.
 * All pointers are device pointers, 16-byte aligned. */
enum { BL_PROD_BF16 = 0, BL_PROD_F32 = 1, BL_PROD_ATTN_V = 2, BL_PROD_RESIDUAL = 3, BL_PROD_RELU2_GATE = 4 };
typedef struct {
    int kind;
    const void* in0;
    const float* in1;
    float* aux_out;
    int n_q, n_kv, head_dim;
    int norm;               /* 0: none; 1: RMS normalisation as above */
    const float* gain;      /* fp32 [K] or NULL */
    float eps;              /* added to the mean square (fp32) */
} bl_producer;

/* One decode product of a group.  Give either X (bf16, fused quantiser), a
 * producer (prod.in0 != NULL, fused producer + quantiser), or q (+ scale if y is
 * wanted, + optional rowsum).  All pointers are device pointers; the descriptor
 * array itself is HOST memory, read during the call.
 * fixed_scale > 0 (fused paths only) replaces absmax/127 in the rescale, i.e.
 * the layer then acts on x/absmax (a normalised input); 0 = normal.
 * residual (fp32 [M][N] or NULL): y = residual + acc*(beta*scale), one fp32 add. */
typedef struct {
    const uint8_t* packed;
    const float* beta;
    const uint16_t* X;
    const int8_t* q;
    const float* scale;
    const int32_t* rowsum;
    int64_t N, K;
    int32_t* acc;
    float* y;
    int8_t* q_out;
    float* scale_out;
    float fixed_scale;
    bl_producer prod;
    const float* residual;
} bl_decode_desc;

/* Up to four INDEPENDENT decode products (same M, same layout, K <= 8192 each)
 * in one kernel launch, e.g. the four BitLinear shapes of a layer on
 * independent inputs.  Results are identical to separate calls; the point is
 * one launch and one continuous weight stream instead of four.
 * Limits: a product with a fused input (X or prod) needs M <= 16, K % 64 == 0 and
 * M*(K+16) <= 96 KiB; a product with int8 input (q, [M][Kp]) takes M <= 64 and any K.
 * Errors: BL_ERR_SHAPE outside these limits or for count outside 1..4. */
bl_status bl_bitlinear_decode_group(const bl_decode_desc* descs, int count, int layout, int64_t M, bl_stream s);

/* Producer + per-token absmax int8 quantiser for prefill (Section 2): like
 * bl_quant_act_int8, but the bf16 activations come from `prod` (HOST pointer to
 * the descriptor; its tensors are device memory).  One workgroup per token.
 * Needs K % 64 == 0 (BL_ERR_SHAPE otherwise). */
bl_status bl_quant_act_ex(const bl_producer* prod, int64_t M, int64_t K,
                          int8_t* q, float* scale, int32_t* rowsum, bl_stream s);

/* bl_gemm_w158a8 with an optional residual (fp32 [M][N] or NULL) added in the
 * epilogue: y = residual + acc*(beta*scale[m]), one fp32 add per element. */
bl_status bl_gemm_w158a8_res(const uint8_t* packed, const float* beta, int layout,
                             const int8_t* q, const float* scale, const int32_t* rowsum,
                             int64_t M, int64_t N, int64_t K, const float* residual,
                             int32_t* acc, float* y, void* workspace, bl_stream s);

/* Prefill product with a FUSED PRODUCER EPILOGUE (Section 2: per-token absmax activation
 * quantisation, ReLU^2 in the FFN): the elementwise step that turns this product's output into
 * the next BitLinear's input runs in the product's epilogue, so the fp32 output is not written
 * and read again just to be narrowed.  The epilogue writes the bf16 input of the next BitLinear
 * and folds the row maximum of its absolute values into absmax[] (an order-free maximum on the
 * float bits, across all workgroups of the launch); bl_quant_from_absmax then quantises in one
 * pass.  Bit for bit the same numbers as bl_gemm_w158a8[_res] followed by bl_quant_act_ex.
 *   BL_EPI_RESIDUAL    t = residual[m][n] + acc*(beta*scale[m]);  N_out = N
 *   BL_EPI_RELU2_GATE  the matrix is a fused [gate | up] pair (rows n and N/2 + n):
 *                      g = acc_g*(beta*scale[m]), u = acc_u*(..), t = (max(g,0)*max(g,0))*u;
 *                      N_out = N/2; needs N % 128 == 0
 *   y       device out fp32 [M][N_out] or NULL: t itself (wanted when t is a later residual)
 *   x_bf16  device out bf16 [M][N_out]: bf16(t); 2-byte aligned (4-byte aligned is faster)
 *   absmax  device in/out fp32 [M]: must hold 0 (or an earlier partial maximum of the same rows)
 *           before the launch; receives max_n |bf16(t)|.  bl_quant_from_absmax clears it again.
 *   acc     device out int32 [M][N] or NULL (the raw accumulators, natural column order).
 * Needs layout BL_LAYOUT_K16, K % 128 == 0 and rowsum (BL_ERR_LAYOUT / BL_ERR_SHAPE / BL_ERR_NULL). */
enum { BL_EPI_RESIDUAL = 1, BL_EPI_RELU2_GATE = 2 };
typedef struct {
    int kind;
    const float* residual;   /* BL_EPI_RESIDUAL: fp32 [M][N] */
    float* y;
    uint16_t* x_bf16;
    float* absmax;
} bl_gemm_epilogue;
bl_status bl_gemm_w158a8_fused(const uint8_t* packed, const float* beta, int layout,
                               const int8_t* q, const float* scale, const int32_t* rowsum,
                               int64_t M, int64_t N, int64_t K, const bl_gemm_epilogue* ep /* HOST */,
                               int32_t* acc, bl_stream s);
/* One-pass quantiser for rows whose absmax is already known: like bl_quant_act_int8 with
 * gamma = absmax[m] given; clears absmax[m] to 0 afterwards.  Needs K % 64 == 0. */
bl_status bl_quant_from_absmax(const uint16_t* X, float* absmax, int64_t M, int64_t K,
                               int8_t* q, float* scale, int32_t* rowsum, bl_stream s);

/* Persistent streaming decode over a TABLE of products (Section 5.1: the decode kernel is
 * there to use as little memory bandwidth as possible, which on this GPU means the weight
 * stream of a whole stack of BitLinears must never stop).  One launch walks every product
 * of the table with as many workgroups as stay resident; each product is the same
 * arithmetic, bit for bit, as one entry of bl_bitlinear_decode_group.  Entries with a fused
 * input are quantised (Section 2) without a pass of their own: a plain bf16 input (X) inside
 * the stream launch, by each workgroup that meets the product (about five hundred workgroups
 * over the table, each meeting one or two products; no data crosses workgroups); a
 * producer or a normalised input (prod) by a small preparation launch in front of it (one
 * workgroup per such entry, into scratch inside `table`; the same launch computes a missing
 * rowsum of an int8 entry); int8 entries are streamed as they are.
 * The products of one table are INDEPENDENT: none may read what another writes.
 * Entries with a fused input need K % 64 == 0; int8 entries (q of Kp bytes) take any K.
 *   bl_stack_table_bytes  device bytes `table` needs for these descriptors (HOST array): the
 *                         table itself plus the scratch for quantised rows.  0: bad count or K.
 *   bl_stack_build        setup call: checks the descriptors (HOST array), lays the work out
 *                         over the grid, copies the table to `table` (device, 256-byte
 *                         aligned, caller-owned) and fills *plan (HOST, caller-owned).  It
 *                         waits for that copy on `s` (the only call here that synchronises).
 *                         Limits: 1 <= count <= 1024; M = 1: K <= 20480 per product (M > 1:
 *                         the batched form below).
 *   bl_stack_run          at most two kernel launches on `s` (preparation, stream); no
 *                         allocation, no synchronisation; may be captured in a HIP graph and
 *                         replayed.  The table and every tensor it names must stay alive and
 *                         in place; runs on one table must not overlap (they share the scratch).
 * BATCHED FORM, 2 <= M <= BL_STACK_MAX_TOKENS tokens per product (batched decode: the weights
 * of the table are still read once per run): bl_stack_build with M > 1 takes int8 entries only
 * (q [M][Kp], scale [M] when y is wanted, rowsum [M]; outputs [M][N]; BL_ERR_VALUE for X / prod,
 * BL_ERR_NULL without rowsum), layout BL_LAYOUT_K16 (BL_ERR_LAYOUT otherwise), any N and K;
 * `table` needs bl_stack_table_bytes_batched bytes (0: bad count, M, N or K).  The kernel keeps
 * the token rows of a table entry in LDS and multiplies on the matrix cores, 32 tokens to a tile.
 * How a product becomes table entries is the library's business and never changes a result:
 * up to 64 tokens in one entry where their rows fit LDS whole, else groups of at most 32 tokens
 * (the weights are then read once per group); rows too long for LDS are cut into k parts whose
 * partial sums meet in scratch inside `table` through integer atomics (exact, order-free) and
 * are finished (row sum, rescale, residual) by a second small launch of the same run, which
 * also clears the scratch.  plan->entries tells how many entries the table holds.
 * With more than 48 tokens (33 to 48: tables that are large against their longest row), and every row length a multiple of 128
 * after padding, the table is walked by the prefill tile kernel instead (Section 5.1: packed tiles expanded to int8 on chip
 * for the int8 matrix cores): tiles of all tokens x 256 weight rows, both operands streamed
 * through LDS, the tiles of all products balanced over the resident workgroups by their k steps, one
 * launch, weights read once; plan->red_ints then holds the table's blocks of 128 weight rows (one token:
 * which form of the kernel walks the table, or, in the k-major form, the partial sums kept in LDS).
 * Same arithmetic, bit for bit, as bl_gemv_w158a8 on each product. */
enum { BL_STACK_MAX_COUNT = 1024, BL_STACK_MAX_TOKENS = 64 };
typedef struct {
    int32_t count, blocks, prep_count, inline_count, norm, lds_bytes, layout, red_ints;
    int64_t wg_offset, prep_offset;   /* byte offsets inside `table`                            */
    int64_t packed_bytes;             /* packed weight bytes of the products: what one run streams */
    int64_t table_bytes;
    int32_t tokens, entries;          /* M; table entries (> count when products were split)    */
} bl_stack_plan;
size_t    bl_stack_table_bytes(const bl_decode_desc* descs, int count);
size_t    bl_stack_table_bytes_batched(const bl_decode_desc* descs, int count, int64_t M);
bl_status bl_stack_build(const bl_decode_desc* descs, int count, int layout, int64_t M,
                         void* table, bl_stack_plan* plan, bl_stream s);
bl_status bl_stack_run(void* table, const bl_stack_plan* plan, bl_stream s);

/* bl_gemm_w158a8 for callers that cannot allocate device memory or bring a workspace:
 * code running under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same product and same results as bl_gemm_w158a8 called with rowsum = NULL;
 * the scratch for the row sums sum_k q[m][k] is a static device array inside the library
 * (64 KiB per GPU, held until the process ends), so the call allocates and frees nothing.
 * Limit: 1 <= M <= 16384, else BL_ERR_SHAPE.  All calls on one GPU share that array:
 * calls that overlap on the same GPU (different streams or threads) race; calls on one
 * stream, or otherwise ordered, are safe.  Nothing needs clearing between calls. */
bl_status bl_gemm_w158a8_noalloc(const uint8_t* packed, const float* beta, int layout,
                                 const int8_t* q, const float* scale,
                                 int64_t M, int64_t N, int64_t K,
                                 int32_t* acc, float* y, bl_stream s);

/* KEY/VALUE CACHE OF 8-BIT CODES, and the attention that reads it: what stands between the QKV and the output
 * BitLinear of a layer when a model is served.  Three calls (the first also with a limit), each one descriptor (HOST memory, read during the call)
 * and a stream: block tables and slot maps of a step from the requests' lengths; the rotary append of new tokens;
 * causal attention over the cache for any number of new tokens per request.
 *
 * The cache is a pool of blocks of `block` tokens (16, 32, 64 or 128); a request's tokens fill the blocks that its row of a
 * block table names.  Token j of a request is in block table[j / block] at offset j % block; its slot is
 * that block * `block` + the offset.
 *   k        codes [n_blocks][n_kv][block][head_dim]
 *   v        codes [n_blocks][n_kv][head_dim][block]: transposed, so that sixteen tokens of a feature are 16 bytes, which
 *            is what a lane hands to the matrix cores
 *   k_scale, v_scale  fp32 [n_blocks][n_kv]: a code c stands for c * scale of its block and head
 *   k_stride, v_stride  bytes from a block to the next (multiples of 16; at least n_kv * block * head_dim, below 2^36),
 *   scale_stride        floats from a block's scales to the next's (at least n_kv): other layers' blocks may lie between
 * kind BL_KV_INT8: codes are integers of -127..127; BL_KV_E4M3: OCP e4m3 values (no NaN codes).  head_dim 64 or 128.
 * Scales are >= 0.  What no token has written may hold anything.  n_blocks * block < 2^31. */
enum { BL_KV_INT8 = 0, BL_KV_E4M3 = 1 };
enum { BL_KV_MAX_REQUESTS = 4096 };
typedef struct {
    int kind, block, n_kv, head_dim;
    int64_t n_blocks;
    void* k;
    void* v;
    float* k_scale;
    float* v_scale;
    int64_t k_stride, v_stride, scale_stride;
} bl_kv_cache;

/* Block tables and slot maps of a step, built on the GPU (nothing is read back, so that a step may sit in a HIP graph).
 * Request b holds seq_len[b] tokens and brings new_len[b] more; new_len[b] < 0: it ends.
 *   - Ended requests push their blocks on the stack free_list[0 .. free_count) in their order, and their length becomes 0
 *     (what goes beyond free_cap is dropped).
 *   - Every other request has new_len[b] rows of the batch, in order: q_start[0..B] are their first rows (no row beyond
 *     `rows`).  It takes the blocks that it lacks from the top of the stack into its row of the table.
 *   - Refused is a request whose rows end beyond `rows` (those of refused ones count; also one of no rows behind such), that would need more than max_blocks blocks, or whose
 *     blocks the stack cannot give (then also every later one that needs a block).  It keeps what it has: no new tokens.
 *   seq_len_out    lengths with the new tokens (may be seq_len itself)
 *   free_count_out entries left on the stack (1 int; may be free_count itself)
 *   start          [B] position of the first new token; -1: refused or ended
 *   positions, slots  [rows] of each new token; 0 and -1 for the tokens of refused requests and behind the last row
 *                     (-2 where the table's entry names no block: negative, or of slots beyond 2^31 - 1)
 *   bad            1 int, SET to the number of refused requests and of ended ones whose blocks were dropped
 * table [B][table_stride], max_blocks <= table_stride entries of a row are used.  A seq_len outside 0 .. max_blocks * block
 * is taken as the nearer end.  1 <= B <= BL_KV_MAX_REQUESTS, 1 <= rows <= 2^24, 0 <= free_cap < 2^31 (0: no stack,
 * free_list may be NULL). */
typedef struct {
    int64_t B, rows, table_stride, free_cap;
    int32_t block, max_blocks;
    const int32_t* seq_len;
    const int32_t* new_len;
    const int32_t* free_count;
    int32_t* table;
    int32_t* free_list;
    int32_t* seq_len_out;
    int32_t* free_count_out;
    int32_t* start;
    int32_t* q_start;
    int32_t* positions;
    int32_t* slots;
    int32_t* bad;
} bl_kv_batch;
bl_status bl_kv_tables(const bl_kv_batch* b, bl_stream s);

/* The same with a limit: a request that brings more than max_new tokens (at least 1) is refused too, its rows counted like those of
 * the other refused ones.  For a step whose attention takes max_new as its max_q. */
typedef struct {
    bl_kv_batch batch;
    int64_t max_new;
} bl_kv_limited_batch;
bl_status bl_kv_tables_limited(const bl_kv_limited_batch* b, bl_stream s);

/* The same for requests whose first blocks are another's too (a shared prefix): an ended request gives back the blocks of its row from
 * held[b] on only (held [B]; negative is 0).  Row and length of such a request are set up by its owner: seq_len[b] = held[b] * block where
 * its own tokens begin.  max_new as above; 0: no limit. */
typedef struct {
    bl_kv_batch batch;
    int64_t max_new;
    const int32_t* held;
} bl_kv_held_batch;
bl_status bl_kv_tables_held(const bl_kv_held_batch* b, bl_stream s);

/* New tokens into the cache: row t of the fused projection [Q | K | V] ((n_q + 2 * n_kv) heads, fp32 or bf16), rotary
 * embedding on Q and K (x[i], x[i + d/2] -> x[i]*c - x[i+d/2]*s, x[i+d/2]*c + x[i]*s with c, s = cos, sin[position][i],
 * fp32 [n_pos][head_dim/2]; every operation one rounded fp32 step; cos and sin NULL: no rotation and positions unused),
 * Q to bf16, K and V to codes at slots[t].
 * A block's scale for a head, T = 127 or 448 (e4m3), g the largest |value| of the block's new tokens, NaN passed over:
 *   s = max(g, 1e-5f) * (1.0f / T); where the block holds tokens already (the first new offset is not 0): s = max(s, its old scale);
 *   code = round(clamp(x * (1.0f / s), -T, T)) to the nearest integer or e4m3 value, ties to even;
 *   the codes in front of the first new offset, if s grew: c = round(c * (old scale / s)).
 * The cache holds no NaN: a NaN's code is that of -T.  An infinity makes s infinite, and what reads that block and head is no result.
 * So a block always has the scale of the largest value in it, at the price of one more rounding of what it held
 * each time that a new token raises it.
 * A step's tokens of one block stand in rows as far apart as their slots (consecutive rows, as bl_kv_tables gives them; rows between
 * them may go nowhere), and no block is written by two requests.  slots[t] = -1: K and V of the row go nowhere.  A slot outside the cache or a position
 * outside 0 .. n_pos-1: the same, the Q row of such a position is zeros, and *bad (1 int or NULL) is INCREASED by one.
 *   q_out     bf16 [T][n_q * head_dim] or NULL, rows q_stride values apart
 *   qkv       rows qkv_stride values apart (a multiple of 4 for fp32, 8 for bf16); kind 0 fp32, 1 bf16
 * n_q >= 0, 1 <= T <= 2^24, T * n_q * head_dim at most 2^36; pointers 16-byte aligned (positions, slots, bad: 4), q_stride a multiple of 8. */
enum { BL_KV_FROM_F32 = 0, BL_KV_FROM_BF16 = 1 };
typedef struct {
    bl_kv_cache cache;
    const void* qkv;
    int64_t qkv_stride, q_stride, T, n_pos;
    int32_t qkv_kind, n_q;
    const int32_t* positions;
    const int32_t* slots;
    const float* cos;
    const float* sin;
    uint16_t* q_out;
    int32_t* bad;
} bl_kv_tokens;
bl_status bl_kv_append(const bl_kv_tokens* t, bl_stream s);

/* The same with an RMS norm of every Q and K head in front of the rotation (V is left alone): per row and head
 *   ss = sum_i x[i]^2 with exact fp64 squares and an fp64 sum; r = fp32(1 / sqrt(ss / head_dim + eps)) in fp64; x[i] = (x[i] * r) * gain[i]
 * (gain NULL: no second product), every product one rounded fp32 step.  An infinity or a NaN in a head makes that head's NaN or zeros, and no other's.
 *   q_gain, k_gain  fp32 [head_dim] or NULL, 16-byte aligned, for all heads;  eps > 0 */
typedef struct {
    bl_kv_tokens tokens;
    const float* q_gain;
    const float* k_gain;
    float eps;
} bl_kv_norm_tokens;
bl_status bl_kv_append_norm(const bl_kv_norm_tokens* t, bl_stream s);

/* Causal attention over the cache.  Request b's queries are rows q_start[b] .. q_start[b+1]-1 of q (bf16, n_q heads; query head h reads
 * key/value head h / (n_q / n_kv)); they are its last tokens: query i of n has the position p = seq_len[b] - n + i and sees
 * the tokens 0 .. p (window > 0: p - window + 1 .. p) that are in the cache.
 *   out[row][h] = bf16( sum_j softmax_j( softmax_scale * <q, k_j> ) v_j ),  zeros where nothing is seen.  A NaN or an infinity
 * in q makes its own row and head NaN.
 * Products with K take the codes as they are against q in two 8-bit pieces of 16 bits in all of its largest value (e4m3: two e4m3 pieces, 8 significant bits;
 * int8 with heads of 64 and many queries: q in fp16 times a power of two);
 * softmax weights are rounded to fp16 (11 bits; those below 2^-20 of a row's largest to 2^-30 of it) in front of the product with V; maxima, sums and outputs are held in fp32.
 *   q, out     rows q_stride / out_stride values apart (multiples of 8), 16-byte aligned.  Rows of no request are left alone.
 *   table      [B][table_stride]; an entry outside 0 .. n_blocks-1: its tokens are not seen.  Blocks in front of every query's window
 *              may be another request's, or anyone's
 *   seq_len    taken as the nearer end outside 0 .. max_blocks * block; q_start: ascending, inside 0 .. T
 *   max_q      no request has more queries (the rows of one that has are computed all the same, or are NaN: nothing else is ever left in them)
 *   max_len    about the longest seq_len: sizes the split over a long axis only (0: max_blocks * block)
 *   workspace  bl_attn_workspace_bytes(a) bytes (it depends on the sizes, max_q, max_len and window of the descriptor, not on seq_len), 256-byte aligned; no content is expected
 * One launch on `s`, or two, neither of which waits for the host.  1 <= B <= BL_KV_MAX_REQUESTS, 1 <= T <= 2^24, softmax_scale > 0, n_q a multiple of
 * n_kv; max_blocks * block, T * n_q / n_kv and B * n_kv * max_blocks * block / 64 at most 2^30. */
typedef struct {
    bl_kv_cache cache;
    const uint16_t* q;
    int64_t q_stride, out_stride, table_stride, B, T;
    const int32_t* q_start;
    const int32_t* seq_len;
    const int32_t* table;
    int32_t n_q, max_blocks, max_q, max_len, window;
    float softmax_scale;
    uint16_t* out;
    void* workspace;
} bl_attn_desc;
size_t    bl_attn_workspace_bytes(const bl_attn_desc* a);
bl_status bl_attn_kv8(const bl_attn_desc* a, bl_stream s);

/* The same where requests share long prefixes, each of which is read once for all of its requests.  Request b belongs to the group
 * group[b] (outside 0 .. n_groups-1: to none; a group's requests need not stand together).  The tokens of its first S =
 * shared_blocks[group[b]] blocks (taken as the nearer end outside 0 .. max_shared) are those of row group[b] of shared_table, and its own row of `table` begins with the
 * same ones: either may be read.  Results are bl_attn_kv8's but for the order of the sums: lengths and positions count the prefix, causality and window hold inside it
 * too, a request may be shorter than it.  What shares a read: all requests of less than 128 rows (queries times n_q / n_kv), but where max_q lets one bring 128 or more, those of up to
 * 16 rows; others read the prefix for themselves, and so do all in short contexts.  So max_q is worth giving: with the batch's rows in its place, requests of few queries may share nothing.
 *   shared_table   [n_groups][shared_stride], max_shared <= shared_stride entries of a row are used; its blocks are whole (every token written)
 *   max_own        about the most tokens that a request has behind its shared blocks: sizes a split only (0: as attn.max_len)
 *   attn.workspace bl_attn_shared_workspace_bytes(a) bytes
 * 1 <= n_groups <= BL_KV_MAX_REQUESTS, max_shared >= 1 (max_shared * block at most 2^30), T * n_q * head_dim < 2^34. */
typedef struct {
    bl_attn_desc attn;
    const int32_t* group;
    const int32_t* shared_blocks;
    const int32_t* shared_table;
    int64_t shared_stride, n_groups;
    int32_t max_shared, max_own;
} bl_attn_shared_desc;
size_t    bl_attn_shared_workspace_bytes(const bl_attn_shared_desc* a);
bl_status bl_attn_kv8_shared(const bl_attn_shared_desc* a, bl_stream s);

/* A MATRIX OF 8-BIT FLOATING POINT CODES (OCP e4m3) with a scale for each block of 128 x 128: what a model keeps that is not ternary, its
 * vocabulary above all.  Weight [n][k] stands for codes[n * stride + k] * scale[n / 128 * scale_stride + k / 128] (blocks at the edges are cut off).
 * K % 64 == 0; stride, bytes from a row to the next, a multiple of 16; codes 16-byte aligned. */
typedef struct {
    const uint8_t* codes;
    const float* scale;
    int64_t N, K, stride, scale_stride;
} bl_f8_matrix;
enum { BL_F8_OUT_F32 = 0, BL_F8_OUT_BF16 = 1 };

/* Product with it, M >= 1 rows.  The rows X[m][k] are the bf16 values of a producer (norm included, as for the BitLinears); each group of 128
 * consecutive k of a row gets a scale of its own:
 *   g = max |X| of the group; s = max(g, 1e-5f) * (1.0f / 448.0f); code = e4m3(X * (1.0f / s)), every step one rounded fp32
 *   operation, ties to even;
 *   y[m][n] = sum over the groups b of (s[m][b] * scale[n / 128][b]) * sum_k code[m][k] * codes[n][k], in fp32, then to the output's type.
 * A row with a NaN or an infinity in it is NaN.  The norm's sum of squares has one order per kernel: up to 16 rows of up to 1024 values are made in the product's own, whose order is another
 * than the other producers'; r is the same but for a row in about 10^8.
 *   y          fp32 or bf16 [M][N], rows y_stride values apart, aligned to its type
 *   workspace  bl_f8_workspace_bytes(p) bytes, 256-byte aligned; no content is expected
 * y, the workspace and a producer's aux_out share no byte with each other or with what is read (BL_ERR_VALUE): a sum is not stored in place.
 * M < 2^24, N and K <= 2^24, and (M / 128) * (N / 128) < 2^24, both rounded up. */
typedef struct {
    bl_f8_matrix w;
    bl_producer prod;
    int64_t M, y_stride;
    void* y;
    int32_t y_kind;
    void* workspace;
} bl_f8_product;
size_t    bl_f8_workspace_bytes(const bl_f8_product* p);
bl_status bl_f8_linear(const bl_f8_product* p, bl_stream s);

/* Rows of it: out[t][k] = (codes[ids[t]][k] * scale) * multiplier, each one rounded fp32 step, then to the output's type.  An id outside
 * 0 .. N-1: zeros, and *bad (1 int or NULL) is INCREASED by one, but for -1 (no token).
 *   out  fp32 or bf16 [T][K], rows out_stride values apart, 16-byte aligned.  1 <= T <= 2^24. */
typedef struct {
    bl_f8_matrix w;
    const int32_t* ids;
    int64_t T, out_stride;
    void* out;
    int32_t out_kind;
    float multiplier;
    int32_t* bad;
} bl_f8_lookup;
bl_status bl_f8_embed(const bl_f8_lookup* l, bl_stream s);

/* Test hook: which decode kernel the M <= 64 entry points take, so that tests can put every
 * kernel through every case.  0 = the measured default, 1 = the dot4 kernel where it applies
 * (M <= 4), 2 = the row-resident matrix-core kernel, 3 = the streaming panel kernel where it
 * applies (int8 inputs).  Process-wide and atomic; results never depend on it, only the route.
 * BL_ERR_VALUE outside 0..3. */
bl_status bl_debug_force_path(int path);

/* Measurement aids (not part of the product path): the achievable roofs the kernels are
 * priced against beside the datasheet peaks.
 *   bl_probe_stream_read  one launch that reads `bytes` (a multiple of 16) of device memory
 *                         at `buf` with 128-bit loads and does nothing else; time it over a
 *                         buffer much larger than the caches to get the streaming-read rate.
 *                         workgroups_per_cu: 256-thread workgroups per compute unit, 1..8
 *                         (0 = 8, the fastest); 2 is the occupancy of the streaming decode.
 *   bl_probe_stream_write one launch that fills a row-major fp32 matrix [rows][cols] (device, both
 *                         multiples of 128) with the store pattern of the prefill epilogue (128 x 128
 *                         tiles, dword stores of 32 consecutive floats per row, non-temporal) and
 *                         does nothing else: the rate at which the outputs of a prefill launch can be
 *                         written when every workgroup stores at once.  workgroups_per_cu 1..8
 *                         (0 = 3).
 *   bl_probe_mfma_i8      one launch of `iters` x 4 back-to-back v_mfma_i32_32x32x32_i8 per
 *                         wave, operands in registers; *ops (HOST, optional) receives the
 *                         integer operations of the launch (2 per multiply-accumulate).
 *   bl_probe_mfma_i8_ex   the same loop with its operands read once from `operands` (device,
 *                         64 KiB of int8, or NULL for the constants of bl_probe_mfma_i8): with
 *                         random operands the loop draws more power and the chip runs it at a
 *                         lower clock, which is the rate a real contraction can hope for.
 *                         stamps (device, 2 x int64, or NULL) receives what workgroup 0 counted
 *                         between its first and last instruction: [0] shader clocks, [1] ticks of
 *                         the constant-rate wall clock (bl_probe_wall_clock_khz), so
 *                         stamps[0] / stamps[1] x that rate is the clock the kernel ran at.
 *   bl_probe_wall_clock_khz  rate of that wall clock in kHz (0 on error).  Host-only query.
 *   bl_debug_clock_stamps  measurement hook for the prefill kernels: while a device buffer
 *                         of 2 x int64 is registered, every product launch of bl_gemm_w158a8 and
 *                         its variants leaves the same two counts of its workgroup 0 there; NULL (the default) switches it off.
 *                         Process-wide and atomic; results never depend on it.
 * sink: device, 64 int32, never written in practice (it keeps the work observable). */
bl_status bl_probe_stream_read(const void* buf, size_t bytes, int workgroups_per_cu, int32_t* sink,
                               bl_stream s);
bl_status bl_probe_stream_write(float* buf, int64_t rows, int64_t cols, int workgroups_per_cu, bl_stream s);
bl_status bl_probe_mfma_i8(int iters, int32_t* sink, double* ops, bl_stream s);
bl_status bl_probe_mfma_i8_ex(int iters, const void* operands, int64_t* stamps, int32_t* sink, double* ops /* HOST */,
                              bl_stream s);
int       bl_probe_wall_clock_khz(void);
bl_status bl_debug_clock_stamps(int64_t* stamps);

#ifdef __cplusplus
}
#endif
#endif /* BITLINEAR_H */
