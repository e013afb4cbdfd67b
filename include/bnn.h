/*
 * bnn.h - C ABI of the MI355X (gfx950) library for the forward hot path of
 * Binarized Neural Networks (Courbariaux, Hubara, Soudry, El-Yaniv, Bengio).
 *
 * The path is the hidden-layer loop of Alg. 4 ("Running a BNN"):
 *     a_k   = XnorDotProduct(a^b_{k-1}, W^b_k)
 *     a^b_k = Sign(BatchNorm(a_k, theta_k))
 * on +-1 values concatenated 32 per 32-bit word (Sec. 4, Eq. (5)).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Packed rows: bit = 1 <=> +1, bit = 0 <=> -1.  Element k of a row lives in
 *    word k / 32 at bit k % 32 (least significant bit first).  A row of K
 *    elements occupies bnn_words_per_row(K) words; the unused high bits of its
 *    last word ("pad bits") are written as 0 by this library, and are ignored
 *    (masked) wherever this library reads packed operands.
 *  - Matrices are row-major with a leading dimension ("ld", counted in
 *    elements of the array's own type: floats, words, int32 or bytes).
 *  - Unless an argument is marked HOST, every pointer is a DEVICE pointer on
 *    the current HIP device, owned by the caller.  The library allocates
 *    nothing, keeps no pointer after returning, and never synchronises: work
 *    is enqueued on `stream` (a hipStream_t passed as void*; NULL = the
 *    default stream) and the caller orders it against its own work.
 *  - Inputs and outputs must not overlap.
 *  - Every function returns a bnn_status.  On any status other than BNN_OK no
 *    kernel was launched and no output was written.  A dimension of 0 for
 *    rows/M/N/B is a valid empty problem: BNN_OK, nothing launched.
 *  - Limits: every dimension < 2^31; K <= 2^31 - 32 for every product, so that
 *    |dot| <= K, the threshold K + 1 and the word count (K + 31) / 32 stay inside
 *    32-bit arithmetic (bnn_bn_fold alone accepts a range up to 2^31 - 2).
 */
#ifndef BNN_H
#define BNN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BNN_VERSION 100 /* 0.1.0 */

typedef enum bnn_status {
    BNN_OK = 0,
    BNN_ERR_INVALID_ARG = 1, /* null pointer, negative size, ld too small, K out of range */
    BNN_ERR_ALIGNMENT = 2,   /* pointer not aligned to its element type */
    BNN_ERR_UNSUPPORTED = 3, /* valid request this build has no kernel for */
    BNN_ERR_LAUNCH = 4       /* the HIP runtime refused the launch */
} bnn_status;

int bnn_version(void);
const char *bnn_status_string(int status);

/* ceil(K / 32): words in a packed row of K elements (Sec. 4: 32 binary
 * variables per 32-bit register).  Returns -1 if K < 0. */
int64_t bnn_words_per_row(int64_t K);

/*
 * Eq. (1) + Sec. 4 packing:  out[r][k/32] bit (k%32) = (x[r][k] >= 0).
 * The comparison is the IEEE one: +0.0, -0.0 -> 1; negative subnormals -> 0;
 * NaN -> 0.
 *   x     [rows][ld_x] float32, ld_x >= cols
 *   out   [rows][ld_out] uint32, ld_out >= ceil(cols/32); words
 *         [ceil(cols/32), ld_out) of each row are left untouched
 * Any alignment of x (4 bytes or more) and any ld_x take 16-byte loads; rows that are
 * whole numbers of 128 elements, 16-byte aligned, also leave in 16-byte stores.
 */
int bnn_pack_sign(const float *x, int64_t rows, int64_t cols, int64_t ld_x,
                  uint32_t *out, int64_t ld_out, void *stream);

/*
 * Sec. 4, Eq. (5) over whole matrices (the XnorDotProduct of Alg. 4):
 *   C[m][n] = sum_{k<K} a[m][k] * b[n][k],  a, b in {-1,+1}
 *           = 2 * popcount(xnor(A[m], B[n]) over the K valid bits) - K
 * computed as K - 2 * sum_w popcount(A[m][w] ^ B[n][w]) with the pad bits of
 * both operands masked off, so their content never matters.
 *   A  [M][lda] packed rows of K bits (activations a^b)
 *   B  [N][ldb] packed rows of K bits: row n is output unit n's weight vector,
 *      i.e. B is the transpose of W^b in s = a W (both operands K-contiguous)
 *   C  [M][ldc] int32, ldc >= N
 * lda, ldb >= ceil(K/32).  Any 4-byte alignment of A, B and any lda, ldb run on the matrix
 * engine; the whole-tile forms of the largest products (kernel ids 8 and 9 below and the
 * int32 form of 5) ask for 16-byte aligned rows.
 * K == 0 writes C = 0.
 */
int bnn_xnor_gemm(const uint32_t *A, int64_t lda, const uint32_t *B, int64_t ldb,
                  int32_t *C, int64_t ldc, int64_t M, int64_t N, int64_t K,
                  void *stream);

/* Same contract, with the kernel chosen by the caller (for tests and
 * profiling): 0 = automatic (what bnn_xnor_gemm does), 1 = one thread per
 * output, 2 = 128x128 LDS-tiled register-blocked XNOR-popcount kernel,
 * 3 = K-split kernel with wavefront reduction (skinny outputs), 4 = 64x64
 * tiled XNOR-popcount kernel, 5 = bits-in / matrix-engine-inside kernel (bits
 * widened to 4-bit floats in registers, MFMA, 256x128 tiles; needs
 * K <= 2^24, else BNN_ERR_UNSUPPORTED), 6 = the same with 128x128 tiles (of
 * 64x128 on small grids; K <= 96 takes these two sizes by either id),
 * 7 = the same arithmetic organised for short K (a workgroup keeps its 128
 * columns of B in LDS and walks over several 128-row tiles of A; needs
 * 96 < K <= 1152, A and B 16-byte aligned, lda and ldb multiples of 4, else
 * BNN_ERR_UNSUPPORTED), 8 = kernel 5 as a tile walk (one workgroup per
 * resident slot walks over several 256x128 tiles, fetching the next tile's
 * first operands under the current tile's last products; needs more tiles
 * than slots, K a multiple of 512 with 1024 <= K <= 2^24, N a multiple of
 * 128, M >= 256, A and B 16-byte aligned, lda and ldb multiples of 4 below
 * 2^22, else BNN_ERR_UNSUPPORTED; what 0 picks when the last round of tiles
 * would fill only part of the chip), 9 = a kernel of the fused product
 * only (BNN_ERR_UNSUPPORTED here), 10 = the arithmetic of kernel 5 on 32x32
 * output tiles with K split over the four wavefronts of a workgroup and the
 * operands read from memory straight into the MFMA's registers (for small
 * outputs with a long K, such as fully connected layers at batch 256; needs
 * K a positive multiple of 128 up to 2^24, A and B 16-byte aligned, lda and
 * ldb multiples of 4, else BNN_ERR_UNSUPPORTED; what 0 picks, for any
 * alignment and 96 < K <= 2^24, for outputs of at most 512 such tiles or at
 * most 1024 with K >= 512, as it picks 7 for any alignment).  Unknown ids give BNN_ERR_INVALID_ARG. */
int bnn_xnor_gemm_kernel(const uint32_t *A, int64_t lda, const uint32_t *B, int64_t ldb,
                         int32_t *C, int64_t ldc, int64_t M, int64_t N, int64_t K,
                         int kernel_id, void *stream);

/*
 * HOST function.  Folds Sign(BatchNorm(s)) of Alg. 4 (inference BatchNorm with
 * running statistics, evaluated in float32 as
 *     y = gamma * ((float(s) - mean) * (1 / sqrt(var + eps))) + beta,
 * every operation rounded separately) into one integer compare per channel:
 *     Sign(y(s)) = +1  <=>  (s >= thr[n]) XOR flip[n]     for all integer s in [-K, K].
 * The threshold is found by searching the float expression itself (which is
 * monotone in s), not by solving it algebraically, so the equivalence is exact
 * at rounding boundaries.  gamma < 0 reverses the inequality (flip = 1);
 * gamma == 0 gives a constant bit (thr = -K or K + 1).
 *   gamma, beta, mean, var  HOST [N] float32; all finite, var + eps > 0
 *   thr        HOST [N] int32, each in [-K, K + 1]
 *   flip_bits  HOST [ceil(N/32)] uint32, channel n at word n/32 bit n%32, pad bits 0
 * Non-finite parameters or var + eps <= 0 give BNN_ERR_INVALID_ARG.
 */
int bnn_bn_fold(const float *gamma, const float *beta, const float *mean,
                const float *var, float eps, int64_t N, int64_t K, int32_t *thr,
                uint32_t *flip_bits);

/*
 * Alg. 4, a^b_k = Sign(BatchNorm(a_k, theta_k)), on folded parameters, packed
 * for the next layer:
 *   out[m][n/32] bit (n%32) = (C[m][n] >= thr[n]) XOR flip[n]
 *   C    [M][ldc] int32, ldc >= N
 *   thr  [N] int32 (device), flip_bits [ceil(N/32)] uint32 (device), from bnn_bn_fold
 *        (any int32 is a valid threshold; pad bits of the last flip word must be 0)
 *   out  [M][ld_out] uint32, ld_out >= ceil(N/32); pad bits of the last word 0;
 *        words beyond ceil(N/32) untouched
 * Any alignment of C and thr (4 bytes or more) and any ldc take 16-byte loads; rows that are
 * whole numbers of 128 channels, 16-byte aligned, also leave in 16-byte stores.
 */
int bnn_bn_sign_pack(const int32_t *C, int64_t ldc, int64_t M, int64_t N,
                     const int32_t *thr, const uint32_t *flip_bits, uint32_t *out,
                     int64_t ld_out, void *stream);

/*
 * One hidden layer of Alg. 4 in a single launch:
 *     a_k   = XnorDotProduct(a^b_{k-1}, W^b_k)
 *     a^b_k = Sign(BatchNorm(a_k, theta_k))
 * i.e. bnn_xnor_gemm followed by bnn_bn_sign_pack with the int32
 * pre-activations kept in registers (they never reach memory):
 *   out[m][n/32] bit (n%32) = (C[m][n] >= thr[n]) XOR flip[n],
 *   C[m][n] = K - 2 * sum_w popcount(A[m][w] ^ B[n][w]).
 * Arguments as in those two calls (A [M][lda], B [N][ldb] packed rows of K bits;
 * thr [N], flip_bits [ceil(N/32)] device arrays from bnn_bn_fold;
 * out [M][ld_out], ld_out >= ceil(N/32), pad bits 0, words beyond untouched).
 * The result is bit-identical to the two-call sequence for every int32 threshold.
 */
int bnn_xnor_gemm_bn_sign_pack(const uint32_t *A, int64_t lda, const uint32_t *B, int64_t ldb,
                               int64_t M, int64_t N, int64_t K, const int32_t *thr,
                               const uint32_t *flip_bits, uint32_t *out, int64_t ld_out,
                               void *stream);

/*
 * The first hidden layer on real inputs, bnn_pack_sign(x -> a_bits) followed by
 * bnn_xnor_gemm_bn_sign_pack(a_bits, B -> out), in one launch where that is faster
 * (small batches, K <= 1024), else in two.  Same arguments, results and status as
 * those calls; x [M][ldx] float32, ldx >= K; a_bits [M][ld_a] receives the packed input.
 * Two launches also where out reaches into x, or a_bits into B, thr or flip_bits.
 */
int bnn_sign_gemm_bn_sign_pack(const float *x, int64_t ldx, const uint32_t *B, int64_t ldb,
                               int64_t M, int64_t N, int64_t K, const int32_t *thr,
                               const uint32_t *flip_bits, uint32_t *a_bits, int64_t ld_a,
                               uint32_t *out, int64_t ld_out, void *stream);

/* bnn_xnor_gemm_bn_sign_pack with the kernel chosen by the caller: 0 = automatic, 2, 4, 5, 6, 7, 8 as
 * in bnn_xnor_gemm_kernel (the other kernels have no fused form), 9 = the arithmetic of
 * kernel 5 on 256x256 tiles with one wavefront per SIMD and one workgroup per compute
 * unit, which takes a strip of rows of one 256-column tile as 256-row tiles and at most
 * one 128-row tile (needs K a multiple of 512 with 2048 <= K <= 2^19, N a multiple of
 * 256 whose tile count N/256 divides the compute units, M / (compute units / (N/256))
 * >= 256, A and B 16-byte aligned, lda and ldb multiples of 4 below 2^22, out 8-byte
 * aligned, ld_out even, else BNN_ERR_UNSUPPORTED; what 0 picks for such products when
 * a strip has at least 512 rows or exactly 256), 10 as in bnn_xnor_gemm_kernel. */
int bnn_xnor_gemm_bn_sign_pack_kernel(const uint32_t *A, int64_t lda, const uint32_t *B, int64_t ldb,
                                      int64_t M, int64_t N, int64_t K, const int32_t *thr,
                                      const uint32_t *flip_bits, uint32_t *out, int64_t ld_out,
                                      int kernel_id, void *stream);

/*
 * First layer on 8-bit fixed-point inputs (Sec. 1.6; Alg. 4 step 1):
 *     a_1 = sum_{n=1..8} 2^(n-1) * <a_0^n, W^b_1>,   a_0^n in {0,1} the n-th bit plane.
 *
 * bnn_pack_bitplanes splits uint8 inputs into packed bit planes:
 *   out[r][8*w + p] bit j = bit p (p = 0 least significant, the paper's n = p+1) of x[r][32*w + j]
 *   x   [rows][ld_x] uint8, ld_x >= cols
 *   out [rows][ld_out] uint32, ld_out >= 8*ceil(cols/32); elements >= cols read as 0; words beyond
 *       8*ceil(cols/32) untouched.  Any alignment of x and ld_x takes the same path.
 *
 * bnn_bitplane_gemm:  C[m][n] = sum_k x[m][k] * w[n][k],  x in [0,255] given as bit planes (layout
 *   above, Xp [M][ldx], ldx >= 8*ceil(K/32)), w in {-1,+1} given as packed rows B [N][ldb] as in
 *   bnn_xnor_gemm; C [M][ldc] int32.  The planes are turned back into bytes on chip and multiplied on the
 *   int8 matrix engine with int32 accumulation, exact for every K taken.  255*K must fit int32
 *   (255*K <= 2^31 - 32), else BNN_ERR_INVALID_ARG.  Pad bits of the last K-word of either operand
 *   are ignored.
 *
 * bnn_bitplane_gemm_bn_sign_pack: the same product followed by Sign(BatchNorm(a_1, theta_1)) on
 *   folded thresholds (bnn_bn_fold with 255*K as the range argument), written as packed bits:
 *   out[m][n/32] bit (n%32) = (C[m][n] >= thr[n]) XOR flip[n]; out as in bnn_bn_sign_pack.
 */
int bnn_pack_bitplanes(const uint8_t *x, int64_t rows, int64_t cols, int64_t ld_x,
                       uint32_t *out, int64_t ld_out, void *stream);
int bnn_bitplane_gemm(const uint32_t *Xp, int64_t ldx, const uint32_t *B, int64_t ldb,
                      int32_t *C, int64_t ldc, int64_t M, int64_t N, int64_t K, void *stream);
int bnn_bitplane_gemm_bn_sign_pack(const uint32_t *Xp, int64_t ldx, const uint32_t *B, int64_t ldb,
                                   int64_t M, int64_t N, int64_t K, const int32_t *thr,
                                   const uint32_t *flip_bits, uint32_t *out, int64_t ld_out,
                                   void *stream);

/*
 * Lowers a binary kh x kw convolution (3 x 3 in the paper's nets, Sec. 3.3) to
 * the matrix product above: row m = (b*Ho + oy)*Wo + ox of `out` holds the
 * receptive field of output pixel (b, oy, ox) as K = kh*kw*Cin bits,
 *   bit (ky*kw + kx)*Cin + ci = in(b, oy*stride + ky - pad, ox*stride + kx - pad, ci),
 * and taps that fall outside the image read as +1 (bit 1): zero padding
 * binarised by Eq. (1), Sign(0) = +1.  Ho = (H + 2*pad - kh)/stride + 1, same for Wo.
 *   in   packed NHWC [B][H][W][ceil(Cin/32)] uint32 (pad bits ignored)
 *   out  [B*Ho*Wo][ld_out] uint32, ld_out >= ceil(kh*kw*Cin/32); pad bits 0
 * Weights for the product are [Cout][kh][kw][Cin] packed along (ky,kx,ci).
 * Cin % 32 == 0 copies whole words; other Cin take a bit-gather path.
 * Requires kh, kw, stride >= 1, pad >= 0 and Ho, Wo >= 1.
 */
int bnn_conv_im2col_pack(const uint32_t *in, int64_t B, int64_t H, int64_t W,
                         int64_t Cin, int kh, int kw, int stride, int pad,
                         uint32_t *out, int64_t ld_out, void *stream);

/*
 * A whole binary convolution layer without the intermediate matrix (implicit GEMM): the
 * receptive fields described under bnn_conv_im2col_pack are taken straight from the packed NHWC
 * input - from a patch of it held on chip where that fits and is faster, gathered by the
 * product's tile loader otherwise.
 *   S[(b*Ho + oy)*Wo + ox][co] = sum_{ky,kx,ci} in(b, oy*stride+ky-pad, ox*stride+kx-pad, ci) * Wt[co][ky][kx][ci]
 *   in   packed NHWC [B][H][W][Cin/32] uint32, out-of-image taps read as +1
 *   Wb   packed filters [Cout][ldw], row co = Wt[co] flattened as (ky, kx, ci), ldw >= kh*kw*Cin/32
 *   bnn_conv_xnor:          S [B*Ho*Wo][lds] int32, lds >= Cout
 *   bnn_conv_bn_sign_pack:  out [B*Ho*Wo][ld_out] packed bits = (S >= thr[co]) XOR flip[co]
 *                           (= packed NHWC input of the next layer), thr/flip from bnn_bn_fold
 * Bit-identical to bnn_conv_im2col_pack followed by bnn_xnor_gemm (and bnn_bn_sign_pack).
 * Receptive fields of more than 2^24 bits (beyond the matrix engine's exact range) take a slow, exact
 * xor/popcount kernel for any geometry with Cin % 32 == 0.
 * Requires H, W, pad, Ho, Wo <= 32767, an input of fewer than 2^32 words, and either
 *   Cin % 128 == 0 with `in` 16-byte aligned (any kh, kw, stride, pad), or
 *   Cin % 32 == 0 on a same-size stride-1 layer (kh = kw = 2*pad + 1) whose image rows fit the kernel's
 *   128-pixel tiles (W divides 128; H a multiple of 128/W or the reverse), with kh*kw*Cin <= 2560 and
 *   Wb 16-byte aligned, ldw % 4 == 0 (e.g. the 64-channel 3 x 3 layers of the half-width net of Sec. 2.3);
 * otherwise BNN_ERR_UNSUPPORTED (use the im2col path).
 */
int bnn_conv_xnor(const uint32_t *in, int64_t B, int64_t H, int64_t W, int64_t Cin,
                  const uint32_t *Wb, int64_t ldw, int64_t Cout, int kh, int kw, int stride, int pad,
                  int32_t *S, int64_t lds, void *stream);
int bnn_conv_bn_sign_pack(const uint32_t *in, int64_t B, int64_t H, int64_t W, int64_t Cin,
                          const uint32_t *Wb, int64_t ldw, int64_t Cout, int kh, int kw, int stride,
                          int pad, const int32_t *thr, const uint32_t *flip_bits, uint32_t *out,
                          int64_t ld_out, void *stream);

/*
 * The pooled layer of the paper's ConvNets in one launch: convolution, pool x pool max pooling
 * (stride pool) of the pre-activations, BatchNorm, Sign (Alg. 4 for the last two).  Sec. 2.2 only says
 * that its ConvNet has the architecture of the BinaryConnect network it cites; that pooling sits between
 * a convolution and its BatchNorm is this library's reading of that cited architecture, not a statement
 * the paper prints.
 *   out [B*(Ho/pool)*(Wo/pool)][ld_out] packed bits, the packed NHWC input of the next layer;
 *   every other argument as in bnn_conv_bn_sign_pack.
 * Bit-identical to bnn_conv_bn_sign_pack followed by bnn_maxpool_bits (see there for why pooling
 * the output bits equals pooling the pre-activations).  Only pool = 2 on same-size stride-1
 * convolutions whose tiles hold whole, even numbers of image rows is taken (even H and W; W a power
 * of two up to 16, or 32 or 64; the requirements of bnn_conv_bn_sign_pack); anything else returns
 * BNN_ERR_UNSUPPORTED before any launch: use the two calls then.
 */
int bnn_conv_pool_bn_sign_pack(const uint32_t *in, int64_t B, int64_t H, int64_t W, int64_t Cin,
                               const uint32_t *Wb, int64_t ldw, int64_t Cout, int kh, int kw, int stride,
                               int pad, int pool, const int32_t *thr, const uint32_t *flip_bits,
                               uint32_t *out, int64_t ld_out, void *stream);

/*
 * The same pooled layer on any map: pool = 2, even Ho and Wo, any window, stride and padding, Cin a multiple of 128, Wb 16-byte
 * aligned with ldw % 4 == 0, and an input patch that fits the compute unit's local memory.  Anything else returns
 * BNN_ERR_UNSUPPORTED before any launch.  Not every layer that it takes is faster in one launch: see bnn_conv_pool_form.
 */
int bnn_conv_pool_windows_bn_sign_pack(const uint32_t *in, int64_t B, int64_t H, int64_t W, int64_t Cin,
                                       const uint32_t *Wb, int64_t ldw, int64_t Cout, int kh, int kw, int stride,
                                       int pad, int pool, const int32_t *thr, const uint32_t *flip_bits,
                                       uint32_t *out, int64_t ld_out, void *stream);

/*
 * The fastest form of a pooled layer whose input and filters are 16-byte aligned (ldw % 4 == 0).  Host only: nothing is launched.
 * BNN_POOL_IN_CONV, BNN_POOL_WINDOWS: bnn_conv_pool_bn_sign_pack, bnn_conv_pool_windows_bn_sign_pack;
 * BNN_POOL_APART: neither takes it, or bnn_conv_bn_sign_pack followed by bnn_maxpool_bits is faster.
 */
#define BNN_POOL_APART 0
#define BNN_POOL_IN_CONV 1
#define BNN_POOL_WINDOWS 2
int bnn_conv_pool_form(int64_t B, int64_t H, int64_t W, int64_t Cin, int64_t Cout, int kh, int kw, int stride, int pad, int pool);

/*
 * Max pooling for binarized layers.  In the architecture Sec. 2.2 refers to (the cited BinaryConnect
 * ConvNet, as this library reads it) the pre-activations are pooled between a convolution and its
 * BatchNorm + Sign; since Sign(BatchNorm(.)) is monotone per channel, the bit
 * of the pooled pre-activation is the OR of the window's bits where the channel's folded flip
 * bit is 0 and their AND where it is 1, so pooling runs on the packed output of the fused layer:
 *   out[b][py][px][c] = OR / AND over dy < ph, dx < pw of in[b][py*stride+dy][px*stride+dx][c]
 *   in  packed NHWC [B][H][W][ceil(C/32)], out packed NHWC [B][Hp][Wp][ceil(C/32)],
 *   Hp = (H - ph)/stride + 1, Wp = (W - pw)/stride + 1 (no padding)
 *   flip_bits [ceil(C/32)] device words from bnn_bn_fold, or NULL for OR on every channel.
 * Pad bits of `in` pass through the same operations (zero stays zero under OR).
 */
int bnn_maxpool_bits(const uint32_t *in, int64_t B, int64_t H, int64_t W, int64_t C, int ph, int pw,
                     int stride, const uint32_t *flip_bits, uint32_t *out, void *stream);

/*
 * The competing dense-engine variant of the same product (the role the vendor
 * GEMM plays in Sec. 4 / Fig. 3): +-1 stored one per int8, multiplied on the
 * int8 MFMA units with int32 accumulation.
 *   C[m][n] = sum_k A[m][k] * B[n][k]
 *   A [M][lda] int8, B [N][ldb] int8 (row n = weights of output n), C [M][ldc] int32
 * Exact for any int8 contents with |sum| < 2^31.  Requires A, B 16-byte
 * aligned and lda, ldb multiples of 16 (else BNN_ERR_ALIGNMENT); K need not be.
 */
int bnn_gemm_i8_mfma(const int8_t *A, int64_t lda, const int8_t *B, int64_t ldb,
                     int32_t *C, int64_t ldc, int64_t M, int64_t N, int64_t K,
                     void *stream);

/* Expands packed rows to one int8 (+1 / -1) per element, the operand format of
 * bnn_gemm_i8_mfma: out[r][k] = bit k of in[r] ? +1 : -1 for k < K, and 0 for
 * K <= k < ld_out (so padded columns add nothing to a product).
 *   in [rows][ld_in] uint32, out [rows][ld_out] int8, ld_out >= K.
 * out is written four bytes at a time: it must be 4-byte aligned and ld_out a
 * multiple of 4, else BNN_ERR_ALIGNMENT (bnn_gemm_i8_mfma wants 16 for both anyway). */
int bnn_unpack_i8(const uint32_t *in, int64_t ld_in, int64_t rows, int64_t K,
                  int8_t *out, int64_t ld_out, void *stream);

/* ---- real activations, packed weights: the feed-forward block of a language model with one-bit weights --------------
 *
 * Activations are real matrices of one of three types; weights are packed rows as everywhere in this file (bit 1 = +1),
 * each output channel with an optional real scale.  Sums, statistics and activations are held in float32; a result is
 * rounded once, when it is written.  Rows may start at any address that is a multiple of the element, and a leading
 * dimension is any count of elements from the row's length on.  Vectors (scale, bias, gamma, beta and their gradients)
 * are contiguous float32.
 */
typedef enum bnn_type { BNN_BF16 = 0, BNN_F16 = 1, BNN_F32 = 2 } bnn_type;

typedef enum bnn_act {
    BNN_ACT_NONE = 0,
    BNN_ACT_RELU = 1,      /* max(z, 0); derivative at 0: 0 */
    BNN_ACT_SILU = 2,      /* z / (1 + e^-z) */
    BNN_ACT_GELU = 3,      /* z/2 (1 + erf(z / sqrt 2)) */
    BNN_ACT_GELU_TANH = 4, /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
    BNN_ACT_SIGMOID = 5    /* 1 / (1 + e^-z) */
} bnn_act;

typedef enum bnn_norm {
    BNN_NORM_NONE = 0,     /* v */
    BNN_NORM_RMS = 1,      /* v / sqrt(mean(v^2) + eps) * gamma */
    BNN_NORM_LAYER = 2     /* (v - mean(v)) / sqrt(var(v) + eps) * gamma + beta */
} bnn_norm;

/*
 * A product with its epilogue, one launch:
 *   y[m][n] = act(scale[n] * sum_{k<K} x[m][k] w[n][k] + bias[n]) + residual[m][n]
 *   x [M][ld_x], residual [M][ld_r] (or NULL), y [M][ld_y] of `type`; w [N][ld_w] packed rows of K bits;
 *   scale, bias [N] or NULL (1 and 0).
 * y may be residual itself (same address and leading dimension); nothing else may overlap.  K == 0 is a sum of nothing.
 */
int bnn_linear_bits(int type, const void *x, int64_t ld_x, const uint32_t *w, int64_t ld_w, const float *scale,
                    const float *bias, int act, const void *residual, int64_t ld_r, void *y, int64_t ld_y,
                    int64_t M, int64_t N, int64_t K, void *stream);

/*
 * The gated feed-forward's first half, one launch: both projections, the activation and their product,
 *   h[m][f] = act(z[m][f]) * z[m][F + f],   z = scale * (x w^T) + bias
 *   w [2F][ld_w]: the F rows of the gate, then the F rows of the other projection; scale, bias [2F] or NULL;
 *   h [M][ld_h].
 */
int bnn_gated_bits(int type, const void *x, int64_t ld_x, const uint32_t *w, int64_t ld_w, const float *scale,
                   const float *bias, int act, void *h, int64_t ld_h, int64_t M, int64_t F, int64_t K, void *stream);

/*
 * Backward passes.  With s = x w^T, z = scale * s + bias and dz the gradient of z:
 *   linear:  dz = dy * act'(z)
 *   gated:   dz[m][f] = dh * z[m][F + f] * act'(z[m][f]),   dz[m][F + f] = dh * act(z[m][f])
 *   dx = (dz * scale) w          [M][ld_dx] of `type`
 *   dw = (dz * scale)^T x        [N][ld_dw] of `type`: the gradient of the weights as if they were real, which a
 *                                straight-through estimator hands to the values that were binarized (Alg. 1, the
 *                                backward propagation's g_W)
 *   dscale[n] = sum_m dz s,  dbias[n] = sum_m dz     float32
 * (dresidual is dy.)  Any of dx, dw, dscale, dbias may be NULL: not wanted.  dz * scale is rounded to `type` before the two
 * products that read it (float16: times a power of two, from the largest finite magnitudes of the operands, that keeps it
 * among the normal numbers, and that both products' sums are divided by).  Sums over rows are made in an order that depends on the sizes alone.
 * workspace: 16-byte aligned device memory of at least the bytes that the _workspace function returns for the same sizes
 * (-1 for sizes or a type that the call would refuse); what it holds before and after means nothing.
 */
int64_t bnn_linear_bits_backward_workspace(int type, int64_t M, int64_t N, int64_t K, int act);
int bnn_linear_bits_backward(int type, const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const uint32_t *w,
                             int64_t ld_w, const float *scale, const float *bias, int act, void *dx, int64_t ld_dx,
                             void *dw, int64_t ld_dw, float *dscale, float *dbias, int64_t M, int64_t N, int64_t K,
                             void *workspace, int64_t workspace_bytes, void *stream);
int64_t bnn_gated_bits_backward_workspace(int type, int64_t M, int64_t F, int64_t K, int act);
int bnn_gated_bits_backward(int type, const void *dh, int64_t ld_dh, const void *x, int64_t ld_x, const uint32_t *w,
                            int64_t ld_w, const float *scale, const float *bias, int act, void *dx, int64_t ld_dx,
                            void *dw, int64_t ld_dw, float *dscale, float *dbias, int64_t M, int64_t F, int64_t K,
                            void *workspace, int64_t workspace_bytes, void *stream);

/*
 * What stands between two blocks, one launch: the norm after a block, its gate and residual scale, the sum with the
 * stream, and the norm before the next block,
 *   t = post(y),   r[m] = x[m] + res_scale * gate[m / rows_per_gate] * t[m],   n = pre(r)
 *   y, x (or NULL: 0), r, n [M][ld] of `type`, rows of D; gate [ceil(M / rows_per_gate)][ld_gate] of `type` or NULL (1);
 *   post, pre: bnn_norm, with gamma [D] or NULL (1) and beta [D] or NULL (0; only with BNN_NORM_LAYER).
 * r may be NULL (not wanted) or x itself (same address and leading dimension); n must be NULL exactly if pre is
 * BNN_NORM_NONE.  n is taken of the unrounded r.  rows_per_gate >= 1 also where gate is NULL.  Rows longer than 16384
 * elements are BNN_ERR_UNSUPPORTED, here and backwards: a workgroup holds a row in its registers.
 */
int bnn_norm_residual(int type, const void *y, int64_t ld_y, const void *x, int64_t ld_x, const void *gate,
                      int64_t ld_gate, int64_t rows_per_gate, float res_scale, int post, const float *post_gamma,
                      const float *post_beta, int pre, const float *pre_gamma, const float *pre_beta, float eps, void *r,
                      int64_t ld_r, void *n, int64_t ld_n, int64_t M, int64_t D, void *stream);

/*
 * Its backward pass, from dr (the gradient of r by every other way, or NULL: 0) and dn (the gradient of n; NULL exactly if
 * pre is BNN_NORM_NONE), with y and r as the forward pass had them (r is read only if pre is a norm):
 *   d = dr + pre'(dn);   dx = d;   dgate[g] = sum over the gate's rows of res_scale * d * t;   dy = post'(res_scale * gate * d)
 * dx, dy [M][ld] and dgate [ceil(M / rows_per_gate)][ld_dgate] of `type`; the gradients of the gammas and betas [D] float32.
 * Any output may be NULL.  The gradient of an absent gate cannot be asked for, that of an absent gamma or beta can (it is
 * the one at 1 or 0); betas only with BNN_NORM_LAYER, gammas only with a norm.  workspace as above.
 */
int64_t bnn_norm_residual_backward_workspace(int64_t M, int64_t D, int64_t rows_per_gate);
int bnn_norm_residual_backward(int type, const void *dr, int64_t ld_dr, const void *dn, int64_t ld_dn, const void *y,
                               int64_t ld_y, const void *r, int64_t ld_r, const void *gate, int64_t ld_gate,
                               int64_t rows_per_gate, float res_scale, int post, const float *post_gamma,
                               const float *post_beta, int pre, const float *pre_gamma, float eps, void *dx, int64_t ld_dx,
                               void *dy, int64_t ld_dy, void *dgate, int64_t ld_dgate, float *dpost_gamma,
                               float *dpost_beta, float *dpre_gamma, float *dpre_beta, int64_t M, int64_t D,
                               void *workspace, int64_t workspace_bytes, void *stream);

/* ---- quantised activations, packed weights -----------------------------------------------------------------------
 *
 * Rows of activations as codes of 8 or 4 bits with scales.  x^ is what they stand for:
 *   BNN_ROWS_I8   x^ = s q,   q a whole number in [-127, 127], s a float32 for each row: its largest magnitude / 127, and 2^-126 at
 *                 least.  A row with an infinity or a NaN has the scale NaN and codes of 0.
 *   BNN_ROWS_MX4  x^ = 2^e c, c one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (the 4-bit floating point codes e2m1), e for each 32
 *                 elements of a row the smallest exponent with which the largest magnitude of them does not round past 6, and -126
 *                 at least; held as the byte e + 127, 255 for a block with an infinity or a NaN, whose codes mean nothing.
 * q and c are the nearest ones to x / s and x / 2^e, of two as near the even code.
 *   codes   [M][ld_c] bytes, 16-byte aligned, ld_c a multiple of 16 and at least 32 (I8) or 16 (MX4) times ceil(K / 32): whole
 *           blocks of 32 elements, those past K zero.  Byte 4 i + j of an I8 block is element 8 j + i, nibble 8 i + j of an MX4 block
 *           (the lower half of a byte first) is element 4 j + i.
 *   scales  I8: float [M].  MX4: bytes [M][ld_s], 16-byte aligned, ld_s a multiple of 16 and at least ceil(K / 32); what the bytes past
 *           ceil(K / 32) hold means nothing.
 * Leading dimensions of reals as above.
 */
typedef enum bnn_rows { BNN_ROWS_I8 = 0, BNN_ROWS_MX4 = 1 } bnn_rows;

/*
 * bnn_quantize_rows: x [M][ld_x] of `type` to codes and scales, and x^ rounded to `type` in hat [M][ld_h], which may be NULL or x
 *   itself (same address and leading dimension).  x^ of MX4 is a number of each type, but for float16's range.
 * bnn_dequantize_rows: x^ of codes and scales, rounded to `type`.
 */
int bnn_quantize_rows(int rows, int type, const void *x, int64_t ld_x, uint8_t *codes, int64_t ld_c, void *scales, int64_t ld_s,
                      void *hat, int64_t ld_h, int64_t M, int64_t K, void *stream);
int bnn_dequantize_rows(int rows, int type, const uint8_t *codes, int64_t ld_c, const void *scales, int64_t ld_s, void *x,
                        int64_t ld_x, int64_t M, int64_t K, void *stream);

/*
 * bnn_norm_residual with n quantised: codes and scales of n (of r, if pre is BNN_NORM_NONE), taken of the unrounded values; hat [M][ld_h]
 * of `type` (or NULL) gets n^.  r may be NULL, or x itself.
 */
int bnn_norm_residual_q(int type, const void *y, int64_t ld_y, const void *x, int64_t ld_x, const void *gate, int64_t ld_gate,
                        int64_t rows_per_gate, float res_scale, int post, const float *post_gamma, const float *post_beta, int pre,
                        const float *pre_gamma, const float *pre_beta, float eps, void *r, int64_t ld_r, int rows, uint8_t *codes,
                        int64_t ld_c, void *scales, int64_t ld_s, void *hat, int64_t ld_h, int64_t M, int64_t D, void *stream);

/*
 * bnn_linear_bits and bnn_gated_bits on quantised rows x^ of K elements; residual, y and h of `type`.  The sums of I8 rows are
 * exact (whole numbers, before the scales), those of MX4 rows float32.  K up to 2^18 for I8, else BNN_ERR_UNSUPPORTED: sums are held
 * in 32 bits.
 * The gated product may give its result quantised, for the product that reads it: with out_codes [M][ld_oc] and out_scales
 * [M][ld_os], MX4 rows of F elements taken of the unrounded h, and h (or NULL) gets h^.  Without: NULL.
 */
int bnn_linear_q_bits(int rows, const uint8_t *codes, int64_t ld_c, const void *scales, int64_t ld_s, const uint32_t *w, int64_t ld_w,
                      const float *scale, const float *bias, int act, int type, const void *residual, int64_t ld_r, void *y,
                      int64_t ld_y, int64_t M, int64_t N, int64_t K, void *stream);
int bnn_gated_q_bits(int rows, const uint8_t *codes, int64_t ld_c, const void *scales, int64_t ld_s, const uint32_t *w, int64_t ld_w,
                     const float *scale, const float *bias, int act, int type, void *h, int64_t ld_h, uint8_t *out_codes,
                     int64_t ld_oc, uint8_t *out_scales, int64_t ld_os, int64_t M, int64_t F, int64_t K, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BNN_H */
