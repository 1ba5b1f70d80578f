/*
 * fftsp.h -- C ABI of the MI355X (gfx950) FFT-sparsifying gradient codec.
 *
 * The codec is the per-worker sender/receiver pair of arXiv 1811.08596, Sec. 3.1:
 * linearized gradient -> FFT -> keep the largest
 * frequency components -> range-based N-bit float -> pack; the receiver applies
 * the inverse operations in reverse order.
 *
 * Conventions shared by every entry point
 *   - Pointers named d_* are DEVICE pointers (hipMalloc / torch CUDA memory),
 *     16-byte aligned.  seg_offsets is a HOST pointer.  The caller owns every
 *     buffer; the library allocates nothing (its two 16 KiB twiddle tables are
 *     constants inside the code object).  The per-tensor entry points create
 *     three streams and four events per device on their first call outside a
 *     stream capture; they create nothing while the caller's stream is being
 *     captured (see there).
 *   - Calls only enqueue work on `stream` and return; they never synchronise and
 *     never touch the null stream.  Input buffers are not modified.  Output
 *     regions are written completely (padding bytes zero), so results are
 *     byte-comparable.  Two calls that share a workspace must be ordered by
 *     the caller (same stream, or events).
 *   - `theta` is the KEPT fraction of frequency bins in [0,1].  The paper's theta
 *     (Sec. 3.1.1) is the dropped fraction, i.e. 1 - theta of this interface.
 *   - `chunk_len` L is a power of two in [32, 2^22]; the flat gradient is cut
 *     into C = ceil(n/L) chunks, the last one zero-padded.  One chunk of length
 *     n is exactly the paper's whole-vector transform.
 *   - `bits` N is the code width: 3..16 for the offset-based N-bit float of
 *     Sec. 3.2.1 / Algorithm 1, or 32 for "quantization off" (raw binary32).
 *   - Return value: FFTSP_OK or an error; argument errors are detected on the
 *     host before anything is enqueued.  Non-finite gradient values are not
 *     detected: the call is memory-safe but its output is unspecified.
 *
 * Packed stream (little-endian, all padding zero):
 *   64-byte header: "FSP1", u32 version=1, u64 n, u32 L (0 = per-segment
 *   lengths), u32 C, u32 N, u32 m, u32 k, u32 S, f32 theta, zeros;
 *   then C records of S = align16(16 + 4*W + 4*ceil(2kN/32)) bytes,
 *   W = ceil(B/32), B = L/2+1:
 *     +0  u32 pbase, u32 vmax_bits, u32 k, u32 L-if-segmented-else-0
 *     +16 status bitmap (Sec. 3.2): bit j%32 of word j/32 set = bin j kept
 *     +16+4W codes: code i in bits [iN, iN+N) of an LSB-first u32 stream,
 *         order re0, im0, re1, im1, ... by ascending kept bin (the "dense"
 *         vector of Sec. 3.2; its positions are the prefix sum of the bitmap).
 */
#ifndef FFTSP_H
#define FFTSP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ihipStream_t* fftsp_stream_t; /* a hipStream_t */

typedef enum {
    FFTSP_OK = 0,
    FFTSP_EINVAL = 1,       /* null/misaligned pointer, n = 0, theta outside [0,1] or NaN, bad bits */
    FFTSP_ENOSPC = 2,       /* packed_capacity smaller than fftsp_packed_bytes(...) */
    FFTSP_EWORKSPACE = 3,   /* workspace smaller than fftsp_workspace_bytes(...) */
    FFTSP_EUNSUPPORTED = 4, /* chunk_len not a power of two in [32, 2^22] */
    FFTSP_EHIP = 5,         /* a HIP runtime call or launch failed */
    FFTSP_EFORMAT = 6       /* packed stream does not match the arguments (device status word) */
} fftsp_status;

/* ---- host-side arithmetic: no device access, pure functions of their arguments ---- */

/* k = clamp(floor((double)theta * B + 1/2), 0, B): kept bins per chunk (selection rule of Sec. 3.1.1). */
int fftsp_kept_per_chunk(uint32_t chunk_len, float theta, uint32_t* k_out);
/* default mantissa width m of the N-bit float (Sec. 3.2.1, the split of the N bits); -1 if bits invalid. */
int fftsp_mantissa_bits(int bits);
/* exact size of the packed stream, 0 on invalid arguments. */
size_t fftsp_packed_bytes(size_t n, uint32_t chunk_len, float theta, int bits);
/* bytes of device workspace any entry point below needs for (n, chunk_len, bits); 0 on invalid arguments. */
size_t fftsp_workspace_bytes(size_t n, uint32_t chunk_len, int bits);

/* ---- the codec (Sec. 3.1 steps 1-4 and their inverses) ---- */

/* Sender.  d_grad: n floats.  d_packed: receives fftsp_packed_bytes(...) bytes. */
int fftsp_compress(const float* d_grad, size_t n, uint32_t chunk_len, float theta, int bits,
                   void* d_packed, size_t packed_capacity,
                   void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* The sender for callers that cannot allocate device memory or pass a workspace: code recorded into a HIP graph,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same packed bytes as fftsp_compress; the
 * workspace is a fixed array of FFTSP_STATIC_SCRATCH_BYTES inside the library's code object (every GPU the
 * library runs on holds its own copy until the process ends).  The call allocates nothing, on the host side
 * of HIP or on the device (keep fftsp_profile_enable off: its events are created on demand).
 * Limit: fftsp_workspace_bytes(n, chunk_len, bits) <= FFTSP_STATIC_SCRATCH_BYTES (e.g. n = 2^20 with
 * chunk_len = 2^16, or one chunk of 2^20); beyond that the call returns FFTSP_EWORKSPACE and enqueues nothing.
 * All calls on one GPU share that GPU's array: two calls that may overlap in time (different streams, no event
 * between them) race and must be ordered by the caller.  The array keeps the last call's contents; the kernels
 * clear what they need cleared.  The device status word lives inside the array and cannot be read back. */
#define FFTSP_STATIC_SCRATCH_BYTES (16u << 20)
int fftsp_compress_static(const float* d_grad, size_t n, uint32_t chunk_len, float theta, int bits,
                          void* d_packed, size_t packed_capacity, fftsp_stream_t stream);

/* Receiver.  The same (n, chunk_len, theta, bits) as the sender must be passed; a stream whose
 * header disagrees sets the device status word to FFTSP_EFORMAT and the output is unspecified
 * (reads stay inside d_packed[0, packed_bytes)).  d_grad_out: exactly n floats are written. */
int fftsp_decompress(const void* d_packed, size_t packed_bytes,
                     float* d_grad_out, size_t n, uint32_t chunk_len, float theta, int bits,
                     void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- quantizer options (Sec. 3.2.1: the choice of m and eps; the static [min, max] range) ----
 *
 * The entry points above fix m from the code width and fit the range of every chunk to its largest surviving
 * component.  The _q variants take both from the caller; quantizer == NULL means the defaults.
 *   mantissa_bits: m, 1 .. bits-1 (ignored for bits = 32); 0 = fftsp_mantissa_bits(bits).
 *   range_max:     > 0: static range [-range_max, +range_max] for every chunk, as in the paper's experiments
 *                  (range estimated beforehand); components beyond it clamp to the top code (Algorithm 1) and no
 *                  reduction over the survivors is needed.  0 = fitted per chunk.  Negative, infinite or NaN:
 *                  FFTSP_EINVAL.
 * eps is not an input: for a given range it is the closed form the paper's iterative tuning converges to.
 * The receiver needs the same mantissa_bits (the stream header carries m and a mismatch raises FFTSP_EFORMAT);
 * range_max is ignored there (every record carries its pbase). */
typedef struct fftsp_quantizer {
    int mantissa_bits;
    float range_max;
} fftsp_quantizer;

int fftsp_compress_q(const float* d_grad, size_t n, uint32_t chunk_len, float theta, int bits,
                     void* d_packed, size_t packed_capacity, void* d_workspace, size_t workspace_bytes,
                     const fftsp_quantizer* quantizer, fftsp_stream_t stream);
int fftsp_decompress_q(const void* d_packed, size_t packed_bytes, float* d_grad_out, size_t n, uint32_t chunk_len,
                       float theta, int bits, void* d_workspace, size_t workspace_bytes,
                       const fftsp_quantizer* quantizer, fftsp_stream_t stream);
int fftsp_encode_spectrum_q(const float* d_spec, size_t n, uint32_t chunk_len, float theta, int bits,
                            void* d_packed, size_t packed_capacity, void* d_workspace, size_t workspace_bytes,
                            const fftsp_quantizer* quantizer, fftsp_stream_t stream);
int fftsp_decode_spectrum_q(const void* d_packed, size_t packed_bytes, size_t n, uint32_t chunk_len, float theta,
                            int bits, float* d_spec, void* d_workspace, size_t workspace_bytes,
                            const fftsp_quantizer* quantizer, fftsp_stream_t stream);

/* ---- receiver under an allgather (Sec. 4, "Implementation": every worker collects the packed gradients of all
 *      peers; Sec. 3.1: the receiver applies the inverse steps) ----
 *
 * The inverse transform is linear, so the peers' sparse spectra are added bin by bin and ONE inverse transform is
 * taken:   d_grad_out = scale * iFFT( sum_p D(d_packed[p]) ),   e.g. scale = 1/npeers for the average.
 * The sum starts from zero and adds the peers in list order in binary32; scale multiplies the transform's
 * normalisation 1/L (one binary32 product per output).
 *
 * d_packed: HOST array of npeers DEVICE pointers (16-byte aligned), each to a stream of packed_bytes bytes made
 * with the same (n, chunk_len, theta, bits); the array is read before the call returns.  1 <= npeers <=
 * FFTSP_MAX_PEERS (more: FFTSP_EUNSUPPORTED; call again on the remainder and add).  A stream whose header or
 * bitmaps disagree with the arguments sets the device status word to FFTSP_EFORMAT; reads stay inside each
 * stream.  The workspace must hold fftsp_workspace_bytes_accumulate(...) bytes (0 on invalid arguments). */
#define FFTSP_MAX_PEERS 32
size_t fftsp_workspace_bytes_accumulate(size_t n, uint32_t chunk_len, int bits, int npeers);
int fftsp_decompress_accumulate(const void* const* d_packed, int npeers, size_t packed_bytes, float scale,
                                float* d_grad_out, size_t n, uint32_t chunk_len, float theta, int bits,
                                void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
/* Stage-level: only the summed spectrum, C*(L+2) floats in natural bin order, unscaled (bit-exact against the
 * same binary32 sum on the host). */
int fftsp_decode_accumulate_spectrum(const void* const* d_packed, int npeers, size_t packed_bytes, size_t n,
                                     uint32_t chunk_len, float theta, int bits, float* d_spec,
                                     void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- stage-level entry points (the same kernels the codec runs, exposed for parity checks) ---- */

/* Forward real DFT of each chunk (the sum of Sec. 3.1.1, sign -, unnormalised).
 * d_spec: C*(L+2) floats, chunk c at c*(L+2), bins 0..L/2 as (re,im) pairs; im of bins 0 and L/2 is +0. */
int fftsp_rfft(const float* d_grad, size_t n, uint32_t chunk_len, float* d_spec,
               void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
/* Inverse (1/L, Hermitian extension; im of bins 0 and L/2 ignored); writes the first n samples. */
int fftsp_irfft(const float* d_spec, size_t n, uint32_t chunk_len, float* d_grad_out,
                void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
/* Steps 2-4 of Sec. 3.1 on a given spectrum: magnitude top-k, Algorithm 1, packing (Sec. 3.2). */
int fftsp_encode_spectrum(const float* d_spec, size_t n, uint32_t chunk_len, float theta, int bits,
                          void* d_packed, size_t packed_capacity,
                          void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
/* Inverse of the above: unpack, Nbit_to_32bit of Algorithm 1, scatter into a zeroed spectrum. */
int fftsp_decode_spectrum(const void* d_packed, size_t packed_bytes, size_t n, uint32_t chunk_len,
                          float theta, int bits, float* d_spec,
                          void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- half-precision variant (Sec. 3.1.1, "Our approach": the gradients go to 16 bits for the transform, a loss
 *      the paper calls negligible because gradients are bounded).  Definition: the chunk's DFT times 2^scale_log2,
 *      each component rounded to binary16 (nearest even, saturating at +-65504); selection, Algorithm 1 and packing
 *      as in fftsp_compress on those values; the receiver inverts and divides by 2^scale_log2.  Here the arithmetic
 *      stays binary32 and it is the stored intermediate of the two-pass transform and the stored spectrum that are
 *      binary16 (these kernels are bound by bytes, not by arithmetic), so a result differs from the definition by
 *      one more binary16 rounding inside the transform: about 5e-4 relative L2 on a spectrum, against the 1e-5 of
 *      the binary32 path.  scale_log2 in [-24, 24] is the caller's: choose it so that spectrum magnitudes
 *      (about 2^scale_log2 * sigma * sqrt(chunk_len)) sit well inside binary16's normal range [6e-5, 65504].
 *      The stream layout is that of fftsp_compress with header word 12 (offset 48) = scale_log2; fftsp_decompress
 *      rejects a stream with a non-zero scale and fftsp_decompress_h one with another scale (status
 *      FFTSP_EFORMAT).  chunk_len: power of two in [2^15, 2^22] (FFTSP_EUNSUPPORTED below: one workgroup
 *      transforms such a chunk without touching memory in between).  Everything else as fftsp_compress /
 *      fftsp_decompress, including packed and workspace sizes (fftsp_packed_bytes, fftsp_workspace_bytes). ---- */
int fftsp_compress_h(const float* d_grad, size_t n, uint32_t chunk_len, float theta, int bits, int scale_log2,
                     void* d_packed, size_t packed_capacity,
                     void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
int fftsp_decompress_h(const void* d_packed, size_t packed_bytes, float* d_grad_out, size_t n,
                       uint32_t chunk_len, float theta, int bits, int scale_log2,
                       void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- time-domain Top-k, the sparsifier the paper measures its own against (Sec. 4, "Choice of Algorithms";
 *      the Sec. 3.1.1 figure sets it beside FFT Top-k): the magnitude selection (Sec. 3.1.1), Algorithm 1 and the
 *      packing of Sec. 3.2 applied to the gradient's samples themselves, no transform.  Chunk c is samples
 *      [c*L, (c+1)*L) (the last one zero-padded for the selection; the padding is never written back); a sample
 *      ranks by |x|, ties to the lowest index; k = round-half-up(theta * L) samples are kept per chunk, theta
 *      being the KEPT fraction; bits = 32 is the paper's plain Top-k.  Record: 16-byte header as above, bitmap of
 *      ceil(L/32) words, ONE code per kept sample; stream header word 11 (offset 44) is 1, and each decompress
 *      accepts only its own kind of stream (status FFTSP_EFORMAT otherwise).  chunk_len: power of two in
 *      [32, 2^21].  Pointers, alignment, workspace, stream and error behaviour are those of
 *      fftsp_compress / fftsp_decompress; the workspace here holds no spectrum. ---- */
int fftsp_topk_kept_per_chunk(uint32_t chunk_len, float theta, uint32_t* k_out);
size_t fftsp_topk_packed_bytes(size_t n, uint32_t chunk_len, float theta, int bits);
size_t fftsp_topk_workspace_bytes(size_t n, uint32_t chunk_len, int bits);
int fftsp_topk_compress(const float* d_grad, size_t n, uint32_t chunk_len, float theta, int bits,
                        void* d_packed, size_t packed_capacity,
                        void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
int fftsp_topk_decompress(const void* d_packed, size_t packed_bytes, float* d_grad_out, size_t n,
                          uint32_t chunk_len, float theta, int bits,
                          void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- per-tensor variant: segment i = d_grad[seg_offsets[i] .. seg_offsets[i+1]) is one chunk of
 *      L_i = max(32, next power of two >= its size); seg_offsets (nseg+1 entries, ascending) is on the HOST
 *      and is consumed before the call returns.  Sizes above 2^22 are FFTSP_EUNSUPPORTED.
 *      Records follow tensor order in the stream.  Tensors of up to 2^15 samples, whatever their lengths, run as one
 *      launch per direction (up to 128 at a time).  All longer ones share one launch per kernel, whatever their lengths (up
 *      to 64 of them and 2^26 padded samples at a time).  Where up to 22 longer ones are done soon, their first kernel is
 *      part of the others' launch (and of what fftsp_profile_report calls tensors_compress and tensors_decompress).
 *      Where they take a while, the others run beside them on a stream of the library's own that forks from and
 *      joins back into the caller's, so the call is still one unit of work on the caller's stream and can be
 *      captured into a graph.  That stream belongs to the device and is shared by all callers: calls from several
 *      host threads enqueue one after the other.  A captured call
 *      keeps it inside its capture until that capture ends; a call made meanwhile on another stream, and a captured
 *      call made before it exists, runs everything on the caller's stream alone (same bytes, less overlap). ---- */
size_t fftsp_packed_bytes_segments(const size_t* seg_offsets, int nseg, float theta, int bits);
size_t fftsp_workspace_bytes_segments(const size_t* seg_offsets, int nseg, int bits);
int fftsp_compress_segments(const float* d_grad, const size_t* seg_offsets, int nseg, float theta, int bits,
                            void* d_packed, size_t packed_capacity,
                            void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);
int fftsp_decompress_segments(const void* d_packed, size_t packed_bytes, float* d_grad_out,
                              const size_t* seg_offsets, int nseg, float theta, int bits,
                              void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* ---- around the codec in a training step of a language model: the embedding and the orthogonalised update ----
 *
 * The embedding's gradient is the part of the flat gradient that most of whose rows are zero; the update takes the
 * flat gradient that a receiver leaves, matrix by matrix.  Unlike above, the arrays of this section need only their
 * own element's alignment (tensors of a flat gradient begin anywhere); workspaces are 16-byte aligned and must not
 * overlap them.  Everything else is as stated at the top: device pointers, nothing allocated, nothing but launches on
 * `stream`, same bytes for the same inputs.  These calls leave no status word: fftsp_device_status is for workspaces of the
 * calls above and has nothing to read in one that a call of this section used last.  Element types: */
typedef enum { FFTSP_F32 = 0, FFTSP_BF16 = 1, FFTSP_F16 = 2 } fftsp_type;

/* d_out[t][j] = scale * d_table[token t][j], j < width, a binary32 product, then rounded to out_type; a token outside [0, rows) (padding is
 * usually -1) gives a row of zeros.  Row v of the table begins at element v * table_stride, row t of the output at
 * t * out_stride (strides >= width; elements between width and the stride are neither read nor written).
 * token_bits: 32 or 64 (int32_t, int64_t).  ntokens = 0 does nothing.  rows, ntokens <= 2^30, width <= 2^20, the last row
 * at most 2^48 elements behind the first; FFTSP_EINVAL otherwise.  d_out must not overlap the table or the tokens (FFTSP_EINVAL). */
int fftsp_embedding(const void* d_table, int table_type, size_t rows, uint32_t width, size_t table_stride,
                    const void* d_tokens, int token_bits, size_t ntokens, float scale,
                    void* d_out, int out_type, size_t out_stride, fftsp_stream_t stream);

/* Its gradient with respect to the table, every row of it written:
 *   d_table_grad[v][j] = d_base[v][j] + scale * (sum over the t with token t == v of d_out_grad[t][j]),
 * d_base == NULL standing for zeros.  d_base has the type and stride of d_table_grad and is the same array (the sum is
 * added in place, and only rows that have a token are touched) or does not overlap it.  Tokens outside [0, rows) give
 * nothing.  Sums, their product with scale and the base's sum are binary32, in an order that depends on the tokens, types
 * and sizes alone; then one rounding to table_type.  Limits as above, and ntokens <= 2^24 (FFTSP_EUNSUPPORTED).  The
 * workspace holds fftsp_workspace_bytes_embedding(...) bytes (0 on invalid arguments); ntokens = 0 needs none. */
size_t fftsp_workspace_bytes_embedding(size_t rows, uint32_t width, size_t ntokens);
int fftsp_embedding_gradient(const void* d_out_grad, int out_type, size_t out_stride, const void* d_tokens,
                             int token_bits, size_t ntokens, float scale, const void* d_base, void* d_table_grad,
                             int table_type, size_t rows, uint32_t width, size_t table_stride,
                             void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* A matrix inside flat arrays: `rows` rows of `cols` values, the first at element `offset`, rows `stride` elements
 * apart (stride >= cols).  gain: factor on its orthogonalised form (finite). */
typedef struct fftsp_matrix {
    uint64_t offset, stride;
    uint32_t rows, cols;
    float gain;
    uint32_t reserved; /* 0 */
} fftsp_matrix;

/* Newton-Schulz orthogonalisation of every matrix G of the list, as the Muon optimiser takes it:
 *   X = G / (|G|_F + eps), transposed if it has more rows than columns; then, for each (a, b, c) of `coefficients`,
 *   X <- a X + (b A + c A A) X with A = X X^T;   out = gain * X (transposed back).
 * coefficients: HOST array of 3 * nsteps floats, read before the call returns; NULL: five steps of
 * (3.4445, -4.7750, 2.0315), nsteps is then ignored.  1 <= nsteps <= FFTSP_MAX_STEPS.  Coefficients under which singular
 * values s that begin in [0, 1], or a step's polynomial a + b s^2 + c s^4 of them, pass 4096 are FFTSP_EUNSUPPORTED (the
 * default: 1.3 and 3.4), whatever the matrices are.  eps >= 0; a matrix of zeros gives zeros (with eps = 0, too).  |G|_F is
 * taken in binary64; inside, numbers have 22 bits or more and sums are binary32, whatever the types of d_in and d_out are.
 * Five default steps are 0.5 to 8e-6 of the result's norm off, about as far as plain binary32 products; a result of 16 bits is
 * the one of 32, rounded.  How products are shared out follows from the whole list, so a matrix in another list may come out with
 * other last bits, within that.  (Matrices of up to 64 x 768 are one launch if all of the list's with min(rows, cols) < 512 are that
 * small; one larger takes them to launches of products, a thousand of them for five times as long: two calls are faster then.)
 * Every matrix is at `offset` of d_in and of d_out; d_in == d_out is allowed where the types agree, other overlaps are
 * not.  Matrices of a list must not share elements (FFTSP_EINVAL; columns of one array with one stride may alternate).
 * `matrices` is a HOST array, read before the call returns; nmat = 0 does nothing.  min(rows, cols) <= 16384,
 * max(rows, cols) <= 2^20, nmat <= 2^22 and at most 2^22 blocks of 64 x 64 values in all (FFTSP_EUNSUPPORTED; the largest
 * matrix is that many).  Non-finite values make their own matrix's output unspecified.
 * The workspace holds fftsp_workspace_bytes_orthogonal(matrices, nmat) bytes (0 on invalid arguments). */
#define FFTSP_MAX_STEPS 16
size_t fftsp_workspace_bytes_orthogonal(const fftsp_matrix* matrices, int nmat);
int fftsp_orthogonal(const void* d_in, int in_type, void* d_out, int out_type, const fftsp_matrix* matrices, int nmat,
                     const float* coefficients, int nsteps, float eps,
                     void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* The momentum step round it (Sec. 4: momentum SGD on the received gradient), for every matrix of the list:
 *   M' = beta M + G;  U = G + beta M' (nesterov != 0) or M';  O = the above of U (before its gain);
 *   W' = (1 - lr * weight_decay) W - lr * gain * O in binary32 (1 - lr * weight_decay and its product with W are rounded), then
 * rounded to weight_type.
 * d_grad is of grad_type (a receiver's output: FFTSP_F32), momentum is binary32.  All arrays hold the matrices at the
 * same offsets and strides; d_momentum_out may be d_momentum and d_weights_out may be d_weights (an update in place),
 * other overlaps are not allowed.  Elements outside the matrices are neither read nor written. */
typedef struct fftsp_step {
    float lr, beta, weight_decay, eps; /* finite; beta in [0, 1], eps >= 0 */
    int nesterov;
    int nsteps;                /* as above */
    const float* coefficients; /* HOST, as above */
} fftsp_step;
int fftsp_orthogonal_step(const void* d_grad, int grad_type, const float* d_momentum, float* d_momentum_out,
                          const void* d_weights, void* d_weights_out, int weight_type,
                          const fftsp_matrix* matrices, int nmat, const fftsp_step* step,
                          void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream);

/* Synchronises `stream`'s device and reads the status word the last call on this workspace left
 * (FFTSP_OK or FFTSP_EFORMAT).  Returns FFTSP_EHIP if the copy fails. */
int fftsp_device_status(const void* d_workspace, int* status_out);

/* Per-kernel timing for benchmarks (not part of the method).  While enabled, every kernel the library
 * launches is bracketed by two HIP events on its stream (do not enable under stream capture).
 * fftsp_profile_enable(1) also discards earlier records.  fftsp_profile_report synchronises the device and
 * writes one text line per kernel, "name calls total_ms", NUL-terminated, into buf (HOST memory, cap bytes);
 * it returns the number of bytes the full report needs. */
int fftsp_profile_enable(int on);
size_t fftsp_profile_report(char* buf, size_t cap);

const char* fftsp_strerror(int status);
const char* fftsp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FFTSP_H */
