/*
 * accept.h -- C ABI of the boundary-tensor codec (AccEPT bit-level compression, Sec. 3.3-3.4).
 *
 * The codec turns a flat fp32 tensor x_v (Sec. 3.3, "Forward Quantizer": the boundary tensor is
 * vectorised to N = n*w*h*c values) into k-bit integer codes packed densely into 32-bit words plus
 * fp32 side words, and back.  All compute runs in CUDA kernels built for sm_100a; there is no host
 * fallback.  Every entry point is asynchronous on the stream it is given and allocates nothing.
 *
 * ---------------------------------------------------------------------------------------------
 * Operation (per chunk of chunk_elems consecutive values; the paper's scheme is the case
 * chunk_elems >= n_elems, one range for the whole tensor):
 *
 *   range   ABSMAX (Sec. 3.3 "Backward Quantizer"):  c = max|x|,  L = 2^(k-1)-1,  s = c/L,  o = 0
 *           MINMAX (affine extension):               lo = min x, hi = max x, L = 2^k-1,
 *                                                    s = (hi-lo)/L,  o = lo
 *   scale   inv = L/c  (resp. L/(hi-lo)) rounded toward zero, one IEEE fp32 division per chunk, so that
 *           |x*inv| <= L as in exact arithmetic and no code is clamped.  If the range is 0, or the
 *           quotient overflows, the chunk is degenerate: s = 0, inv = 0, every code is the zero point.
 *   codes   t = x*inv           (MINMAX: t = (x-lo)*inv), each fp32 operation rounded separately
 *           NEAREST:    q = rint(t)                      (ties to even)
 *           STOCHASTIC: q = floor(t) + [U < t-floor(t)]  (Eq. 7), U from the counter-based
 *                       generator described at accept_params.seed; the fraction t-floor(t) and
 *                       the comparison are exact (no rounding of the difference)
 *           ABSMAX: q lies in [-L, L] (inside the paper's [-2^(k-1), 2^(k-1)-1]), stored code
 *           u = q + 2^(k-1)  ("+8" of the "Backward Encoder" for k = 4);  MINMAX: u = q in [0, 2^k-1]
 *   pack    INTERLEAVED ("Backward Encoder"): code of element t of the chunk occupies bits
 *           [k*t, k*t+k) of the chunk's little-endian bit string (k = 8: plain bytes).
 *           BITPLANE ("Forward Encoder"): per group of 32 consecutive elements, k consecutive
 *           32-bit words; bit t of word j is bit j of the code of element t of the group.
 *   decode  ("Backward Decoder/Dequantizer", "Forward Decoder"): unpack u;
 *           ABSMAX: xhat = float(u - 2^(k-1)) * s;   MINMAX: xhat = fl(fl(float(u)*s) + o)
 *
 * Stream layout (little-endian, byte offsets):
 *   [0,32)    header, eight u32: magic 0x54504341 ("ACPT"), version 1, n_elems low, n_elems high,
 *             chunk_elems, k, range | round<<8 | layout<<16, group_stride
 *   [32, 32+8M)   M = ceil(n_elems/chunk_elems) records {float s; float o}, one per chunk
 *   [P, ...)  payload, P = 32+8M rounded up to a multiple of 16.  Chunk m starts at word
 *             m*chunk_elems*k/32 of the payload.  A partial last chunk holds ceil(valid/32)*k
 *             words; codes of padding elements are 0 bits.
 *   total     P + 4*k*ceil(n_elems/32) bytes  (= accept_compressed_size).
 *
 * Pointers named d_* are DEVICE pointers, h_* are HOST pointers.  d_x, d_xhat and d_stream must be
 * 16-byte aligned.  The caller owns every buffer and the stream.
 */
#ifndef ACCEPT_H_
#define ACCEPT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ACCEPT_MAGIC 0x54504341u
#define ACCEPT_VERSION 1u
#define ACCEPT_HEADER_BYTES 32u

/* Return codes of the host entry points (nothing was launched unless ACCEPT_OK). */
typedef enum {
  ACCEPT_OK = 0,
  ACCEPT_ERR_NULL = 1,          /* a required pointer is NULL */
  ACCEPT_ERR_BAD_K = 2,         /* k not in {2,3,4,8}, or k = 3 with INTERLEAVED */
  ACCEPT_ERR_BAD_CHUNK = 3,     /* chunk_elems < 32 or not a multiple of 32 */
  ACCEPT_ERR_BAD_ENUM = 4,      /* range / round / layout out of range */
  ACCEPT_ERR_TOO_SMALL = 5,     /* a buffer is smaller than the size queries say */
  ACCEPT_ERR_BAD_STREAM_HEADER = 6, /* header words do not match the parameters */
  ACCEPT_ERR_CUDA = 7,          /* a CUDA runtime call failed */
  ACCEPT_ERR_NONFINITE = 8,     /* reported through the device status word only */
  ACCEPT_ERR_BAD_SIZE = 9,      /* n_elems = 0 */
  ACCEPT_ERR_MISALIGNED = 10,   /* a device pointer is not 16-byte aligned */
  ACCEPT_ERR_SCRATCH_LIMIT = 11, /* accept_compress_static: the call needs more scratch than the built-in array holds */
  ACCEPT_ERR_UNCHECKED_BUILD = 12 /* accept_bounds_check_report: this library was built without access checks */
} accept_status;

/* Bits of the device status word (word 0 of the workspace); sticky until the caller clears it. */
#define ACCEPT_DEV_NONFINITE 1u   /* some chunk held NaN/Inf (or an overflowing MINMAX range) */
#define ACCEPT_DEV_BAD_HEADER 2u  /* accept_decompress: stream header differs from the parameters */
#define ACCEPT_DEV_COPY_TIMEOUT 4u /* an asynchronous copy inside a kernel did not complete within 0.2 s; output invalid */

typedef enum { ACCEPT_RANGE_ABSMAX = 0, ACCEPT_RANGE_MINMAX = 1 } accept_range;
typedef enum { ACCEPT_ROUND_NEAREST = 0, ACCEPT_ROUND_STOCHASTIC = 1 } accept_round;
typedef enum { ACCEPT_LAYOUT_INTERLEAVED = 0, ACCEPT_LAYOUT_BITPLANE = 1 } accept_layout;

/*
 * Parameters of one call.
 *   n_elems      N >= 1, number of fp32 values.
 *   chunk_elems  C, multiple of 32, >= 32: elements sharing one range.
 *   k            bit width: 2, 3 (BITPLANE only), 4 or 8.
 *   group_stride 0, or F = values per sample (w*h*c): the tensor is (n_elems/F) x F and a pack group is
 *                made of the 32 BATCH neighbours (rows 32g..32g+31) of one feature f: pack groups run
 *                along the batch dimension as in Sec. 3.3, "Forward Encoder" / "Backward Encoder".
 *                Group index G = g*F + f, words G*k .. G*k+k-1 of the payload, element
 *                (row b, feature f) at position t = b % 32 of its group; rows past the last are zero
 *                bits; payload = 4*k*ceil(rows/32)*F bytes.  Ranges stay per chunk of consecutive
 *                values.  Needs n_elems % F == 0 and a 32-byte aligned input; any F >= 1 (the
 *                paper's smallest outputs need not have 8 | w*h*c).  With F % 8 == 0 a thread
 *                codes eight features of eight rows with 32-byte loads;
 *                every other shape takes one feature per thread, slower but for any F.  Runs as
 *                two launches: ranges, side words and constants of every chunk, then the encoder
 *                (workspace: 16 bytes per chunk more, as for chunk_elems > 32768; with such chunks
 *                it is a memset and four launches).  Header word 7 carries F.
 *   seed, rng_offset  STOCHASTIC only.  Element i draws
 *                  U_i = (g >> 8) * 2^-24,
 *                  g   = h * M[ctr & 3] (mod 2^32),  M = {1, 0x9E3779B1, 0x85EBCA77, 0xC2B2AE3D},
 *                  h   = fmix32( lo32(j) ^ fmix32( hi32(j) ^ lo32(seed) ^ 0x9E3779B9 ) ^ hi32(seed) ),
 *                  j   = ctr >> 2,  ctr = rng_offset + i (mod 2^64)
 *                (four neighbouring counters share one hash; each takes it times its own odd constant),
 *                fmix32 = the 32-bit finaliser of MurmurHash3:
 *                  h ^= h>>16; h *= 0x85EBCA6B; h ^= h>>13; h *= 0xC2B2AE35; h ^= h>>16.
 *                The same (seed, rng_offset) reproduces the same stream; advance rng_offset by
 *                n_elems between calls to draw fresh numbers.
 */
typedef struct {
  uint64_t n_elems;
  uint32_t chunk_elems;
  uint32_t k;
  int32_t range;   /* accept_range  */
  int32_t round;   /* accept_round  */
  int32_t layout;  /* accept_layout */
  uint32_t group_stride; /* 0: pack groups of 32 consecutive values; F > 0: see below */
  uint64_t seed;
  uint64_t rng_offset;
} accept_params;

/* Validates p as the compress/decompress entry points do (host only). */
accept_status accept_check_params(const accept_params* p);

/*
 * Size in bytes of the compressed stream for p (layout above); 0 if p is invalid.
 * Sec. 3.3 "Transmission Data Comparison", Eq. 8: payload of k bits per element plus fp32 side words.
 */
size_t accept_compressed_size(const accept_params* p);

/* Byte offset of the payload inside the stream (P above); 0 if p is invalid. */
size_t accept_payload_offset(const accept_params* p);

/*
 * Bytes of device workspace the kernels need: 16, plus 16 per chunk when chunk_elems > 32768 or group_stride != 0
 * (such chunks do not fit on chip: their ranges are gathered in the workspace first, and the input
 * is read twice).  Word 0 is the device status word; the caller zeroes the workspace once (and
 * whenever it wants to clear the status); the workspace must be 16-byte aligned.  0 if p is invalid.
 * This is what accept_compress needs.  accept_decompress touches the status word only: 16 bytes
 * (4-byte aligned) are enough for it, whatever the parameters.
 */
size_t accept_workspace_size(const accept_params* p);

/*
 * Quantizer + encoder (Sec. 3.3): reads n_elems floats at d_x, writes accept_compressed_size(p)
 * bytes at d_stream (header, per-chunk {s,o}, payload), in one kernel launch (three launches and a
 * memset of the workspace records when chunk_elems > 32768, e.g. one range for the whole tensor as
 * in the paper) on cuda_stream
 * (a cudaStream_t, may be NULL for the default stream).  Non-finite input does not fail the call:
 * the chunk is written as degenerate and ACCEPT_DEV_NONFINITE is or-ed into the status word.
 * d_x is only read; d_stream is fully overwritten up to the compressed size.
 */
accept_status accept_compress(const accept_params* p, const float* d_x, void* d_stream,
                              size_t stream_bytes, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * Decoder + dequantizer (Sec. 3.4): reads the stream at d_stream, writes n_elems floats at d_xhat,
 * in one kernel launch.  p carries what the receiver agreed on with the sender (n_elems,
 * chunk_elems, k, range, layout; round/seed are ignored); the kernel compares it with the header
 * words and or-s ACCEPT_DEV_BAD_HEADER into the status word on a mismatch (the output is then
 * unspecified but every access stays inside the buffers as sized by p).  The workspace needs 16 bytes
 * only (the status word), also for wide chunks and batch groups.
 */
accept_status accept_decompress(const accept_params* p, const void* d_stream, size_t stream_bytes,
                                float* d_xhat, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * accept_compress for callers that cannot allocate device memory at all.  (The paper has no counterpart:
 * this is a packaging variant of the quantizer + encoder above, same kernel, same stream.)
 *
 * Who needs it: a pipeline stage on a device whose memory budget is sealed after start-up, or a plug-in
 * living inside a host framework that owns every byte of device memory, has no way to obtain the
 * workspace accept_compress asks for -- cudaMalloc (or the framework's allocator) is off limits to it.
 * Here the workspace is a fixed array of ACCEPT_STATIC_SCRATCH_BYTES (256) bytes that is part of the
 * library image: every GPU that loads the library holds it until the process exits, and the entry point
 * calls no cudaMalloc, cudaFree or any other allocating routine.  The caller still passes the input and
 * the output stream, sized as for accept_compress.
 *
 *   d_status_out  optional DEVICE pointer (4-byte aligned) that receives the ACCEPT_DEV_* status bits of
 *                 THIS call (copied on cuda_stream after the kernel); NULL if not wanted.
 *
 * Limits and rules:
 *   - a call whose workspace need (accept_workspace_size) exceeds ACCEPT_STATIC_SCRATCH_BYTES is rejected
 *     with ACCEPT_ERR_SCRATCH_LIMIT and nothing is launched;
 *   - the first call on each device looks up the array's device address (with that device current); make
 *     that first call before any stream capture begins on that device;
 *   - all calls on a device share the one array.  The status word in it is cleared at the start of every
 *     call (so it does not accumulate across calls as a caller-owned workspace does), and two calls that
 *     overlap on the GPU (different streams) race on it: issue them on one stream, or order them.  Calls
 *     from several host threads must be serialised by the caller even on one stream: a call enqueues a
 *     clear, its kernels and the status copy one after the other, and two threads could interleave them;
 *   - d_x must live on the current device (checked: ACCEPT_ERR_CUDA otherwise), and cuda_stream must
 *     belong to it.
 */
#define ACCEPT_STATIC_SCRATCH_BYTES 256u
accept_status accept_compress_static(const accept_params* p, const float* d_x, void* d_stream,
                                     size_t stream_bytes, uint32_t* d_status_out, void* cuda_stream);

/*
 * Host-buffer variants, for callers whose tensors live in host memory: copy h_x to the staging
 * buffer d_x (host to device), run accept_compress, copy the stream back to h_stream (and the
 * mirror image for decompress), all asynchronously on cuda_stream.  Staging buffers are the
 * caller's; sizes as for the device entry points.  Pinned host memory makes the copies overlap
 * nothing else but avoids a bounce buffer in the driver.
 */
accept_status accept_compress_host(const accept_params* p, const float* h_x, void* h_stream,
                                   size_t stream_bytes, float* d_x, void* d_stream, void* d_ws,
                                   size_t ws_bytes, void* cuda_stream);
accept_status accept_decompress_host(const accept_params* p, const void* h_stream,
                                     size_t stream_bytes, float* h_xhat, void* d_stream,
                                     float* d_xhat, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * ---------------------------------------------------------------------------------------------
 * Forward quantizer of the paper: multi-bit quantization (Sec. 3.3 "Forward Quantizer", Eq. 1-5;
 * "Forward Encoder"; Sec. 3.4 "Forward Decoder", "Forward Dequantizer").
 *
 * x ~ B alpha, B in {-1,+1}^(N x k), alpha in R^k (one alpha per tensor, as in the paper).  Element
 * i carries the code c_i = sum_j [b_ij = +1] << j; level(c) = (+-alpha_0) + ... + (+-alpha_k-1)
 * summed in fp32 in the order j = 0..k-1.
 *   batch_index t >= 1 (init = 0): every value takes the nearest level of alpha_prev (exact
 *     comparison; a tie goes to the lower level; coinciding levels: the smallest code), then
 *     alpha_cur = (B^T B)^-1 B^T x (Eq. 3; kept at alpha_prev if B^T B is singular) and
 *     alpha_next = beta alpha_prev + (1-beta) alpha_cur, beta = min(0.9, (1+t)/(10+t)) (Eq. 4).
 *   init != 0 (batch 0 of an epoch): residue method: r = x; for j = 0..k-1: b_j = [r >= 0],
 *     alpha_j = mean |r|, r <- r - alpha_j b_j; alpha_prev is not read; no Eq. 3/4 update.
 *   The stream carries alpha_next and m_q = mean(B alpha_next - x) (Eq. 5); the receiver
 *     computes xhat = level(c) - m_q.  The sums over the tensor behind Eq. 3 and Eq. 5 (B^T x, the sum
 *     of x, and the mean |r| of the residue method) are taken WITHOUT rounding and rounded once to double:
 *     alpha_next and m_q are a function of the input alone, whatever the order in which threads add (the
 *     k x k system is then solved in double by Gaussian elimination with partial pivoting; a pivot below
 *     1e-9 N counts as singular).  Non-finite input is not supported: ACCEPT_DEV_NONFINITE is set, such
 *     values are left out of the sums and the codes are unspecified.
 * Stream: [0,32) header (magic, version, n low, n high, 0, k, 0, 1), [32, 32+4k) alpha_next,
 *   then m_q, zero pad to a multiple of 16, then bit planes: group g of 32 elements owns words
 *   g*k .. g*k+k-1, bit t of word g*k+j = [b_(32g+t),j = +1] ("-1 replaced by 0").
 * k in {2,3,4} (the paper's forward range); d_alpha_prev / d_alpha_next are DEVICE arrays of k
 * floats (they may be the same array), so successive batches chain without a host round trip.
 * The workspace (accept_mbq_workspace_size bytes = 624, 16-byte aligned, zeroed once by the caller) holds
 * the status word, the residue coefficients and the exact sums (every call leaves them zeroed again; a
 * workspace serves one call at a time).  Launches: 1 (plus k when init).  The encode
 * kernel of a batch >= 1 asks for 128 KB of dynamic shared memory per block (its search table).
 */
typedef struct {
  uint64_t n_elems;
  uint32_t k;
  uint32_t batch_index; /* t of Eq. 4 */
  uint32_t init;        /* 1: residue-based initialisation */
  uint32_t reserved;    /* must be 0 */
} accept_mbq_params;

accept_status accept_mbq_check_params(const accept_mbq_params* p);
size_t accept_mbq_compressed_size(const accept_mbq_params* p); /* 0 if p is invalid */
size_t accept_mbq_payload_offset(const accept_mbq_params* p);
size_t accept_mbq_workspace_size(const accept_mbq_params* p);
accept_status accept_mbq_compress(const accept_mbq_params* p, const float* d_x, const float* d_alpha_prev,
                                  float* d_alpha_next, void* d_stream, size_t stream_bytes, void* d_ws,
                                  size_t ws_bytes, void* cuda_stream);
/* Reads k and n from p; the kernel checks them against the header (ACCEPT_DEV_BAD_HEADER). */
accept_status accept_mbq_decompress(const accept_mbq_params* p, const void* d_stream, size_t stream_bytes,
                                    float* d_xhat, void* d_ws, size_t ws_bytes, void* cuda_stream);

/* ---------------------------------------------------------------------------------------------
 * Operators beside the codec: what the stage that receives a boundary tensor runs on it first.
 * Layer norm forward and backward, quantisation to 8-bit floating point with one power-of-two scale
 * for each block of 128 values, and the matrix product of operands in that form (the linear layer's
 * forward product and both of its gradients).  They follow the rules of the entry points above:
 * asynchronous on the stream, nothing allocated, buffers and workspace owned by the caller.  Of a workspace
 * only the status word (word 0) has a meaning from one call to the next; these entry points may share one,
 * for any sizes, as long as one call at a time uses it.  The paper has no counterpart of them.
 */
typedef enum { ACCEPT_DTYPE_F32 = 0, ACCEPT_DTYPE_BF16 = 1, ACCEPT_DTYPE_F16 = 2 } accept_dtype;
/* 8-bit formats: E4M3 without infinities (largest value 448) and E5M2 (largest finite value 57344). */
typedef enum { ACCEPT_FORMAT_E4M3 = 0, ACCEPT_FORMAT_E5M2 = 1 } accept_format;
/* Values that share a scale: 128 neighbours of a row, or 128 x 128. */
typedef enum { ACCEPT_BLOCK_ROW = 0, ACCEPT_BLOCK_SQUARE = 1 } accept_block;

/*
 * Layer norm over the rows of a rows x cols matrix.
 *   forward   mean = sum x / cols,  var = sum (x - mean)^2 / cols,  rstd = 1 / sqrt(var + eps),
 *             y = (x - mean) rstd gamma + beta
 *   backward  xhat = (x - mean) rstd,  h = dy gamma,
 *             dx = rstd (h - mean(h) - xhat mean(h xhat)),  dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
 *   rows, cols  rows >= 0 (no rows: the forward pass does nothing, the backward pass writes zero dgamma and
 *               dbeta), 1 <= cols < 2^31.
 *   ld_x, ld_y  values between the starts of two rows (>= cols) of x and dx, and of y and dy.
 *   dtype_x     type of x and dx;  dtype_y: of y and dy;  dtype_w: of gamma and beta.  Statistics and the
 *               gradients of gamma and beta are fp32, as is everything computed on the way.
 * Pointers need the alignment of their values; rows that start on 16-byte boundaries are read in 16-byte
 * pieces.  y may be x, and dx may be x or dy (the whole matrix, where type and row stride are the same); no
 * other output may overlap anything.  A row that holds a NaN or an infinity comes out as NaN; other rows do not notice.
 */
typedef struct {
  uint64_t rows, cols;
  uint64_t ld_x, ld_y;
  float eps;       /* >= 0 */
  int32_t dtype_x; /* accept_dtype */
  int32_t dtype_y;
  int32_t dtype_w;
} accept_layer_norm_params;

accept_status accept_layer_norm_check_params(const accept_layer_norm_params* p);
size_t accept_layer_norm_workspace_size(const accept_layer_norm_params* p); /* of the backward pass; 0 if p is invalid */
/* gamma and beta may each be NULL (1 and 0); mean and rstd (rows values each) may be NULL where no backward pass follows. */
accept_status accept_layer_norm_forward(const accept_layer_norm_params* p, const void* d_x, const void* d_gamma,
                                        const void* d_beta, void* d_y, float* d_mean, float* d_rstd, void* cuda_stream);
/* d_gamma may be NULL (1).  dx, or dgamma and dbeta, may be NULL: then they are not written.  dgamma and dbeta are
 * summed in an order that depends on the sizes alone: the same call gives the same bits.  d_ws: 16-byte aligned. */
accept_status accept_layer_norm_backward(const accept_layer_norm_params* p, const void* d_dy, const void* d_x,
                                         const void* d_gamma, const float* d_mean, const float* d_rstd, void* d_dx,
                                         float* d_dgamma, float* d_dbeta, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * Quantisation to 8-bit floating point in blocks of 128.
 *   block  ROW: 128 consecutive values of a row (the last block of a row may be shorter);  SQUARE: 128 x 128
 *   scale  a = the largest finite |x| of the block; e = the least integer with a 2^-e <= F (the format's largest
 *          value), held to [-127, 127]; 0 where a = 0.  Scale byte e + 127.
 *   code   x 2^-e (exact) rounded to the format, ties to even.  NaN and infinities become the format's NaN, and
 *          ACCEPT_DEV_NONFINITE is set in the status word.
 * One read of x gives either or both of
 *   rows     q (rows x cols): blocks run along the columns;
 *   columns  q_t (cols x rows): the transpose, blocks run along the rows.
 * A square block has the same scale in both.  Layout of a coded R x C matrix (R = rows or cols):
 *   codes    R rows of C bytes, each row padded with zero bytes to a multiple of 16
 *            (accept_block_data_size bytes, 16-byte aligned);
 *   scales   the order in which the tensor cores read them: 512 bytes for 128 rows and four blocks; the byte of row r
 *            and block b is at ((b / 4) ceil(R / 128) + r / 128) 512 + (r % 32) 16 + (r / 32 % 4) 4 + b % 4
 *            (accept_block_scale_size bytes, 16-byte aligned; rows and blocks of the padding hold 127).
 *            Square blocks repeat their byte for each row.
 *   rows, cols  >= 0, below 2^31;  ld: values between the starts of two rows of x (>= cols)
 */
typedef struct {
  uint64_t rows, cols;
  uint64_t ld;
  int32_t dtype;  /* accept_dtype of x */
  int32_t format; /* accept_format */
  int32_t block;  /* accept_block */
  int32_t reserved; /* 0 */
} accept_quantize_params;

accept_status accept_block_check_params(const accept_quantize_params* p);
/* Bytes of the codes and of the scales, of q (transposed = 0) or q_t (1); 0 if p is invalid. */
size_t accept_block_data_size(const accept_quantize_params* p, int transposed);
size_t accept_block_scale_size(const accept_quantize_params* p, int transposed);
size_t accept_block_workspace_size(const accept_quantize_params* p);
/* q and its scales, or q_t and its scales, may be NULL; not both. */
accept_status accept_block_quantize(const accept_quantize_params* p, const void* d_x, void* d_q, void* d_scale, void* d_qt,
                                    void* d_scale_t, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * d = a b^T (+ bias) (+ d):  d[i][j] = sum_k a[i][k] 2^(ea - 127) b[j][k] 2^(eb - 127) + bias[j] + (accumulate) d[i][j]
 * for a (m x k) and b (n x k) as accept_block_quantize writes them, scale bytes 0 to 254.  Products are exact, sums are
 * fp32 in an order that depends on the sizes alone, d is rounded once.
 *   linear layer y = x W^T + b:   forward  a = x by rows, b = W by rows;  gradient of x: a = dy by rows, b = W by columns;
 *   gradient of W: a = dy by columns, b = x by columns, accumulate into fp32.
 *   m, n, k >= 0, below 2^31 (k = 0: the sum is empty);  ldd: values between the starts of two rows of d (>= n)
 */
typedef struct {
  uint64_t m, n, k;
  uint64_t ldd;
  int32_t format_a, format_b; /* accept_format */
  int32_t dtype_d;            /* accept_dtype */
  int32_t accumulate;         /* 0 or 1: add to what d holds */
} accept_matmul_params;

accept_status accept_matmul_check_params(const accept_matmul_params* p);
size_t accept_matmul_workspace_size(const accept_matmul_params* p);
/* bias: n fp32 values, or NULL.  d_ws: 16-byte aligned.  The status word gets ACCEPT_DEV_COPY_TIMEOUT if a wait inside the
 * kernel ran out: then d is unspecified, and the whole workspace is to be zeroed before a captured graph repeats that call. */
accept_status accept_block_matmul(const accept_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b,
                                  const void* d_b_scale, const float* d_bias, void* d_d, void* d_ws, size_t ws_bytes,
                                  void* cuda_stream);

/* ---------------------------------------------------------------------------------------------
 * Operators of a residual stage: dropout, the root-mean-square norm of a residual stream and its gradient, and the linear
 * layer in 4 bits.  The rules are those of the operators above.  The paper has no counterpart.
 */

/*
 * Dropout: y[i][j] = residual[i][j] + (U >= p ? x[i][j] / (1 - p) : 0), U the number of counter rng_offset + i cols + j (mod 2^64) under
 * `seed`, drawn as at accept_params.seed.  No mask is stored: the backward pass is the same call with dy in the place of x and no
 * residual (the residual's gradient is dy itself).  Advance rng_offset by rows * cols between calls to draw fresh numbers.
 * Seed and counter are taken when the call is made: a captured call draws the same numbers at every replay.
 *   p            0 (nothing is dropped) to 1 (everything is); 1 / (1 - p) is rounded to fp32 once, product and sum are fp32
 *                operations, y is rounded once.  What is dropped is 0, also where x is a NaN or an infinity.
 *   rows, cols   >= 0;  ld_x, ld_y: values between the starts of two rows of x, and of residual and y (>= cols).
 *   dtype_x      type of x;  dtype_y: of residual and y.
 * residual may be NULL (0).  Pointers need the alignment of their values.  y may be x or residual (the whole matrix, where type and
 * row stride are the same); otherwise it overlaps neither.
 */
typedef struct {
  uint64_t rows, cols;
  uint64_t ld_x, ld_y;
  uint64_t seed, rng_offset;
  float p;
  int32_t dtype_x; /* accept_dtype */
  int32_t dtype_y;
  int32_t reserved; /* 0 */
} accept_dropout_params;

accept_status accept_dropout_check_params(const accept_dropout_params* p);
accept_status accept_dropout(const accept_dropout_params* p, const void* d_x, const void* d_residual, void* d_y, void* cuda_stream);

/*
 * Root-mean-square norm over the rows of a residual stream, to which a branch is added first.
 *   forward   s = x + drop(branch), rounded to dtype_x;  rstd = 1 / sqrt(sum s^2 / cols + eps);  y = s rstd gamma
 *   backward  xhat = s rstd,  h = dy gamma,  dx = rstd (h - xhat mean(h xhat)) + dsum,  dbranch = drop'(dx),
 *             dgamma = sum_rows dy xhat
 * drop() is accept_dropout's with the same p, seed, rng_offset and cols (p = 0: the branch as it is), drop'() its gradient, taken of dx
 * before dx is rounded.  dsum is the gradient that reaches s by the stream itself.
 *   outputs of the forward pass, each of which may be NULL (one at least is not):  sum: s;  y;  q and scale: y in 8 bits, codes and scales
 *             as accept_block_quantize writes them for BLOCK_ROW and `format` (y is not rounded before; ACCEPT_DEV_NONFINITE as there);
 *             rstd: rows fp32 values for the backward pass.
 *   rows, cols  rows >= 0 (below 2^31 with q), 1 <= cols < 2^31.  No rows: the forward pass does nothing, the backward pass writes zero dgamma.
 *   ld_x, ld_y  values between the starts of two rows (>= cols) of x, sum, s, dsum and dx, and of branch, y, dy and dbranch.
 *   dtype_x     type of x, sum, s, dsum and dx;  dtype_y: of branch, y, dy and dbranch;  dtype_w: of gamma.  Statistics, dgamma and everything
 *               computed on the way are fp32.
 * Squares that leave the range of fp32 are taken again with scaled values; rstd itself is an fp32 value (with eps = 0 a row whose root mean
 * square is below 2^-127 comes out as infinities, a row of zeros as NaN).  A NaN makes its row NaN; an infinity makes the finite
 * values of its row 0 and itself NaN.  Pointers need the alignment of their values (q, scale and the backward pass's workspace: 16 bytes); rows that
 * start on 16-byte boundaries are read in 16-byte pieces.  sum may be x, y may be branch, dx may be s or dsum, and dbranch may be dy (the whole
 * matrix); no other output may overlap anything.
 */
typedef struct {
  uint64_t rows, cols;
  uint64_t ld_x, ld_y;
  uint64_t seed, rng_offset;
  float eps;       /* >= 0 */
  float p;         /* 0 to 1 */
  int32_t dtype_x; /* accept_dtype */
  int32_t dtype_y;
  int32_t dtype_w;
  int32_t format;  /* accept_format of q */
} accept_rms_norm_params;

accept_status accept_rms_norm_check_params(const accept_rms_norm_params* p);
size_t accept_rms_norm_workspace_size(const accept_rms_norm_params* p); /* of the backward pass; 0 if p is invalid */
/* branch and gamma may be NULL (0 and 1).  d_ws: the status word, 16 bytes, 4-byte aligned; may be NULL without q. */
accept_status accept_rms_norm_forward(const accept_rms_norm_params* p, const void* d_x, const void* d_branch, const void* d_gamma,
                                      void* d_sum, void* d_y, void* d_q, void* d_scale, float* d_rstd, void* d_ws, size_t ws_bytes,
                                      void* cuda_stream);
/* gamma and dsum may be NULL (1 and 0); dx, dbranch and dgamma may each be NULL (not written), not all.  dgamma is summed in an order
 * that depends on the sizes alone. */
accept_status accept_rms_norm_backward(const accept_rms_norm_params* p, const void* d_dy, const void* d_s, const void* d_gamma,
                                       const float* d_rstd, const void* d_dsum, void* d_dx, void* d_dbranch, float* d_dgamma,
                                       void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * 4-bit floating point (E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) with one power-of-two scale for each 32 values.
 *   block  ROW: 32 consecutive values of a row (the last block of a row may be shorter);  SQUARE: 32 x 32
 *   scale  a = the largest |x| of the block; e = the least integer with a 2^-e <= 6, held to -127 and above; 0 where a = 0.  Scale byte
 *          e + 127.  A block that holds a NaN or an infinity has scale byte 255 (NaN) and zero codes, and ACCEPT_DEV_NONFINITE
 *          is set in the status word.
 *   code   t = |x| 2^-e (exact, but that 2^-150 and less is 0) between two neighbours g < h of the list:  NEAREST: the nearer, a tie to the one with an even place in the
 *          list;  STOCHASTIC: h where U < (t - g) / (h - g), else g, U the number of counter rng_offset + i cols + j (mod 2^64) for x[i][j]
 *          under `seed`, drawn as at accept_params.seed; the comparison is exact.  Bits 0 to 2 are the place in the list, bit 3 the sign.
 * One read of x gives either or both of
 *   rows     q (rows x cols): blocks run along the columns;
 *   columns  q_t (cols x rows): the transpose, blocks run along the rows.
 * An element has the same U in both, and a square block the same scale.  Layout of a coded R x C matrix (R = rows or cols):
 *   codes    two to a byte, the even column in the lower half; R rows of C rounded up to 32 values, those past C zero codes
 *            (accept_micro_data_size bytes, 16-byte aligned);
 *   scales   as for 8-bit codes, with blocks of 32: the byte of row r and block b is at
 *            ((b / 4) ceil(R / 128) + r / 128) 512 + (r % 32) 16 + (r / 32 % 4) 4 + b % 4
 *            (accept_micro_scale_size bytes, 16-byte aligned; rows and blocks of the padding hold 127).
 *   rows, cols  >= 0, below 2^31;  ld: values between the starts of two rows of x (>= cols)
 */
typedef struct {
  uint64_t rows, cols;
  uint64_t ld;
  uint64_t seed, rng_offset; /* STOCHASTIC only */
  int32_t dtype;    /* accept_dtype of x */
  int32_t round;    /* accept_round */
  int32_t block;    /* accept_block */
  int32_t reserved; /* 0 */
} accept_micro_params;

accept_status accept_micro_check_params(const accept_micro_params* p);
/* Bytes of the codes and of the scales, of q (transposed = 0) or q_t (1); 0 if p is invalid. */
size_t accept_micro_data_size(const accept_micro_params* p, int transposed);
size_t accept_micro_scale_size(const accept_micro_params* p, int transposed);
size_t accept_micro_workspace_size(const accept_micro_params* p);
/* q and its scales, or q_t and its scales, may be NULL; not both.  x may have any alignment of its values. */
accept_status accept_micro_quantize(const accept_micro_params* p, const void* d_x, void* d_q, void* d_scale, void* d_qt, void* d_scale_t,
                                  void* d_ws, size_t ws_bytes, void* cuda_stream);
/* The values that codes by rows stand for: x[i][j] = code 2^(scale byte - 127) (byte 255: NaN), rounded to dtype once: exact but where that
 * leaves dtype's range.  So does 2^128, as which the quantiser may code values of fp32 and bf16 from 1.5 2^127 on (NEAREST: from 1.75 2^127
 * on), and 2^16 of fp16 likewise: they come back as infinities, without a bit in the status word; to a product they are the factors
 * 2^128 and 2^16.  p gives rows, cols, ld and dtype of x; its round, block, seed and rng_offset are not used.  Codes of a transpose are those
 * of a cols x rows matrix. */
accept_status accept_micro_dequantize(const accept_micro_params* p, const void* d_q, const void* d_scale, void* d_x, void* cuda_stream);

/*
 * d = a b^T (+ bias) (+ d) for a (m x k) and b (n x k) as accept_micro_quantize writes them, as accept_block_matmul: products are exact, sums are
 * fp32 in an order that depends on the sizes alone, d is rounded once.  A scale byte of 255 makes every sum that it
 * enters NaN.
 *   m, n, k >= 0, below 2^31 (k = 0: the sum is empty);  ldd: values between the starts of two rows of d (>= n)
 */
typedef struct {
  uint64_t m, n, k;
  uint64_t ldd;
  int32_t dtype_d;    /* accept_dtype */
  int32_t accumulate; /* 0 or 1: add to what d holds */
} accept_micro_matmul_params;

accept_status accept_micro_matmul_check_params(const accept_micro_matmul_params* p);
size_t accept_micro_matmul_workspace_size(const accept_micro_matmul_params* p);
/* bias: n fp32 values, or NULL.  d_ws: 16-byte aligned; ACCEPT_DEV_COPY_TIMEOUT as for accept_block_matmul. */
accept_status accept_micro_matmul(const accept_micro_matmul_params* p, const void* d_a, const void* d_a_scale, const void* d_b,
                                const void* d_b_scale, const float* d_bias, void* d_d, void* d_ws, size_t ws_bytes, void* cuda_stream);

/*
 * Synchronises cuda_stream, copies the status word to the host and returns it in *status_bits
 * (ACCEPT_DEV_* bits).  Returns ACCEPT_ERR_CUDA if the stream reports an error.
 */
accept_status accept_last_device_status(const void* d_ws, void* cuda_stream, uint32_t* status_bits);

/*
 * Parses the 32 header bytes (a HOST copy) into *out; ACCEPT_ERR_BAD_STREAM_HEADER if the magic,
 * version or any field is invalid.  For receivers that know nothing but the bytes they got (Sec. 3.4).
 */
accept_status accept_parse_header(const void* h_header, accept_params* out);

/*
 * Bit width the paper's schedule prescribes after n_lr_changes learning-rate changes:
 * forward (Sec. 3.3 "Forward Quantizer"): starts at 2, +1 per change, at most 4;
 * backward ("Backward Quantizer"): 8 until the first change, then 4.
 */
int accept_bitwidth_schedule(int is_backward, int n_lr_changes);

/* Number of kernels the library has launched in this process (all entry points). */
uint64_t accept_launch_count(void);

/*
 * Launches an EMPTY kernel of `blocks` blocks of `threads` threads on cuda_stream exactly as every kernel of
 * this library is launched (same launch attribute, same first instructions).  It measures what a launch
 * costs where a call is bound by launching rather than by bytes (tensors of a few MB): replayed from a
 * CUDA graph beside the codec's own kernels it gives the floor under their times.  The paper has no
 * counterpart.  blocks in [1, 2^31), threads in [32, 1024].
 */
accept_status accept_launch_null(uint32_t blocks, uint32_t threads, void* cuda_stream);

/*
 * For the checking build of this library (the same sources compiled with -DACCEPT_BOUNDS_CHECK, which the
 * tests load in place of a memory checker): every access of a kernel to caller memory is compared with
 * the byte ranges of the call (input, stream up to accept_compressed_size, workspace up to its size
 * query, output), and one that falls outside -- or a write into the input -- is skipped and counted
 * instead of performed.  This call synchronises cuda_stream, returns the number of skipped accesses since
 * the previous report in *violations and, optionally, the address of the first one and its size (low 32
 * bits) and kind (bit 32: write), then clears the count.  The paper has no counterpart.  In the normal
 * build nothing is checked: *violations = 0 and the result is ACCEPT_ERR_UNCHECKED_BUILD.
 */
accept_status accept_bounds_check_report(void* cuda_stream, uint32_t* violations, uint64_t* first_address,
                                         uint64_t* first_size_and_kind);

#ifdef __cplusplus
}
#endif
#endif /* ACCEPT_H_ */
