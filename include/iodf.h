/*
 * libiodf: integer-only inference of an Integer-only Discrete Flow (arXiv
 * 2206.08869) on AMD MI355X (gfx950). C ABI: plain pointers and sizes only.
 *
 * The flow maps an image x in Z^d to a latent z = f(x) of the same size and back
 * (Sec. 3). f is a stack of levels; each level squeezes space to depth, applies K
 * additive couplings  z_a = x_a, z_b = x_b + t(x_a)  (Sec. 3, Eq. 1) and factors
 * half of the channels out. t() is an integer-only network: 8-bit codes, int8 x
 * int8 convolutions with 32-bit accumulator and bias, a per-channel fixed-point
 * rescale back to 8 bit, integer ReLU (Sec. 4.1, Eq. 2-5), with gated-off filters
 * and the matching input columns of their consumers physically removed (Sec. 4.4,
 * Eq. 8); where a residual shortcut needs the unpruned width, a gated-off filter is
 * kept as an all-zero row, which adds exactly the 0 that its removal would.
 *
 * Pointer conventions: "host" = ordinary process memory; "device" = memory of
 * the GPU the context was created on, owned by the caller (for instance a
 * PyTorch-ROCm tensor's data_ptr()). `stream` is a hipStream_t passed as void*
 * (NULL = the default stream). iodf_forward / iodf_inverse only enqueue work on
 * that stream and never synchronise; the caller synchronises before reading.
 * A context must not be used from two streams at once (it owns one workspace).
 * Calls of more than 32 kernels are replayed from HIP graphs kept per (direction, batch,
 * with/without codes): the first call of a shape captures its graph on an internal stream (host
 * work only, a few ms); inputs and outputs pass through internal staging buffers with
 * device-to-device copies on the caller's stream. Shorter calls launch their kernels directly.
 * Setting IODF_NO_GRAPH=1 in the environment before iodf_init launches all kernels directly.
 *
 * Every function returns IODF_OK (0) or a negative IODF_E_* code; nothing throws.
 */
#ifndef IODF_H
#define IODF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct iodf_ctx iodf_ctx;

enum {
    IODF_OK = 0,
    IODF_E_ARG = -1,    /* NULL or out-of-range argument */
    IODF_E_BLOB = -2,   /* malformed model blob (magic, truncation, bad constants) */
    IODF_E_SHAPE = -3,  /* blob is well formed but its layers do not fit the declared family */
    IODF_E_BATCH = -4,  /* batch < 0 or batch > max_batch */
    IODF_E_HIP = -5,    /* a HIP runtime call failed (iodf_last_hip_error has the code) */
    IODF_E_NOMEM = -6,  /* host or device allocation failed */
    IODF_E_SCRATCH = -7 /* iodf_encode_noalloc: the batch needs more than the static scratch holds */
};

/* What iodf_query reports. */
enum {
    IODF_Q_Z_ELEMS = 0,          /* d: int32 latent elements per image (= 3*H*W) */
    IODF_Q_CODE_BYTES = 1,       /* int8 prior-parameter codes per image (0 without heads) */
    IODF_Q_WORKSPACE_BYTES = 2,  /* device memory held by the context */
    IODF_Q_MACS_FORWARD = 3,     /* algorithmic multiply-accumulates per image, kept channels only, true widths */
    IODF_Q_MACS_INVERSE = 4,     /* same for decode (no prior heads) */
    IODF_Q_RANGE_ERRORS = 5,     /* pixels outside [0,255] met by iodf_inverse since the last query;
                                    synchronises the device and resets the counter */
    IODF_Q_MAX_BATCH = 6,
    IODF_Q_IMAGE_H = 7,
    IODF_Q_IMAGE_W = 8,
    IODF_Q_CONV_LAUNCHES = 9,    /* convolution kernels of a forward call of max_batch images, heads included */
    IODF_Q_WIDE_MACS_FORWARD = 10, /* of IODF_Q_MACS_FORWARD, the part in layers whose C_in and C_out are both >= 128 */
    IODF_Q_CODEC_HEADER_WORDS = 11, /* 32-bit words of a container's header: 1 + 3 * 16 * levels */
    IODF_Q_CODEC_MAX_WORDS = 12,    /* capacity no container exceeds: header + d (a latent sheds at most one word) */
    IODF_Q_CODEC_CLAMPED = 13,      /* latents whose residual z - mu left [-8192, 8191] and was clamped (the image
                                       then does NOT decode back); 13..15 synchronise and reset like RANGE_ERRORS */
    IODF_Q_CODEC_OVERFLOWS = 14,    /* containers that needed more than cap_words (truncated, unusable) */
    IODF_Q_CODEC_BROKEN_LANES = 15, /* coder lanes that iodf_decode could not read back to their initial state
                                       (malformed or foreign container) */
    IODF_Q_NOALLOC_MAX_BATCH = 16,  /* largest batch iodf_encode_noalloc accepts for this model (<= max_batch) */
    IODF_Q_GRAPHS = 17              /* call shapes whose graph the context holds */
};

/*
 * Build a context from a model blob (Sec. 4.1, 4.4: weights, per-channel rescale
 * constants, binary gates).
 *   out          host; receives the context (caller releases it with iodf_free).
 *   model_blob   host; little-endian, 4-byte aligned fields:
 *                  header 16 x u32: 'IODF','BLB1', version 1, H, W, levels, couplings per
 *                    level, family (0 plain, 1 residual, 2 dense), width, depth, has_heads,
 *                    n_nets, act_unsigned (0 | 1), 3 x reserved (0)
 *                  per network in flow order (level 1 couplings, level 1 head, level 2, ...):
 *                    8 x 32 bit: kind (0 coupling, 1 head), level, C_level, C_in, C_out,
 *                    n_layers, M_in (i32), s_in; then i32 perm[C_level] for couplings;
 *                    per conv layer: 4 x u32 C_out, C_in, k (1|3), flags (bit0 ReLU, bit1
 *                    shortcut); i8 W[C_out][C_in][k][k]; i32 bias[C_out]; i32 M[C_out];
 *                    u8 shift[C_out]; u8 gate[C_out] (1 = keep); arrays padded to 4 bytes.
 *                The blob is copied/repacked; the caller may free it on return. Filters with
 *                gate 0 and the matching input columns of their consumers are removed here,
 *                so they cost nothing at inference.
 *   device_ordinal  HIP device to run on.
 *   max_batch    largest batch later calls may pass (sizes the workspace); >= 1.
 * act_unsigned = 1 selects the paper's hybrid number format (Sec. 4.1, Eq. 3): every tensor that
 * leaves a ReLU holds unsigned codes 0..255 (saturation at 255), read as such by the next
 * convolution and by the shortcut; the input quantiser's output, the translation and the head
 * codes stay signed. Every hidden layer must then carry a ReLU and the last layer none.
 * Constants must satisfy 0 <= M < 2^31, 0 <= shift <= 62, |bias| < 2^30, and for every filter
 * |bias| + X * sum|w| < 2^31 with X = 128 (256 for a layer reading unsigned codes), so that the
 * 32-bit accumulator of Eq. 4-5 cannot overflow for any input; a blob that breaks one of these is
 * refused with IODF_E_BLOB.
 */
int iodf_init(iodf_ctx** out, const void* model_blob, size_t blob_bytes, int device_ordinal, int max_batch);

/*
 * Encode (Sec. 3: z = f(x)).
 *   x_dev      device, uint8 [batch][3][H][W]; read only.
 *   z_dev      device, int32 [batch][d]; per image the concatenation over levels l = 1..L of
 *              the factored-out chunk [C_z,l][h_l][w_l] (last level: all channels).
 *   codes_dev  device, int8 [batch][code bytes], or NULL to skip the prior heads; per image
 *              the concatenation over heads l = 1..L-1 of [2*C_z,l][h_l][w_l]: first C_z,l maps
 *              are the codes of the logistic prior's mean, the rest of its log-scale (Sec. 3).
 * batch may be 0 (no work).
 */
int iodf_forward(iodf_ctx* ctx, const uint8_t* x_dev, int batch, int32_t* z_dev, int8_t* codes_dev, void* stream);

/*
 * Decode (Sec. 3: x = f^{-1}(z)): couplings replayed in reverse, x_b = z_b - t(z_a).
 *   z_dev  device, int32 [batch][d], layout as written by iodf_forward; read only.
 *   x_dev  device, uint8 [batch][3][H][W]. A z that is no image of any x can decode to a
 *          value outside [0,255]: the byte is saturated and counted (IODF_Q_RANGE_ERRORS).
 */
int iodf_inverse(iodf_ctx* ctx, const int32_t* z_dev, int batch, uint8_t* x_dev, void* stream);

/*
 * Compressor: bits = rANS(f(x); p_Z) and back (Sec. 3 prior, Sec. 5.2 "actual encoding", App. A).
 *
 * Prior of a latent z with mean code m and log-scale code l (int8, from the level's head;
 * m = 0, l = 96 for latents without a head): discretised logistic with mu = 2 m, s = 2^(l/16),
 * evaluated in integers: cumulative mass G(r) = (r + 8192) + floor((2^24 - 16384) *
 * S((2r - 1)/(2s)) / 2^30) over the residual r = z - mu in [-8192, 8191], S a 3073-entry table
 * of round(2^30 sigma(t)) at t = -24 + j/64 with linear interpolation; C = G(r), F = G(r+1) - G(r)
 * >= 1, total mass M = 2^24.
 * Coder: App. A's recurrences on a 64-bit state in [2^31, 2^63) that starts at 2^31 and sheds /
 * refills 32-bit words; a level's latents are dealt round-robin to 16 independent lanes.
 * Container of one image (little-endian u32 words): total word count; words per (level, lane);
 * final state (low, high) per (level, lane); then each lane's words in decoding order.
 *
 * iodf_prior_cf: z_dev int32 [batch][d], codes_dev int8 [batch][code bytes] (required when the
 *   model has heads, ignored otherwise) -> c_dev, f_dev int32 [batch][d] (device).
 * iodf_encode: x_dev uint8 [batch][3][H][W] -> words_dev u32 [batch][cap_words] (one container
 *   per image, never written past cap_words) and sizes_dev u32 [batch] (words each container
 *   needs; larger than cap_words means truncated, see IODF_Q_CODEC_OVERFLOWS).
 * iodf_decode: containers -> x_dev. cap_words must be at least the header size. Malformed
 *   containers never cause out-of-range reads; they are counted (IODF_Q_CODEC_BROKEN_LANES).
 * The first of these calls on a context allocates the compressor's device buffers. Calls on one
 * context must not overlap. iodf_codec_tables copies the two tables (host: int32 sig[3073],
 * int64 inv[256] = round(2^23 * 2^(-l/16)) at index l + 128); it needs no GPU.
 */
int iodf_prior_cf(iodf_ctx* ctx, const int32_t* z_dev, const int8_t* codes_dev, int batch, int32_t* c_dev,
                  int32_t* f_dev, void* stream);
int iodf_encode(iodf_ctx* ctx, const uint8_t* x_dev, int batch, uint32_t* words_dev, int64_t cap_words,
                uint32_t* sizes_dev, void* stream);
int iodf_decode(iodf_ctx* ctx, const uint32_t* words_dev, int64_t cap_words, int batch, uint8_t* x_dev, void* stream);
int iodf_codec_tables(int32_t* sig_host, int64_t* inv_host);

/*
 * iodf_encode for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc. Same arguments, same containers, word for word.
 * The coder's working buffers (the batch's latents and codes, the words each lane sheds, lane
 * states, the prior's tables and the error counters), which iodf_encode allocates on its first
 * call, live in a 64 MiB array that is part of the library's device image; each GPU holds one copy
 * from the moment the library is loaded until the process ends, and iodf_init prepares it. The call
 * allocates and frees nothing and launches the flow kernel by kernel instead of replaying a graph.
 * A batch whose buffers do not fit returns IODF_E_SCRATCH before anything is enqueued
 * (IODF_Q_NOALLOC_MAX_BATCH tells the limit for a model: 554 images of 3x64x64 with prior heads on four levels).
 * All contexts on one GPU share that GPU's array: calls that overlap on one GPU (from any context,
 * on any streams) race; serialise them. The error counters of these calls are shared per GPU too and
 * are reported, and reset, by iodf_query(IODF_Q_CODEC_*) of any context that used this entry point.
 */
int iodf_encode_noalloc(iodf_ctx* ctx, const uint8_t* x_dev, int batch, uint32_t* words_dev, int64_t cap_words,
                        uint32_t* sizes_dev, void* stream);

/*
 * Patch-based coding of images larger than the flow's H x W (Sec. 5.2: a large image is coded as
 * a batch of patches). img_dev: device, planar uint8 [3][img_h][img_w]. The image is covered by a
 * row-major grid of ceil(img_h/H) x ceil(img_w/W) patches; iodf_tile_patches writes patches
 * first_patch .. first_patch + n_patches - 1 to x_dev (uint8 [n_patches][3][H][W], ready for
 * iodf_forward / iodf_encode), reading 128 where a patch sticks out of the image;
 * iodf_untile_patches copies decoded patches back, dropping what lies outside. Patches beyond the
 * grid are an argument error.
 */
int iodf_tile_patches(iodf_ctx* ctx, const uint8_t* img_dev, int img_h, int img_w, int first_patch, int n_patches,
                      uint8_t* x_dev, void* stream);
int iodf_untile_patches(iodf_ctx* ctx, const uint8_t* x_dev, int first_patch, int n_patches, uint8_t* img_dev,
                        int img_h, int img_w, void* stream);

/*
 * One integer-only convolution layer on its own: the isolated shapes the paper times in its
 * architecture argument (Sec. 4.3, Table 1). All tensors are HOST memory, channel-first:
 * x int8 [batch][c_in][h][w], w int8 [c_out][c_in][k][k], bias / m int32 [c_out], shift u8 [c_out]
 * (same constraints as in a blob), y int8 [batch][c_out][h][w] = sat8(relu?(rq(conv(x) + bias))).
 * The layer is packed and run exactly as inside a flow (same kernels, zero padding (k-1)/2); the
 * call allocates and frees its own device buffers, runs the layer once for y and then `iters` more
 * times between two events: *us_per_call (may be NULL) is the mean device time of one launch.
 * k is 1 or 3; h, w <= 8192; c_in, c_out <= 65536; anything else is IODF_E_ARG.
 * Measurement support, not part of the coding path.
 */
int iodf_conv_probe(int device_ordinal, int c_in, int c_out, int k, int h, int w, int batch, int relu,
                    const int8_t* x_host, const int8_t* w_host, const int32_t* bias_host, const int32_t* m_host,
                    const uint8_t* shift_host, int8_t* y_host, int iters, float* us_per_call);

/*
 * iodf_conv_probe plus a per-tile timeline of one more launch that follows `iters` further back-to-back
 * launches (so it sees the clocks of sustained work). timeline_host: int64 [max_tiles][8], one row per
 * output tile that ran (*n_tiles rows): [0..3] the constant 100 MHz counter when the tile's workgroup
 * started on it, when its first k-tile had landed, after its k loop and after its epilogue; [4], [5] the
 * shader-clock counter at start and end, so (row[5] - row[4]) / (row[3] - row[0]) x 100 MHz is the clock the
 * compute unit ran at; [6], [7] zero. y is what the traced launch wrote. A layer over so few pixels that a flow
 * runs it by a kernel without stamps is run, timed and traced by the one that a flow takes for more of them.
 * Measurement support for the roofline analysis, not part of the coding path.
 */
int iodf_conv_probe_timeline(int device_ordinal, int c_in, int c_out, int k, int h, int w, int batch, int relu,
                             const int8_t* x_host, const int8_t* w_host, const int32_t* bias_host,
                             const int32_t* m_host, const uint8_t* shift_host, int8_t* y_host, int iters,
                             float* us_per_call, int64_t* timeline_host, int max_tiles, int* n_tiles);

/*
 * Per-kernel timing for roofline reports (the paper reports latency only, Sec. 5.2; this is
 * measurement support, not part of the method). Between begin and end every kernel launch of
 * iodf_forward / iodf_inverse is bracketed by HIP events on the caller's stream (no
 * synchronisation is added). max_launches bounds the launches recorded; later ones run untimed.
 * iodf_profile_end waits for the recorded work, then fills stats (host, caller-owned, up to
 * max_stats entries, one per kernel that ran) and *n_stats.
 */
typedef struct iodf_kernel_stat {
    char name[48];      /* kernel, e.g. "k_quant_in"; a conv kernel's launches are listed per filter size:
                           "conv_igemm<256,256,2,4,4> 3x3" and "conv_igemm<256,256,2,4,4> 1x1"; entries whose
                           name starts with "view:" sum conv launches already listed (the wide layers, alone in their
                           launch; "k_chain", a whole network in one, is in no view) */
    int64_t launches;
    double total_ms;    /* sum of event-measured durations */
    int64_t macs;       /* algorithmic multiply-accumulates of those launches (kept channels, true widths) */
    int64_t bytes;      /* algorithmic bytes: live inputs + outputs (+ weights) read or written once */
    int64_t issued_macs; /* multiply-accumulates the matrix cores ran: whole tiles at padded widths (0: not a conv) */
} iodf_kernel_stat;
int iodf_profile_begin(iodf_ctx* ctx, int max_launches);
int iodf_profile_end(iodf_ctx* ctx, iodf_kernel_stat* stats, int max_stats, int* n_stats);

/*
 * Training operators of residual blocks, for fitting a network such as a prior head to the latents that iodf_forward gives. They
 * need no context: they work on the current device of the calling thread, only enqueue on `stream`, allocate nothing and keep
 * nothing between calls; scratch is the caller's (iodf_join_workspace, iodf_weight_grad_workspace). All pointers are device
 * memory. A tensor is rows x cols with consecutive columns; strides count elements from row to row and are at least the columns.
 * Any element address will do. rows may be 0 (no work; gradients that sum over rows are then 0); 0 <= rows <= 2^30,
 * 1 <= cols <= 65536, rows * (cols rounded up to 32) <= 2^34. `live` (may be NULL) holds a byte for each row, 0 where the row
 * is padding: its entries in tensors may be anything, NaN included, and add nothing to any gradient.
 *
 * What the backward pass needs is kept as a checkpoint in 8 bits. For rows x cols values, with pitch = cols rounded up to 32:
 * q int8 [rows][pitch] (16-byte aligned) and e uint8 [rows][pitch / 32], one exponent for 32 columns; q * 2^(e - 133) is the value.
 * e is the biased exponent of the group's largest magnitude, or one more where that would round to 128 steps, limited to
 * 16..254; q is rounded to nearest, ties to even, limited to -127..127. e = 255: the group held a NaN or an infinity and reads
 * as NaN throughout. Columns past cols are written as 0. Padded rows are written as 0.
 */
enum { IODF_T_F32 = 0, IODF_T_BF16 = 1, IODF_T_F16 = 2 };
enum { IODF_ACT_RELU = 0, IODF_ACT_SILU = 1, IODF_ACT_GELU = 2 /* the tanh form */ };

/* x [rows][cols] of x_type -> checkpoint, and a checkpoint -> y of y_type (F32 or BF16, in both of which it is exact). */
int iodf_pack(const void* x, int x_type, int64_t x_stride, int64_t rows, int cols, const uint8_t* live, int8_t* q, uint8_t* e,
              void* stream);
int iodf_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int cols, void* y, int y_type, int64_t y_stride, void* stream);

/*
 * The join of two blocks of a residual network: the norm behind a block's output f, its gate and residual scale, the addition
 * to the stream h, and the norm before the next block, in one pass.
 *   n = f / rms(f),  h' = h + alpha * gate * w_post * n,  x = h' / rms(h'),  u = w_pre * x      rms(v) = sqrt(mean(v^2) + eps)
 * Sums and everything between loads and stores are 32-bit floats; x is taken from h' before it is rounded to the stream's type.
 * w_post NULL: no norm behind the block, n = f. w_pre NULL: none before the next, no x and no u. gate NULL and alpha NULL: 1.
 * Row t reads gate row t / gate_rows (gate_rows 1: a gate for each row; gate_rows >= rows: one gate for all). In a padded row
 * h' = h, to the bit, and u = 0, whatever stands in its gate, too. out_stream may be in_stream (same stride); otherwise outputs overlap no inputs.
 * The stream's type is F32 or the block's type; 1 <= cols <= 16384; eps > 0.
 *
 * iodf_join_forward: in_stream = h, in_block = f -> out_stream = h', out_block = u; with xq, not NULL, also the checkpoints of
 *   x and n and the factors inv_pre = 1 / rms(h'), inv_post = 1 / rms(f) of each row (0 in padded rows).
 * iodf_join_backward: in_stream = dL/dh', in_block = dL/du and the checkpoint -> out_stream = dL/dh, out_block = dL/df
 *   (rounded to those types; may not overlap anything) and the sums dalpha [1], dgate [gate rows][cols], dw_post [cols],
 *   dw_pre [cols] (each NULL exactly where its parameter is). x and n stand for what the checkpoint holds. At most 2^21 gate rows,
 *   or one for each row; with no rows dgate is one row. The result is the same bits on every call.
 */
typedef struct iodf_join {
    int64_t rows, gate_rows;
    int32_t cols, stream_type, block_type;
    float eps;
    const float* alpha;
    const float* gate;
    const float* w_post;
    const float* w_pre;
    const uint8_t* live;
    const void* in_stream;
    const void* in_block;
    void* out_stream;
    void* out_block;
    int64_t in_stream_stride, in_block_stride, out_stream_stride, out_block_stride;
    int8_t* xq;
    uint8_t* xe;
    int8_t* nq;
    uint8_t* ne;
    float* inv_pre;
    float* inv_post;
    float* dalpha;
    float* dgate;
    float* dw_post;
    float* dw_pre;
} iodf_join;
int iodf_join_forward(const iodf_join* args, void* stream);
int iodf_join_backward(const iodf_join* args, void* work, int64_t work_bytes, void* stream);
int iodf_join_workspace(const iodf_join* args, int64_t* bytes);

/*
 * The gated activation y = act(a) * b of a block's hidden layer.
 * iodf_glu_forward: a, b -> y; with aq not NULL also the checkpoints of a and b.
 * iodf_glu_backward: the checkpoints and dy = dL/dy -> a_out = dL/da, b_out = dL/db and, with yq not NULL, the checkpoint of
 *   y as the checkpoints of a and b give it: the input of the projection behind, for that one's weight gradient.
 * One type for a, b, y, dy and the gradients.
 */
typedef struct iodf_glu {
    int64_t rows;
    int32_t cols, type, act;
    const uint8_t* live;
    const void* a;
    const void* b;
    void* y;
    const void* dy;
    void* da;
    void* db;
    int64_t a_stride, b_stride, y_stride, dy_stride, da_stride, db_stride;
    int8_t* aq;
    uint8_t* ae;
    int8_t* bq;
    uint8_t* be;
    int8_t* yq;
    uint8_t* ye;
} iodf_glu;
int iodf_glu_forward(const iodf_glu* args, void* stream);
int iodf_glu_backward(const iodf_glu* args, void* stream);

/*
 * Gradient of a linear layer's weight W [out][cols] from the checkpoint of its input:
 *   dw[o][c] = (accumulate ? dw[o][c] : 0) + col_scale[c] * sum_t dy[t][o] * X[t][c]
 * dy [rows][out] of dy_type, X what the checkpoint stands for, dw F32 with rows dw_stride apart. col_scale (may be NULL): the
 * weight of the norm between the checkpoint and the layer (w_pre of iodf_join). In a padded row neither dy nor the checkpoint adds
 * anything, whether the checkpoint was packed with `live` or without. Products are exact for every dy_type
 * (in 32 bits of numbers from 2^-109 on; of smaller ones, what lies below 2^-133 may be lost),
 * sums are 32-bit floats, in an order that depends on the sizes alone. 1 <= out <= 65536,
 * rows * (out rounded up to 32) <= 2^34.
 */
typedef struct iodf_wgrad {
    int64_t rows;
    int32_t cols, out, dy_type, accumulate;
    const void* dy;
    int64_t dy_stride;
    const int8_t* q;
    const uint8_t* e;
    const float* col_scale;
    const uint8_t* live;
    float* dw;
    int64_t dw_stride;
} iodf_wgrad;
int iodf_weight_grad(const iodf_wgrad* args, void* work, int64_t work_bytes, void* stream);
int iodf_weight_grad_workspace(const iodf_wgrad* args, int64_t* bytes);

/*
 * The two ends of a training step: the loss over a table of classes, and orthogonalised updates of weights. Memory, streams, rows and padding
 * are as for the training operators above.
 *
 * Softmax cross entropy of rows u [rows][cols] against a table W [classes][cols], both of `type`, without the logits ever being in memory:
 *   s[t][v] = sum_c u[t][c] W[v][c],  lse[t] = log sum_v exp s[t][v],  loss[t] = lse[t] - s[t][target[t]]
 * iodf_class_loss_forward: loss, lse (F32 [rows]; 0 in padded rows). dloss, dlse, du and dw are not looked at.
 * iodf_class_loss_backward: lse as the forward pass gave it, dloss = dL/dloss and dlse = dL/dlse (either may be NULL: 0) ->
 *   du[t][c] = sum_v g[t][v] W[v][c] and dw[v][c] = sum_t g[t][v] u[t][c] of `type` (either may be NULL: not computed), with
 *   g[t][v] = (dloss[t] + dlse[t]) exp(s[t][v] - lse[t]) - (v == target[t]) dloss[t], the exponential being 1 at most.
 *   It goes over the classes in pieces whose g fits 512 MB (a tile's 64 to 256 classes at least). In 16-bit types g is rounded to that type after it is multiplied so that
 *   the first dloss that is not 0, of 64 rows spread over all, is a power of two (in half precision the largest); where few of them make up a gradient (16 rows, 32
 *   classes, 128 columns or 2^16 of them) it has two parts, so that gradients are off by hardly more than their own rounding; elsewhere by 1.1 to 1.3 times that. In F32 numbers are multiplied
 *   exactly but for what is 2^-25 of a product and less, however large or small others are. The forward pass multiplies F32 numbers of more than 64 rows in two
 *   parts of 11 bits each, exact to 2^-22 of the number, or to 2^-51 of its own row's or class's largest.
 * `live` as above: a padded row's u, target, lse, dloss and dlse may be anything; its du is 0. A target outside 0..classes-1 in any other row makes that
 * row's loss, du and all of dw NaN. Sums are in an order that depends on the sizes and the type, not on which gradients are asked
 * for, and in the forward pass of up to 16 rows of 16 bits on whether w's columns are a multiple of 64 and its rows start at multiples of 16 bytes. With no rows dw is 0.
 * 0 <= rows <= 2^24, 1 <= classes <= 2^20, 1 <= cols <= 65536, rows and classes times cols <= 2^34, rows times classes <= 2^38. Outputs overlap no
 * inputs. The workspace depends on sizes, type, strides, on which of the pointers are NULL and on how u and w are aligned: it is asked for with the same
 * arguments.
 */
typedef struct iodf_class_loss {
    int64_t rows;
    int32_t classes, cols, type, reserved;
    const void* u;
    const void* w;
    int64_t u_stride, w_stride;
    const int64_t* target;
    const uint8_t* live;
    float* loss;
    float* lse;
    const float* dloss;
    const float* dlse;
    void* du;
    void* dw;
    int64_t du_stride, dw_stride;
} iodf_class_loss;
int iodf_class_loss_forward(const iodf_class_loss* args, void* work, int64_t work_bytes, void* stream);
int iodf_class_loss_backward(const iodf_class_loss* args, void* work, int64_t work_bytes, void* stream);
int iodf_class_loss_workspace(const iodf_class_loss* args, int backward, int64_t* bytes);

/*
 * A gradient made nearly orthogonal: G [rows][cols] divided by its Frobenius norm + eps, then `steps` times an odd polynomial of its singular values,
 *   X <- a X + b (X X') X + c (X X')^2 X,
 * which brings all but the smallest of them near 1 and leaves the singular vectors. `count` matrices at once, in_batch and out_batch elements apart.
 * coefficients: host memory, a, b, c of each step. For out_type BF16 the numbers that are multiplied are rounded to 11 bits (of X X' only
 * what lies beside its diagonal; X itself is kept in 22), which shows in the result as less than its own rounding; for F32 and F16 they have 22 bits, or are exact to 2^-38
 * where 1 is X's norm (a G far below eps has little left).
 * Norms and sums are 32 bits or more. A matrix of zeros gives zeros; one with a NaN or an infinity gives NaN.
 * 0 <= count <= 4096, 1 <= rows, cols <= 65536, the shorter side at most 16384, count * rows * cols (each rounded up to 64) <= 2^32,
 * 1 <= steps <= 16, eps above 0. Polynomials that let singular values from 0..1 grow past 64 are refused. out may be in (same type and strides). As many matrices go together as have 2^26
 * elements, one at least: the workspace is about 1 GB at most, but for a matrix that wants more by itself.
 *
 * iodf_muon_step: the step of an optimiser around that, for `count` weights of one shape, each a tensor of its own (arrays of pointers, host memory):
 *   M <- beta M + G,  D = G + beta M (nesterov) or M,  W <- (1 - rate * decay) W - rate * scale * orthogonalise(D)
 * M F32 with consecutive rows; W and G strided, of their types. Products are as for out_type = weight_type. 0 <= count <= 64, whatever their
 * size together. Tensors of one call do not overlap.
 */
enum { IODF_ORTH_MOST = 16, IODF_MUON_MOST = 64 };
typedef struct iodf_orth {
    int64_t count, in_batch, out_batch, in_stride, out_stride;
    int32_t rows, cols, in_type, out_type, steps;
    float eps;
    const float* coefficients;
    const void* in;
    void* out;
} iodf_orth;
int iodf_orthogonalise(const iodf_orth* args, void* work, int64_t work_bytes, void* stream);
int iodf_orthogonalise_workspace(const iodf_orth* args, int64_t* bytes);

typedef struct iodf_muon {
    int64_t count, weight_stride, grad_stride;
    int32_t rows, cols, weight_type, grad_type, steps, nesterov;
    float eps, rate, beta, decay, scale, reserved;
    const float* coefficients;
    void* const* weights;
    const void* const* grads;
    float* const* momenta;
} iodf_muon;
int iodf_muon_step(const iodf_muon* args, void* work, int64_t work_bytes, void* stream);
int iodf_muon_workspace(const iodf_muon* args, int64_t* bytes);

/* Read one IODF_Q_* quantity into *out (host). */
int iodf_query(iodf_ctx* ctx, int what, int64_t* out);

/* Release the context and its device memory. NULL is ignored. */
void iodf_free(iodf_ctx* ctx);

/* Static, NUL-terminated description of an IODF_E_* code. */
const char* iodf_strerror(int code);

/* The hipError_t value behind the most recent IODF_E_HIP on this thread (0 if none). */
int iodf_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif
