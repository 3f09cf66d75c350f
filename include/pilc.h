/*
 * pilc.h -- C ABI of libpilc: the entropy-coding stage of PILC (arXiv 2206.05279)
 * for AMD MI355X (gfx950).
 *
 * The stage turns uint8 subpixels plus per-subpixel distribution parameters into a
 * bitstream and back (Sec. 3.1 "Compress"/"Decompress": the coder receives the symbols
 * and the predicted logistic parameters; the decoder regenerates the same parameters and
 * recovers the symbols losslessly).
 *
 * Conventions for every entry point
 *   - All `*_dev` pointers and the pointers inside pilc_params are DEVICE memory owned by
 *     the caller; pilc_geom, pilc_params and `*_host` pointers are HOST memory.
 *   - The library never allocates or frees device memory on behalf of a call: images,
 *     parameters, workspace and output are caller-owned.  (Four small constant tables
 *     live in the library's own device globals and are filled on first use per device.)
 *   - Work is enqueued on `hip_stream` (a hipStream_t passed as void*, NULL = default
 *     stream).  Every call synchronises that stream before it returns, so the status and
 *     all outputs are final on return; the calls under "Fitting the laws" below do not, they
 *     return once their kernels are enqueued.
 *   - Return value: 0 on success, a negative PILC_E_* code otherwise.  No exceptions.  Calls on
 *     different streams may run concurrently, from any threads, if they use different workspaces.
 *     The library's only process-wide state: the constant tables (filled once per device under a
 *     lock), the knobs pilc_set_timing, pilc_set_kernel_policy, pilc_set_one_pass_wait and
 *     pilc_set_ansai_decode_waves (atomic integers, read once at the start of a call), the scratch array of pilc_encode_static, four
 *     sets of words (8 MB each, on every GPU) that calls of pilc_twar_inverse on tall images pass rows on
 *     through, one a call, and a few KB of pinned host memory in which calls that encode or decode, and
 *     pilc_twar_inverse on tall images, report their outcome (64 places, one a call; allocated by the first such
 *     call and kept).
 *   - Tensors are dense, row-major, channel-interleaved: index ((i*h + y)*w + x)*3 + c.
 */
#ifndef PILC_H
#define PILC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PILC_VERSION 1u

enum {
    PILC_OK = 0,
    PILC_E_ARG = -1,       /* null / misaligned pointer, bad geometry                      */
    PILC_E_WORKSPACE = -2, /* workspace smaller than pilc_workspace_size reports            */
    PILC_E_CAPACITY = -3,  /* coded output does not fit coded_capacity (nothing usable out) */
    PILC_E_TOO_LARGE = -4, /* payload would reach 4 GiB (32-bit lane offsets)               */
    PILC_E_FORMAT = -5,    /* decode: bad magic / version / geometry mismatch / size        */
    PILC_E_CORRUPT = -6,   /* decode: offsets not monotone or out of bounds, a lane runs
                              past its end, or does not return to its initial state         */
    PILC_E_HIP = -7,       /* HIP runtime failure (see pilc_last_hip_error)                 */
    PILC_E_TIMEOUT = -8    /* a bounded wait between workgroups or wavefronts ran out (see
                              pilc_set_one_pass_wait); outputs undefined                    */
};

/* Geometry of a batch.  M = prec_bits is the constant of Sec. 3.2 for which every
 * symbol's integer masses sum to 2^M (the paper uses 10..15 for 8-bit data; 16 is also
 * accepted here).  A "lane" is one independent rANS stream:
 *   lane_mode 0: lane j codes the flat pixel range [j*lane_a, min((j+1)*lane_a, n*h*w));
 *                lane_a must divide h*w or be a multiple of it.
 *   lane_mode 1: lane j codes one tile of lane_a rows x lane_b columns; tiles are numbered
 *                row-major inside an image, images in order; edge tiles are clipped.
 * Inside a lane the decode order is raster order of its pixels, R,G,B inside a pixel. */
typedef struct {
    uint32_t n, h, w;   /* images, rows, columns; 3 interleaved channels */
    uint32_t prec_bits; /* M, 10..16 */
    uint32_t lane_mode; /* 0 or 1 */
    uint32_t lane_a, lane_b;
} pilc_geom;

/* Per-subpixel logistic parameters (Sec. 3.1 eq. (7), Sec. 3.3) in fixed point, plus the
 * per-image coefficients that condition G on R and B on R,G of the same pixel (Sec. 3.1
 * eqs. (3)-(4), applied as  mu'_G = mu_G + a_GR*(x_R-mu_R),
 * mu'_B = mu_B + a_BR*(x_R-mu_R) + a_BG*(x_G-mu_G), each product rounded to Q8.8). */
typedef struct {
    const uint16_t *mu;        /* device [n,h,w,3]  Q8.8 unsigned                          */
    const int16_t *log_scale;  /* device [n,h,w,3]  Q4.12, natural log of the scale;
                                  values outside [-4, 6) act as the nearest bound         */
    const int16_t *chan_coef;  /* device [n,3]      Q2.14: a_GR, a_BR, a_BG                */
} pilc_params;

/* Number of lanes of a geometry (Sec. 3.2's independent coder instances, "one thread per
 * piece" in Sec. 4.3); 0 if the geometry is invalid. */
uint64_t pilc_lane_count(const pilc_geom *geom);

/* Sizes a caller must provide: bytes of device workspace for encode and decode of this
 * geometry, and an upper bound of the container size (64-byte header + 4*(lanes+1) offset
 * table + per lane 4 bytes of state + at most one 16-bit word per symbol).
 * Errors: PILC_E_ARG. */
int pilc_workspace_size(const pilc_geom *geom, size_t *workspace_bytes_host,
                        size_t *max_coded_bytes_host);

/* Compress (Sec. 3.1 "Compress", coder part; Sec. 3.2 tables; App. A eq. (11) per symbol).
 *   img_dev        uint8 [n,h,w,3]
 *   params         see pilc_params
 *   workspace_dev  >= workspace_bytes from pilc_workspace_size, 256-byte aligned; contents
 *                  are scratch, undefined afterwards
 *   coded_dev      output container, 16-byte aligned, capacity coded_capacity bytes
 *   coded_bytes_host  receives the container size
 * Container (little endian): 64-byte header {"PILC", version, n, h, w, 3, M, lane_mode,
 * lane_a, lane_b, lanes, 0, payload_bytes u64, 0 u64}; u32 offsets[lanes+1] (exclusive
 * prefix sum of lane byte counts, relative to the payload); payload = for each lane its
 * final 32-bit state followed by its 16-bit words in the order the decoder reads them.
 * Errors: PILC_E_ARG, PILC_E_WORKSPACE, PILC_E_CAPACITY (coded_dev contents undefined),
 * PILC_E_TOO_LARGE, PILC_E_HIP, PILC_E_TIMEOUT. */
int pilc_encode(const pilc_geom *geom, const uint8_t *img_dev, const pilc_params *params,
                void *workspace_dev, size_t workspace_bytes, uint8_t *coded_dev,
                size_t coded_capacity, uint64_t *coded_bytes_host, void *hip_stream);

/* pilc_encode for callers that cannot allocate device memory or carry a workspace: code under
 * HIP graph capture set-up, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, container, alignment rules and errors as pilc_encode, without the workspace: the
 * scratch memory is an array of PILC_STATIC_SCRATCH_BYTES inside the library (one copy per GPU,
 * held until the process ends), and the call allocates and frees nothing (no HIP events either:
 * pilc_last_timing reports nothing for it).  A geometry whose pilc_workspace_size exceeds
 * PILC_STATIC_SCRATCH_BYTES is refused with PILC_E_WORKSPACE before anything runs (16 MiB holds
 * one 1920x1080 frame, or about 2.7 million pixels in all).  All calls on one GPU share that
 * GPU's array: calls that overlap in time on the same GPU, from any threads or streams, race and
 * give undefined output; calls one after another are independent (nothing is kept between them). */
#define PILC_STATIC_SCRATCH_BYTES (16u << 20)
int pilc_encode_static(const pilc_geom *geom, const uint8_t *img_dev, const pilc_params *params,
                       uint8_t *coded_dev, size_t coded_capacity, uint64_t *coded_bytes_host,
                       void *hip_stream);

/* Decompress (Sec. 3.1 "Decompress", coder part; App. A eq. (12) per symbol, the symbol
 * being the x with C_x <= S mod 2^M < C_x + P_x).  The geometry and parameters must be the
 * ones used to encode.  img_out_dev uint8 [n,h,w,3]; on error its contents are undefined.
 * coded_dev is 16-byte aligned; the decoder reads the stream in aligned 16-byte blocks and may
 * therefore read (never use) up to 15 bytes beyond coded_bytes, inside the block that holds the
 * container's last byte.
 * Errors: PILC_E_ARG, PILC_E_WORKSPACE, PILC_E_FORMAT, PILC_E_CORRUPT, PILC_E_HIP. */
int pilc_decode(const pilc_geom *geom, const uint8_t *coded_dev, size_t coded_bytes,
                const pilc_params *params, void *workspace_dev, size_t workspace_bytes,
                uint8_t *img_out_dev, void *hip_stream);

/* The integer tables of Sec. 3.2 for the symbols actually present: for every subpixel (image
 * layout [n,h,w,3]) its cumulative count C_x and mass P_x (sum_x P_x = 2^M, P_x >= 1).
 * cum_out_dev, freq_out_dev: device uint32 [n,h,w,3].  A verification entry point: encode
 * computes the same values on the fly and never materialises them.
 * Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_symbol_tables(const pilc_geom *geom, const uint8_t *img_dev, const pilc_params *params,
                       uint32_t *cum_out_dev, uint32_t *freq_out_dev, void *hip_stream);

/* ---- mixture of K logistic laws per subpixel ------------------------------------------
 * The workload Sec. 2 ("Entropy Coder") and the "Data transfer" item of Sec. 1 name as the
 * slow case of earlier learned codecs: a dynamic rANS coder (App. A eqs. (11)-(12)) whose
 * distribution per symbol is a mixture of ten logistic laws.  The paper gives no formula; this
 * library takes: a pixel carries K weights w_j in Q0.15 that sum to 2^15 exactly (shared by its
 * three subpixels), a subpixel K means and K log-scales (formats of pilc_params); the mixed
 * 24-bit edge CDF is F(k) = floor(sum_j w_j F_j(k) / 2^15), F_j the single-law edge CDF, and
 * C(k) = k + floor(F(k) (2^M - 256) / 2^24), so K = 1 is the single law of pilc_encode; G and B
 * are conditioned as in pilc_params, every component's mean shifted with that component's own
 * innovations. */
typedef struct {
    const uint16_t *mu;        /* device [n,h,w,3,K] Q8.8                                  */
    const int16_t *log_scale;  /* device [n,h,w,3,K] Q4.12                                 */
    const uint16_t *weight;    /* device [n,h,w,K]   Q0.15, sum over K = 32768 per pixel   */
    const int16_t *chan_coef;  /* device [n,3]       Q2.14: a_GR, a_BR, a_BG               */
    uint32_t num_comp;         /* K, 1..16                                                 */
} pilc_mix_params;

/* As pilc_encode / pilc_decode (same geometry, workspace size from pilc_workspace_size,
 * alignment, ownership and container), with the magic "PMIX" and K in header word 11 (bytes
 * 44..47).  Runs one thread per lane whatever the number of lanes.
 * Errors: those of pilc_encode / pilc_decode; PILC_E_ARG also for K outside 1..16 and, found on
 * the device, for a pixel whose weights do not sum to 32768 (outputs then undefined). */
int pilc_mix_encode(const pilc_geom *geom, const uint8_t *img_dev, const pilc_mix_params *params,
                    void *workspace_dev, size_t workspace_bytes, uint8_t *coded_dev,
                    size_t coded_capacity, uint64_t *coded_bytes_host, void *hip_stream);
int pilc_mix_decode(const pilc_geom *geom, const uint8_t *coded_dev, size_t coded_bytes,
                    const pilc_mix_params *params, void *workspace_dev, size_t workspace_bytes,
                    uint8_t *img_out_dev, void *hip_stream);

/* Per-kernel timing, off by default.  When enabled, pilc_encode / pilc_decode bracket each
 * kernel with HIP events on the stream the kernel is launched on.  pilc_last_timing returns
 * the durations in milliseconds of the most recent call on the calling thread: index 0 is
 * the whole GPU part of the call, 1.. are its kernels in launch order (pilc_timing_name
 * gives the kernel's function name; "scan" covers the kernels of the scan, which a
 * batch of few lanes has not: up to 8192, fewer where they are long; "k_twar_inverse" the launches
 * of the residual's inverse).  Returns the number of entries written (<= capacity), 0 if timing was off. */
void pilc_set_timing(int enabled);
int pilc_last_timing(float *ms_out_host, int capacity);
const char *pilc_timing_name(int index_in_last_call);

/* Which lane kernels encode and decode use: 0 = chosen from the lane count (default), 1 = one
 * thread per lane, 2 = the kernels for few long lanes (workgroup-cooperative encode, a row of 16
 * threads per lane in decode), 3 = one thread per lane with the one-pass encoder (the lane kernel
 * also computes the offsets and places its lanes in the container, instead of leaving that to the
 * scan and pack kernels; measured no faster, kept for comparison).  pilc_mix_decode goes a thread per
 * lane under 1 and 3 and a row per lane under 2; pilc_mix_encode does not look at it.  Lanes of 2^25 symbols and more
 * are encoded by the kernels for few long lanes whatever is set (their words are out of the other
 * encoder's reach), so that under 3 the bounded wait below has nothing to bound in the encoder.
 * All choices produce the same
 * bytes; the knob exists for tuning and for testing every kernel on the same input.  Process-wide.
 * Errors: PILC_E_ARG for any other value. */
int pilc_set_kernel_policy(int policy);

/* The one-pass encoder's (policy 3) workgroups learn where their lanes go from the workgroups
 * before them (the scan of Sec. 4.1's container offsets, fused into the lane kernel); a workgroup
 * waits for an earlier one at most `ticks` ticks of the GPU's constant-rate clock (0 = the
 * default, two seconds) and then gives up: the call returns PILC_E_TIMEOUT and every kernel still
 * ends.
 * `withhold_first` != 0 makes the first workgroup publish nothing, which forces that path: for
 * tests of the give-up path only.  The same bound and switch apply to the bands of
 * pilc_twar_inverse and to pilc_decode with few lanes, where every decoding wavefront waits for
 * a second one that prepares its next batch (the switch: nothing is ever said to be ready).
 * Process-wide. */
void pilc_set_one_pass_wait(uint64_t ticks, int withhold_first);

/* ------------------------------------------------------------------------------------------
 * The paper's own coder variant: ANS-AI (Sec. 3.2, Alg. 3 "Encode x", Alg. 4 "Decode one
 * symbol"), the table-driven form of the modified rANS of Alg. 1 / Alg. 2.  The state lives in
 * [2^M, 2^(M+1)); every symbol carries the index d of one of D fixed distributions over X
 * symbols; encode looks up delta[d,x], phi[d,x], decode looks up Theta[d,S], B[d,S], N[d,S].
 * A "piece" is one independent coder instance of `count` symbols (Sec. 4.3: one thread per
 * piece).  Readings the paper leaves open: a piece is encoded last symbol first so that decode
 * returns the symbols in order; the state starts at 2^M and decode must return there with the
 * stream used up; a pushed group of bits keeps its order, bit 0 of S first.
 * Container (little endian): 64-byte header {"PANS", 1, pieces, count, M, D, X, 0.., payload
 * bytes u64 at byte 48, 0}; u32 offsets[pieces+1] (bytes, relative to the payload); per piece
 * {final state u32, bit count u32, ceil(bits/32) words of 32 bits, bit i of the stream at bit
 * i%32 of word i/32}.
 * ------------------------------------------------------------------------------------------ */
typedef struct {
    uint32_t pieces, count; /* independent pieces, symbols per piece; rounded-up pieces*count < 2^32 */
    uint32_t prec_bits;     /* M, 1..15, 2^M >= num_sym */
    uint32_t num_dist;      /* D, 1..255 */
    uint32_t num_sym;       /* X, 2..256 */
} pilc_ansai_shape;

/* Bytes of device memory pilc_ansai_build_tables fills for these M, D, X (0 if invalid):
 * 8*(D*256+1) for delta and phi plus 3*D*2^M (5*D*2^M when M > 12) for Theta, B, N, plus padding. */
size_t pilc_ansai_table_bytes(uint32_t prec_bits, uint32_t num_dist, uint32_t num_sym);

/* Builds the tables of Sec. 3.2 on the device from integer masses.
 *   mass_dev    device uint32 [D, X], every P_x >= 1, each row summing to 2^M
 *   tables_dev  device, 256-byte aligned, tables_bytes >= pilc_ansai_table_bytes(); opaque to
 *               the caller, valid for any number of encode / decode calls with the same M, D, X
 * Errors: PILC_E_ARG (bad sizes or pointers, or masses that break the two conditions above:
 * the blob is then marked unusable), PILC_E_WORKSPACE (tables_bytes too small), PILC_E_HIP. */
int pilc_ansai_build_tables(uint32_t prec_bits, uint32_t num_dist, uint32_t num_sym,
                            const uint32_t *mass_dev, void *tables_dev, size_t tables_bytes,
                            void *hip_stream);

/* Re-centring of Sec. 3.3: the residual r ~ L(mu, s, 0, 255) is coded as (r - mu + 128) mod 256
 * ~ L(128, s, 0, 255), so that the distribution index only has to tell the scale.  mu is the
 * predicted location rounded to an integer.  inverse = 0: out = (in - mu + 128) mod 256 (before
 * pilc_ansai_encode); inverse != 0: out = (in + mu - 128) mod 256 (after pilc_ansai_decode).
 * in_dev, mu_dev, out_dev: device uint8 [count], 16-byte aligned; out_dev may be in_dev.
 * Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_ansai_center(const uint8_t *in_dev, const uint8_t *mu_dev, uint64_t count, int inverse,
                      uint8_t *out_dev, void *hip_stream);

/* Device workspace needed by pilc_ansai_encode / pilc_ansai_decode and an upper bound of the
 * container size (header + offsets + per piece 8 bytes and ceil(count*M/32) words).
 * Errors: PILC_E_ARG, PILC_E_TOO_LARGE. */
int pilc_ansai_workspace_size(const pilc_ansai_shape *shape, size_t *workspace_bytes_host,
                              size_t *max_coded_bytes_host);

/* Alg. 3 over a batch.  sym_dev, dist_dev: device uint8 [pieces, count], 16-byte aligned;
 * workspace_dev 256-byte aligned scratch; coded_dev 16-byte aligned output.
 * Errors: PILC_E_ARG (also: a symbol >= X or an index >= D in the data, or tables built for
 * other M, D, X), PILC_E_WORKSPACE, PILC_E_CAPACITY, PILC_E_TOO_LARGE, PILC_E_HIP; on error
 * the contents of coded_dev are undefined. */
int pilc_ansai_encode(const pilc_ansai_shape *shape, const uint8_t *sym_dev, const uint8_t *dist_dev,
                      const void *tables_dev, void *workspace_dev, size_t workspace_bytes,
                      uint8_t *coded_dev, size_t coded_capacity, uint64_t *coded_bytes_host,
                      void *hip_stream);

/* Alg. 4 over a batch; dist_dev must hold the indices used to encode.  sym_out_dev: device
 * uint8 [pieces, count], 16-byte aligned; on error its contents are undefined.
 * Errors: PILC_E_ARG (as above), PILC_E_WORKSPACE, PILC_E_FORMAT (header does not match the
 * shape or coded_bytes), PILC_E_CORRUPT (bad offsets or record, a piece that runs out of bits,
 * keeps some, or does not return to the initial state), PILC_E_HIP. */
int pilc_ansai_decode(const pilc_ansai_shape *shape, const uint8_t *coded_dev, size_t coded_bytes,
                      const uint8_t *dist_dev, const void *tables_dev, void *workspace_dev,
                      size_t workspace_bytes, uint8_t *sym_out_dev, void *hip_stream);

/* How many wavefronts a workgroup of pilc_ansai_decode's kernel has: 0 = chosen from the batch and
 * the table size (default: as many as fit beside the tables in LDS, fewer for a batch that would
 * not fill every compute unit that densely), 1 .. 12 = that many (less if fewer fit).  Every
 * choice decodes the same symbols; the knob exists for tuning and for testing every workgroup
 * shape on the same input.  Process-wide.  Errors: PILC_E_ARG for any other value. */
int pilc_set_ansai_decode_waves(int waves);

/* ------------------------------------------------------------------------------------------
 * The Three-Way Auto-regressive residual transform (Sec. 3.1, eqs. (2)-(4)): every subpixel is
 * predicted from three known values -- R(u,v) from R(u-1,v-1), R(u-1,v), R(u,v-1); G(u,v) from
 * G(u,v-1), R(u,v-1), R(u,v); B(u,v) from B(u,v-1), G(u,v-1), G(u,v); u the row, v the column --
 * with three weights and a bias per channel (12 parameters), and the residual goes to the coder.
 * Readings the paper leaves open: zero padding above and to the left; fixed-point weights,
 * x^ = clamp((w . ctx + bias + 2^13) >> 14, 0, 255) with an arithmetic shift; residual
 * r = (x - x^) mod 256, so that x = (r + x^) mod 256.
 * Images: device uint8 [n, h, w, 3], channel-interleaved; input and output must not overlap.
 * ------------------------------------------------------------------------------------------ */
typedef struct {
    int16_t w[3][3]; /* [channel][context value in the order above], Q2.14 */
    int32_t bias[3]; /* Q8.14, |bias| <= 2^30 */
} pilc_twar_params;

/* res = image minus prediction.  Errors: PILC_E_ARG, PILC_E_TOO_LARGE, PILC_E_HIP. */
int pilc_twar_forward(uint32_t n, uint32_t h, uint32_t w, const uint8_t *img_dev,
                      const pilc_twar_params *params_host, uint8_t *res_dev, void *hip_stream);

/* The image back from the residual (Sec. 3.1: the anti-diagonal / column schedule of the paper's
 * decoding figure, here one walk along the anti-diagonals of 64 rows at a time).  Images of more than
 * 64 rows, unless there are so many that they fill the GPU with one such band each, are decoded in bands
 * of 64 rows that follow each other through words in the library's device globals (32 MB on every GPU,
 * there from the time the library is loaded); their wait for the band above is bounded
 * like the one-pass encoder's (pilc_set_one_pass_wait) and ends in PILC_E_TIMEOUT.
 * Errors: PILC_E_ARG, PILC_E_TOO_LARGE, PILC_E_HIP, PILC_E_TIMEOUT (img_dev contents undefined). */
int pilc_twar_inverse(uint32_t n, uint32_t h, uint32_t w, const uint8_t *res_dev,
                      const pilc_twar_params *params_host, uint8_t *img_dev, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * Fitting the laws.  The coder takes the laws of its symbols as given; what follows is for the
 * program that learns them: what symbols cost under a model's logits and what else they might
 * have been, the gradient of that cost, the norm before the layer that makes the logits, and the
 * step that moves the weights.
 *
 * These entry points differ from the coder's in two ways.  They only ENQUEUE their kernels on
 * `hip_stream` and return: nothing that happens on the device decides their status, and outputs
 * are final when the stream gets there, as with a kernel of the caller's own (they may be
 * captured into a graph).  And tensors need no more alignment than their elements have, except
 * the workspace (256 bytes); what is aligned to 16 bytes, rows included, is read faster.
 * pilc_last_timing reports nothing for them.  Inputs and outputs must not overlap unless a
 * comment says that they may.  Sums, statistics and states are held in 32 bits; a value is
 * rounded to its tensor's type once, to the nearest, ties to even.
 * ------------------------------------------------------------------------------------------ */
enum { PILC_F32 = 0, PILC_BF16 = 1, PILC_F16 = 2 }; /* types of values */
enum { PILC_U8 = 0, PILC_I32 = 1, PILC_I64 = 2 };   /* types of symbols */

/* rows x num_sym logits, row r at r * stride elements; what lies between rows is never used. */
typedef struct {
    uint32_t rows;        /* 0: the calls do nothing                                        */
    uint32_t num_sym;     /* 1 .. 2^31 - 1                                                  */
    uint64_t stride;      /* >= num_sym, in elements                                        */
    uint32_t dtype;       /* PILC_F32, PILC_BF16, PILC_F16                                  */
    uint32_t target_type; /* PILC_U8, PILC_I32, PILC_I64                                    */
    uint32_t top;         /* alternatives a row, 0 .. 32                                    */
} pilc_logits_shape;

/* Device workspace of pilc_logprobs and pilc_logprobs_train for this shape (at least 256).
 * Errors: PILC_E_ARG. */
int pilc_logprobs_workspace_size(const pilc_logits_shape *shape, size_t *workspace_bytes_host);

/* What symbols cost under the law that a row of logits x stands for, p_j = exp(x_j - lse),
 * lse = ln sum_j exp(x_j).  Per row, in nats (a symbol's length in a container is about
 * -logp / ln 2 bits):
 *   logp_dev       f32 [rows]  x_t - lse of the target t; NULL: not wanted
 *   entropy_dev    f32 [rows]  -sum_j p_j ln p_j; NULL: not wanted
 *   lse_dev        f32 [rows]  NULL: not wanted
 *   top_sym_dev    int32 [rows, top], top_logp_dev f32 [rows, top]: the `top` most likely symbols,
 *                  most likely first, the lower symbol first among equals, and ln p of each;
 *                  symbol -1 and -inf where fewer symbols have a probability above 0
 *   target_dev     [rows]; NULL if logp_dev is NULL.  A negative target does not count: its logp
 *                  is 0.  A target >= num_sym: NaN
 * Logits of -inf are symbols that cannot occur.  A row that has no others has no law: lse and
 * logp are -inf, the entropy 0, there are no alternatives.  A row with a NaN or +inf among its
 * logits: lse, entropy, logp and top_logp are NaN, top_sym -1.
 * Errors: PILC_E_ARG, PILC_E_WORKSPACE, PILC_E_HIP. */
int pilc_logprobs(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev,
                  float *logp_dev, float *entropy_dev, float *lse_dev, int32_t *top_sym_dev,
                  float *top_logp_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* The gradient of sum_r up_logp[r] logp[r] + up_entropy[r] entropy[r] by the logits:
 *   grad_j = a (1[j = t] - p_j) - b p_j (ln p_j + entropy),  a = up_logp[r] (0 where the target does
 * not count), b = up_entropy[r].
 *   lse_dev, entropy_dev   f32 [rows], from pilc_logprobs.  p is what this lse, in its 32 bits, says:
 *                          a |lse| 2^-24th of it is lost, which logits that lie far from zero show;
 *                          pilc_logprobs_train loses nothing to it
 *   up_logp_dev            f32 [rows]
 *   up_entropy_dev         f32 [rows]; NULL: no such term, entropy_dev is then not read
 *   grad_dev               [rows, num_sym] of the logits' type, row r at r * grad_stride; may be the
 *                          logits themselves (same address and stride)
 * A row whose a and b are both 0 gets zeros whatever its logits are, and so does a row without a
 * law; a row with a NaN, a +inf or a target >= num_sym (a or b not 0) gets NaN throughout.
 * `top` is not looked at.  Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_logprobs_grad(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev,
                       const float *lse_dev, const float *entropy_dev, const float *up_logp_dev,
                       const float *up_entropy_dev, void *grad_dev, uint64_t grad_stride,
                       void *hip_stream);

/* Both in one call, for a loss whose weights are known beforehand: the logp, entropy and lse of
 * pilc_logprobs (entropy_dev, lse_dev NULL: not wanted) and the gradient of pilc_logprobs_grad.
 * `top` has to be 0.  Errors: PILC_E_ARG, PILC_E_WORKSPACE, PILC_E_HIP. */
int pilc_logprobs_train(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev,
                        const float *up_logp_dev, const float *up_entropy_dev, float *logp_dev,
                        float *entropy_dev, float *lse_dev, void *grad_dev, uint64_t grad_stride,
                        void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* rows x width values; strides between rows in elements, >= width. */
typedef struct {
    uint32_t rows;        /* 0: forward does nothing, backward's weight gradients are 0     */
    uint32_t width;       /* 1 .. 2^31 - 1                                                  */
    uint64_t x_stride;    /* of x                                                           */
    uint64_t y_stride;    /* of y, in the backward pass of dy                               */
    uint64_t dx_stride;   /* of dx; not looked at by the forward pass                       */
    uint32_t dtype;       /* of x, y, dy, dx: PILC_F32, PILC_BF16, PILC_F16                 */
    uint32_t weight_type; /* of weight, bias and their gradients: dtype or PILC_F32         */
    float eps;            /* >= 0                                                           */
} pilc_norm_shape;

/* y = (x - mean) rstd weight + bias, rstd = 1 / sqrt(mean of (x - mean)^2 + eps), over each row.
 * weight_dev, bias_dev [width], NULL: 1 and 0.  mean_dev, rstd_dev f32 [rows], NULL: not wanted.
 * y_dev may be x_dev (same stride).  Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_norm_forward(const pilc_norm_shape *shape, const void *x_dev, const void *weight_dev,
                      const void *bias_dev, void *y_dev, float *mean_dev, float *rstd_dev,
                      void *hip_stream);

/* Device workspace of pilc_norm_backward (at least 256).  Errors: PILC_E_ARG. */
int pilc_norm_workspace_size(const pilc_norm_shape *shape, size_t *workspace_bytes_host);

/* With xh = (x - mean) rstd and q = dy weight:
 *   dx = rstd (q - mean of q - xh mean of (q xh)) over each row, dweight = sum over rows of dy xh,
 *   dbias = sum over rows of dy.
 * mean_dev, rstd_dev f32 [rows] from the forward pass; weight_dev NULL: 1.  dx_dev, dweight_dev,
 * dbias_dev: NULL: not wanted, one at least is.  dx_dev may be dy_dev (dx_stride = y_stride).  The
 * sums over rows are taken in an order that the shape and the GPU's number of compute units fix.
 * Errors: PILC_E_ARG, PILC_E_WORKSPACE, PILC_E_HIP. */
int pilc_norm_backward(const pilc_norm_shape *shape, const void *dy_dev, const void *x_dev,
                       const void *weight_dev, const float *mean_dev, const float *rstd_dev,
                       void *dx_dev, void *dweight_dev, void *dbias_dev, void *workspace_dev,
                       size_t workspace_bytes, void *hip_stream);

/* One tensor of an AdamW step: `count` values, dense. */
typedef struct {
    void *param;       /* device, param_type; updated                                       */
    const void *grad;  /* device, grad_type                                                 */
    void *m, *v;       /* device, f32, or uint8 codes with state_bits 8; updated            */
    uint8_t *m_scale;  /* device, a byte for each 256 values (the last ones maybe fewer);   */
    uint8_t *v_scale;  /*   state_bits 8 only                                               */
    uint64_t count;    /* 0: left out                                                       */
    float lr_mult;     /* lr of this tensor = lr * lr_mult                                  */
    float decay;       /* weight decay                                                      */
} pilc_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps; /* 0 <= beta < 1, eps >= 0 (above 0 it counts as 2^-126 at least) */
    double grad_scale;            /* the gradients are multiplied by it                     */
    uint64_t step;                /* of this step, from 1                                   */
    uint32_t param_type, grad_type;
    uint32_t state_bits;          /* 32 or 8                                                */
    uint32_t dither;              /* state_bits 8: another number every step, say its own   */
} pilc_adamw_params;

/* One step over `num_tensors` tensors (tensors_host is read before the call returns):
 *   g = grad grad_scale;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   param = param (1 - lr decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * with the new m and v as they are before they are put into 8 bits.  PILC_E_ARG for numbers that 32 bits
 * do not hold: eps, grad_scale, lr lr_mult / (1 - beta1^step), 1 - lr lr_mult decay.
 *
 * State in 8 bits: 256 values in a row share a scale 2^(e-126), e the exponent field of the
 * largest of them (at least 1), held as a byte; e = 255 says that the block is not finite, its
 * values are NaN.  A value is coded as a short floating number of its distance from zero plus a
 * constant, y = |value| / scale + 2^-k (k = 15 for m, 31 for v), three bits behind the leading one:
 *   code = ((bits(y) + r) >> 20) - ((127 - k) << 3),  value = sign (y(code) - 2^-k) scale
 * m has its sign in bit 7, v none.  Even steps near zero (2^-18 of the scale for m, 2^-34 for v),
 * an eighth of the value above.  r = 16 n + 8, n being 16 bits of a hash of the value's number in
 * the list and `dither` (low half m, high half v), so that rounding up or down is as likely as it
 * is near: an average that moves by less than a step at a time, as beta2 makes them, still moves.
 * A v above 0 never gets code 0: a denominator does not vanish under an m that does not.
 * A value's number is 256 times the whole or begun blocks of the tensors before its own, plus its
 * place in it; hash, with 32-bit wrap-around: h = low * 0x9E3779B9 + high * 0x6A09E667 + dither *
 * 0xBB67AE85; h ^= h >> 16; h *= 0x3C6EF373; h ^= h >> 15; h *= 0xA54FF53B; h ^= h >> 16.
 * States start as zero bytes.
 * Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_adamw_step(const pilc_adamw_params *params_host, const pilc_adamw_tensor *tensors_host,
                    uint32_t num_tensors, void *hip_stream);

/* The values that `count` codes stand for, in 32 bits (for a checkpoint, or to look at them).
 * is_signed: 1 for m, 0 for v.  Errors: PILC_E_ARG, PILC_E_HIP. */
int pilc_adamw_values(const uint8_t *code_dev, const uint8_t *scale_dev, uint64_t count, int is_signed,
                      float *values_dev, void *hip_stream);

const char *pilc_strerror(int code);
const char *pilc_last_hip_error(void); /* text of the last HIP failure on this thread */
uint32_t pilc_version(void);

#ifdef __cplusplus
}
#endif
#endif
