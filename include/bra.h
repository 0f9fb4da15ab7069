/*
 * bra.h - C boundary of the B200 (sm_100a) Bi-Level Routing Attention library.
 *
 * The library computes the hot path of BRA (BiFormer, arXiv 2303.08810,
 * Section 3.2, Algorithm 1) starting from already-projected Q, K, V:
 *   1. region mean pooling of Q and K            (Section 3.2, "per-region average")
 *   2. region affinity A^r = Q^r (K^r)^T         (Eq. 4)
 *   3. row-wise top-k routing index I^r          (Eq. 5)
 *   4. token-to-token softmax attention over the keys/values of the k routed
 *      regions, K^g / V^g never written to memory (Eq. 6, Eq. 7 with Eq. 1)
 *   5. + LCE(V), a 5x5 depthwise convolution of V (Eq. 7)
 * and the gradients of step 4-5 for a fixed routing index.
 *
 * Common rules for every entry point
 *   - All tensor pointers are DEVICE pointers owned by the caller, 16-byte
 *     aligned, dense and contiguous.  The library allocates no device memory
 *     and keeps no state between calls besides kernel attributes and launch
 *     choices remembered per device and problem shape, and one helper stream
 *     with two events per device and host thread (created by the first
 *     bra_backward call; its work is forked from and joined back into `stream`).
 *   - Q, K, V, O, dO, dQ, dK, dV: [B, H, W, C], element type p->dtype, channel
 *     c = head * (C / heads) + j (concat order of Eq. 2).
 *   - Regions: S x S non-overlapping blocks of (H/S) x (W/S) tokens, numbered
 *     row-major r = ry * S + rx (region partition, Section 3.2).  Where S does
 *     not divide H or W (Appendix C picks S as a divisor "to avoid padding"),
 *     the map counts as zero-padded at the bottom and the right to the next
 *     multiples of S: the zero tokens are pooled, routed to and attended to like
 *     real ones, and O, lse and the gradients are those of the H x W tokens.
 *     Most kernels work on the map as it is; those that want whole regions
 *     (BRA_IMPL_TC and BRA_IMPL_IMG) get padded copies, which live in ws
 *     (bra_workspace_bytes accounts for them) and cost one extra kernel per
 *     tensor.
 *   - index: int32 [B, heads, S*S, topk] (or [B, 1, S*S, topk] when
 *     p->shared_routing != 0).  Row i lists the key regions that the queries of
 *     region i attend to.  It is a list: any order, duplicates count twice.
 *   - ws: scratch of at least bra_workspace_bytes(p) bytes, 256-byte aligned.
 *     It holds a device status block (error words and, for the one-launch
 *     forward, barrier counters) that the kernels expect to find ZERO and
 *     leave zero: before its first use fill ws with zeros or call
 *     bra_workspace_init().  bra_device_status() restores that state when it
 *     reports an error.  Calls that share a ws must be ordered on one stream.
 *   - Every call is asynchronous on `stream` (a cudaStream_t passed as void*).
 *   - Errors a host check can find return synchronously, nothing launched,
 *     outputs untouched.  Errors only the device can see (an out-of-range
 *     entry in a caller's index) never trap: the offending work is skipped,
 *     a code is recorded in ws and bra_device_status() reports it.
 *   - Outputs must not alias inputs.
 */
#ifndef BRA_H_
#define BRA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum bra_status {
    BRA_OK = 0,
    BRA_ERR_NULL = 1,        /* a required pointer is NULL */
    BRA_ERR_SHAPE = 2,       /* B,H,W,C,heads,S <= 0; heads does not divide C */
    BRA_ERR_TOPK = 3,        /* topk < 1 or topk > S*S */
    BRA_ERR_DTYPE = 4,       /* dtype is not BRA_F32 / BRA_BF16 */
    BRA_ERR_ALIGN = 5,       /* a pointer is not 16-byte aligned (ws: 256) */
    BRA_ERR_WORKSPACE = 6,   /* ws_bytes < bra_workspace_bytes(p) */
    BRA_ERR_UNSUPPORTED = 7, /* valid problem this build has no kernel for (head dim, lce_ksize, impl) */
    BRA_ERR_CUDA = 8,        /* a CUDA runtime call failed (launch, attribute) */
    BRA_ERR_INDEX = 9,       /* device-detected: routing index entry outside [0, S*S) */
    BRA_ERR_TIMEOUT = 10,    /* device-detected: a bounded wait gave up */
    BRA_ERR_STATIC_LIMIT = 11 /* bra_route_static only: B*S*S*C > BRA_ROUTE_STATIC_MAX_MEAN_FLOATS */
} bra_status;

typedef enum bra_dtype { BRA_F32 = 0, BRA_BF16 = 1 } bra_dtype;

/* Which kernel family runs the token-to-token attention (step 4-5). */
typedef enum bra_impl {
    BRA_IMPL_AUTO = 0,  /* fastest kernel that supports the problem */
    BRA_IMPL_SIMT = 1,  /* fp32 CUDA-core kernels: any dtype, any map, region size, topk and batch; C/heads 16, 32, 64 or 128
                           (gradients: up to 64) */
    BRA_IMPL_MMA = 2,   /* bf16 warp-level tensor-core kernels with operands straight from global memory (C/heads == 32 or 64,
                           regions at most 128 tokens wide) */
    BRA_IMPL_TC = 3,    /* bf16 tcgen05/TMEM kernels (C/heads == 32; regions of 8 x 8 tokens, or 16 wide and a multiple of 8 high) */
    BRA_IMPL_IMG = 4,   /* bf16 warp-level tensor-core kernel with a whole (image, head) of K and V resident in
                           shared memory (C/heads == 32, H*W <= ~1500 tokens): small maps, small regions */
    BRA_IMPL_TC_FUSED = 5 /* as BRA_IMPL_TC, and bra_forward runs pooling, routing and attention as three phases of
                           ONE launch (8 x 8-token regions, topk = 1, per-head routing, <= 64 regions,
                           C <= 128): results equal to the chain of launches bit for bit */
} bra_impl;

/*
 * Failure injection for tests of the error path (no GPU fault, trap or hang is involved).
 * BRA_INJECT_LOSE_POOLED_UNIT: in the one-launch forward (bra_forward with BRA_IMPL_TC_FUSED) one pooled
 * unit is never counted as done, so every CTA's bounded wait for the end of the pooling phase runs out
 * after a few thousand polls, before any tensor-core work or tile copy has been issued;
 * the kernel returns normally, O is not written and bra_device_status() reports BRA_ERR_TIMEOUT.
 * Ignored by every other path.
 */
typedef enum bra_inject { BRA_INJECT_NONE = 0, BRA_INJECT_LOSE_POOLED_UNIT = 1 } bra_inject;

/* Problem statement in the notation of Algorithm 1 (H, W, C, S, k) plus batch and heads. */
typedef struct bra_problem {
    int32_t B, H, W, C;     /* batch, feature-map height and width, channels */
    int32_t heads;          /* attention heads; head dim d = C / heads (Eq. 2) */
    int32_t S;              /* regions per side: S x S regions */
    int32_t topk;           /* k of Eq. 5, 1 <= k <= S*S */
    int32_t dtype;          /* bra_dtype of Q, K, V, O and their gradients */
    float   scale;          /* softmax scale of Eq. 1; <= 0 selects 1/sqrt(C/heads) */
    int32_t shared_routing; /* 0: one index per head (affinity over the head's channels);
                               1: one index for all heads (Eq. 4 read over all C channels) */
    int32_t lce_ksize;      /* 5: add LCE(V) (Eq. 7); 0: attention term only */
    int32_t impl;           /* bra_impl */
    int32_t inject;         /* bra_inject: 0 in production */
} bra_problem;

/* Scratch size in bytes every call on problem p needs (0 if p is invalid). Host only. */
size_t bra_workspace_bytes(const bra_problem* p);

/*
 * Puts ws into the state the kernels expect: status block (error words, barrier counters) zero
 * (an asynchronous memset on `stream`; the rest of ws needs no initial value).  Needed once before the
 * first use of a ws that was not zero-filled.  (Housekeeping of this library: Algorithm 1 has no
 * counterpart.)
 */
bra_status bra_workspace_init(const bra_problem* p, void* ws, size_t ws_bytes, void* stream);

/*
 * Region-to-region routing (Section 3.2: per-region average; Eq. 4; Eq. 5).
 *   Q, K     in   [B,H,W,C]
 *   q_mean   out  fp32 [B, S*S, C], Q^r; may be NULL (kept in ws only)
 *   k_mean   out  fp32 [B, S*S, C], K^r; may be NULL
 *   index    out  int32 [B, heads|1, S*S, topk]; row order: affinity descending,
 *                 equal affinities by ascending region number
 * Means are accumulated and the affinity evaluated in fp32 whatever the dtype.
 */
bra_status bra_route(const bra_problem* p, const void* Q, const void* K,
                     float* q_mean, float* k_mean, int32_t* index,
                     void* ws, size_t ws_bytes, void* stream);

/*
 * bra_route for callers that cannot hand over scratch memory.  (The paper has
 * no counterpart: this is a packaging variant of bra_route, same arithmetic.)
 *
 * Who needs it: code that runs where device memory must not be allocated or
 * sized at call time - a plug-in inside a host application that owns the
 * memory pool and forbids cudaMalloc, a real-time loop where an allocation's
 * implicit synchronisation is not acceptable, or a caller that simply has no
 * allocator to ask for a `ws` buffer.  bra_route needs `ws` (or caller
 * buffers) for the region means Q^r, K^r between its pooling and its routing
 * kernel; here those means live in a fixed array inside the library image.
 *
 *   Q, K     in   [B,H,W,C] device pointers, as for bra_route
 *   index    out  int32 [B, heads|1, S*S, topk], as for bra_route (bit-identical result)
 *
 * Limits and rules
 *   - B * S*S * C must not exceed BRA_ROUTE_STATIC_MAX_MEAN_FLOATS, otherwise
 *     BRA_ERR_STATIC_LIMIT is returned and nothing is launched.  The array
 *     (2 x that many floats = 4 MiB) is part of the library: every GPU that
 *     loads it carries the array until the process exits.
 *   - The call itself allocates nothing on host or device and frees nothing.
 *   - The first call on each device looks up the array's device address (a
 *     driver query, no allocation).  Make that first call outside any stream
 *     capture; later calls on that device only launch kernels.
 *   - All calls on a device share the one array.  Two calls whose kernels can
 *     overlap on the GPU (different streams, no dependency) race on it: order
 *     them.  The array keeps the previous call's means; nothing in it has to
 *     be zero, because pooling overwrites every element routing then reads.
 *   - The region means are not returned; use bra_route to get them.
 *   - S must divide H and W here (BRA_ERR_UNSUPPORTED otherwise): the padded
 *     copies of Q and K that bra_route makes for other maps would need scratch.
 */
#define BRA_ROUTE_STATIC_MAX_MEAN_FLOATS (512 * 1024)
bra_status bra_route_static(const bra_problem* p, const void* Q, const void* K,
                            int32_t* index, void* stream);

/*
 * Token-to-token attention over routed regions plus LCE (Eq. 6, Eq. 7, Eq. 1):
 *   O = softmax(scale * Q K^g^T) V^g + LCE(V).
 *   index    in   as above (the caller's or bra_route's)
 *   lce_w    in   fp32 [C,5,5]; out[y,x,c] += sum_ij w[c,i,j] V[y+i-2, x+j-2, c], zero outside
 *                 the map; NULL allowed iff p->lce_ksize == 0
 *   lce_b    in   fp32 [C] bias added with LCE; may be NULL
 *   O        out  [B,H,W,C]
 *   lse      out  fp32 [B, heads, H*W]: log of the softmax denominator (natural log, scaled
 *                 scores) of each query; may be NULL.  bra_backward needs it.
 */
bra_status bra_attend(const bra_problem* p, const void* Q, const void* K, const void* V,
                      const int32_t* index, const float* lce_w, const float* lce_b,
                      void* O, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Algorithm 1 from the projected Q, K, V on: bra_route then bra_attend in one call; same results,
 * bit for bit, as the two calls.  The library's kernels are chained on `stream` and overlap at their
 * ends; with BRA_IMPL_TC_FUSED the whole call is one kernel launch.
 *   index    out  may be NULL (then kept in ws only)
 *   lse      out  may be NULL
 */
bra_status bra_forward(const bra_problem* p, const void* Q, const void* K, const void* V,
                       const float* lce_w, const float* lce_b, void* O,
                       int32_t* index, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Gradients of Eq. 7 for a fixed routing index (top-k is not differentiable,
 * so nothing flows through pooling or Eq. 4).  With P the softmax of Eq. 1:
 *   dV^g = P^T dO, dP = dO V^g^T, dS = P o (dP - rowsum(P o dP)),
 *   dQ = scale dS K^g, dK^g = scale dS^T Q, rows of dK^g / dV^g added back to
 *   the regions they were gathered from; LCE: dV += corr^T(dO, w),
 *   d_lce_w[c,i,j] = sum_{b,y,x} dO[b,y,x,c] V[b,y+i-2,x+j-2,c], d_lce_b[c] = sum dO.
 *   lse      in   from bra_attend / bra_forward on the same inputs
 *   dQ,dK,dV out  [B,H,W,C], dtype of p
 *   d_lce_w  out  fp32 [C,5,5]; may be NULL iff p->lce_ksize == 0
 *   d_lce_b  out  fp32 [C]; may be NULL
 * The summation order is fixed: results are bit-identical from run to run.
 */
bra_status bra_backward(const bra_problem* p, const void* Q, const void* K, const void* V,
                        const int32_t* index, const float* lce_w, const float* lse,
                        const void* dO, void* dQ, void* dK, void* dV,
                        float* d_lce_w, float* d_lce_b,
                        void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * What stands around the attention of a block.  The rules at the top hold here too (device pointers,
 * 16-byte aligned, asynchronous on `stream`, errors found on the host return before any launch).
 * Tensors are [B, N, channels] by tokens (a feature map's H x W tokens are N = H * W of them); a
 * stride counts ELEMENTS from one token to the next, 0 stands for dense rows, images follow one
 * another N * stride elements apart, so a tensor may be a slice of channels of a wider one.
 * ------------------------------------------------------------------------------------------------ */

/* Channels of a head that make a pair: neighbours (2i, 2i+1), or (i, i + n/2) of a block of n. */
typedef enum bra_rope_layout { BRA_ROPE_INTERLEAVED = 0, BRA_ROPE_HALF = 1 } bra_rope_layout;

/*
 * Rotary positions.  The first rot_dim channels of every head are rotated, the others copied.  With axes
 * = 2 the rotated channels are two blocks of n = rot_dim / 2, the first turned by a token's first
 * coordinate (its row), the second by its second (its column); with axes = 1 they are one block.
 * Pair i of a block turns by the angle coordinate * freq[i], formed in 64 bits:
 *   (u, v) -> magnitude * (u cos - v sin, u sin + v cos).
 */
typedef struct bra_rope_problem {
    int32_t B, N;             /* images (or sequences), tokens of each */
    int32_t heads, kv_heads;  /* heads of Q and of K (kv_heads 0: there is no K) */
    int32_t head_dim;
    int32_t rot_dim;          /* a multiple of 2 * axes, at most head_dim */
    int32_t layout;           /* bra_rope_layout */
    int32_t axes;             /* 1 or 2 */
    int32_t width;            /* axes = 2 without positions: token t is at row t / width, column t % width */
    int32_t first;            /* axes = 1 without positions: token t is at first + t (>= 0) */
    int32_t dtype;            /* bra_dtype */
    float   magnitude;        /* factor on rotated channels; <= 0 selects 1 */
    int64_t q_stride, k_stride;
} bra_rope_problem;

/* How frequencies are stretched for contexts longer than those a network was trained on. */
typedef enum bra_rope_scaling {
    BRA_ROPE_PLAIN = 0,   /* f_i = base^(-2i/n) */
    BRA_ROPE_LINEAR = 1,  /* f_i / factor */
    BRA_ROPE_BASE = 2,    /* base * factor^(n/(n-2)) in the place of base: the slowest pair is stretched by factor (n > 2) */
    BRA_ROPE_PARTS = 3    /* pairs with r = original_length * f_i / 2 pi >= high turns keep f_i, those with r <= low get
                             f_i / factor, those between a mean of the two, linear in r */
} bra_rope_scaling;

/* Host only: the rot_dim / axes / 2 frequencies of a block, into the HOST array freq. */
bra_status bra_rope_frequencies(int32_t rot_dim, int32_t axes, double base, int32_t scaling, double factor,
                                double original_length, double low, double high, double* freq);

/*
 * Rotates Q and K (K NULL iff kv_heads is 0) in one launch.
 *   positions in   int32 [B, N, axes], or NULL: those that the problem implies
 *   freq      in   double [rot_dim / axes / 2], on the device; a pair whose frequency is infinite or NaN comes out NaN
 *   inverse   in   nonzero: by the negative angle.  That is the transpose, so it is also the gradient:
 *                  dQ = bra_rope(inverse) of the gradient of Qo.
 *   Qo, Ko    out  laid out like Q, K; each may be the very same tensor (in place)
 */
bra_status bra_rope(const bra_rope_problem* p, const void* Q, const void* K, const int32_t* positions,
                    const double* freq, int32_t inverse, void* Qo, void* Ko, void* stream);

/*
 * Cross attention: the queries of a map attend to an encoder's states.  Query head h reads key / value
 * head h / (heads / kv_heads).  Key j of image b is visible iff j < key_len[b] (where key_len is given;
 * below 0 counts as 0) and key_mask[b, j] != 0 (where key_mask is given).  What stands in hidden keys and
 * values, infinities and NaN included, reaches no output.  A query that sees no key (or whose scores
 * are all -inf) has O = 0, lse = -inf and adds nothing to any gradient.  Of what is visible, an infinity
 * makes its scores or sums NaN in fp32 problems, whose operands are split in two for the tensor cores.
 */
typedef struct bra_cross_problem {
    int32_t B, Nq, Nk;        /* images, queries and keys of each */
    int32_t heads, kv_heads;  /* kv_heads divides heads */
    int32_t head_dim;         /* 16, 32, 64 or 128 */
    int32_t dtype;            /* bra_dtype */
    float   scale;            /* softmax scale; <= 0 selects 1/sqrt(head_dim) */
    int64_t q_stride, k_stride, v_stride;   /* multiples of 16 bytes */
} bra_cross_problem;

/* Scratch size in bytes of both calls (0 if p is invalid).  Host only.  Like the routed attention's, this scratch has to be
 * zero before its first use and is left ready for the next one; calls that share it must be ordered on one stream, and
 * bra_device_status reads it (BRA_ERR_TIMEOUT: a wait inside a kernel gave up, the outputs are not complete).  Problems of
 * different sizes may share the scratch of the one that needs most. */
size_t bra_cross_workspace_bytes(const bra_cross_problem* p);

/*
 * O = softmax(scale * Q K^T over visible keys) V.
 *   Q        in   [B, Nq, heads, head_dim], q_stride
 *   K, V     in   [B, Nk, kv_heads, head_dim], k_stride and v_stride
 *   key_len  in   int32 [B]; may be NULL.   key_mask  in  uint8 [B, Nk]; may be NULL
 *   O        out  [B, Nq, heads, head_dim], dense
 *   lse      out  fp32 [B, heads, Nq], natural log of the softmax denominator of the scaled scores; may be NULL
 */
bra_status bra_cross_attend(const bra_cross_problem* p, const void* Q, const void* K, const void* V,
                            const int32_t* key_len, const uint8_t* key_mask, void* O, float* lse,
                            void* ws, size_t ws_bytes, void* stream);

/*
 * Its gradients, from O and lse of bra_cross_attend on the same inputs and dO (dense, like O).
 *   dQ, dK, dV  out  laid out like Q, K, V (same strides); hidden keys get zeros.  dK and dV of a key head are
 *                    the sums over its query heads.  The order of every sum is fixed.
 */
bra_status bra_cross_backward(const bra_cross_problem* p, const void* Q, const void* K, const void* V,
                              const int32_t* key_len, const uint8_t* key_mask, const void* O, const float* lse,
                              const void* dO, void* dQ, void* dK, void* dV,
                              void* ws, size_t ws_bytes, void* stream);

typedef enum bra_norm { BRA_NORM_NONE = 0, BRA_NORM_RMS = 1, BRA_NORM_LAYER = 2 } bra_norm;
typedef enum bra_gate { BRA_GATE_NONE = 0, BRA_GATE_CHANNEL = 1, BRA_GATE_IMAGE = 2 } bra_gate;

/*
 * The norms on both sides of a block's end, fused with its gate and residual scale:
 *   y' = post(y) * post_w + post_b       (post = BRA_NORM_NONE: y' = y)
 *   h  = alpha * x + gate * y'           the residual stream behind the block
 *   n  = pre(h) * w + b                  what the next block reads (pre = BRA_NORM_NONE: no n)
 * with rms(v) = v / sqrt(mean(v^2) + eps) and layer(v) = (v - mean v) / sqrt(var v + eps) over the C channels of
 * a token.  Everything between x, y and the outputs is fp32; n is made from h before its rounding.
 */
typedef struct bra_norm_problem {
    int32_t B, N, C;          /* images, tokens of each (at most 2^30 together), channels (at most 8192) */
    int32_t pre, post;        /* bra_norm */
    int32_t gate;             /* bra_gate: no gate, fp32 [C], fp32 [B, C] */
    int32_t per_image;        /* nonzero: w and b are fp32 [B, C] (modulated by a condition), else [C] */
    int32_t dtype;            /* bra_dtype of x, y, h, n and their gradients */
    float   eps, alpha;
} bra_norm_problem;

/* Scratch size in bytes of bra_residual_norm_backward (0 if p is invalid).  Host only.  It needs no initial value. */
size_t bra_norm_workspace_bytes(const bra_norm_problem* p);

/*
 *   x     in   [B, N, C]
 *   y     in   [B, N, C], the block's output; NULL: h = alpha * x (the first norm of a network; gate and post must be 0)
 *   gate  in   NULL iff p->gate is BRA_GATE_NONE.   post_w, post_b, w, b  in  each may be NULL (ones, zeros)
 *   h     out  [B, N, C]; may be NULL, may be x or y.   n  out  [B, N, C]; NULL iff p->pre is BRA_NORM_NONE
 * BRA_ERR_UNSUPPORTED: h shares only a part of its bytes with x or y, or n shares any with x, y or h.
 */
bra_status bra_residual_norm(const bra_norm_problem* p, const void* x, const void* y, const float* gate,
                             const float* post_w, const float* post_b, const float* w, const float* b,
                             void* h, void* n, void* stream);

/*
 * Gradients.  dh: of h from what follows in the stream, may be NULL (zeros).  dn: of n, NULL iff p->pre is
 * BRA_NORM_NONE.  dx [B, N, C]; dy [B, N, C], NULL iff y is; the others are fp32 in the shapes of their
 * inputs, each may be NULL where it is not wanted.  The forward pass is made again from x and y, so nothing
 * else has to be kept; the order of every sum is fixed.  BRA_ERR_UNSUPPORTED: dx or dy shares bytes with x, y, dh, dn or the other.
 */
bra_status bra_residual_norm_backward(const bra_norm_problem* p, const void* x, const void* y, const float* gate,
                                      const float* post_w, const float* post_b, const float* w,
                                      const void* dh, const void* dn, void* dx, void* dy, float* d_gate,
                                      float* d_post_w, float* d_post_b, float* d_w, float* d_b,
                                      void* ws, size_t ws_bytes, void* stream);

/*
 * Synchronises `stream`, then returns and clears the first device-detected
 * error recorded in ws (BRA_OK, BRA_ERR_INDEX, BRA_ERR_TIMEOUT, or BRA_ERR_CUDA
 * if the synchronisation itself failed).  When it reports an error it also puts the
 * barrier counters in ws back to zero (as bra_workspace_init does), so the next call
 * starts clean.  ws must have been initialised and used by an earlier call.
 */
bra_status bra_device_status(void* ws, void* stream);

/* Number of kernels launched by the last bra_* call on this thread (host-side count). */
int32_t bra_last_launch_count(void);

/* Static description of a status code. Never NULL. */
const char* bra_status_string(bra_status s);

/* Library version: major * 10000 + minor * 100 + patch. */
int32_t bra_version(void);

#ifdef __cplusplus
}
#endif
#endif /* BRA_H_ */
