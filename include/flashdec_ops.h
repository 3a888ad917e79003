/*
 * flashdec_ops.h - kernel-level entry points of the FlashDecoder library.
 *
 * Each call enqueues one of the decoder's kernels on caller-owned device buffers and returns
 * after enqueueing (stream-ordered, no host synchronisation). They exist so each step of the
 * decode path (Algorithm 1) can be checked and timed on its own; fd_decode_chunk runs the
 * same kernels. All pointers are device pointers unless stated; `stream` is a cudaStream_t
 * as void*. `err_dev` is a device int32 the kernel ORs error bits into when one of its
 * bounded waits gives up (1 TMA load, 2 MMA commit, 4 accumulator release, 8 shared-memory
 * alignment); the caller zeroes it and reads it after synchronising. Argument errors are
 * reported synchronously as FD_ERR_INVALID_ARG; nothing is launched then.
 */
#ifndef FLASHDEC_OPS_H
#define FLASHDEC_OPS_H

#include "flashdec.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FD_EPI_F32 = 0,   /* out fp32 [M][N]  = A W^T + b                                   */
  FD_EPI_RESID = 1, /* out fp32 [M][N] += A W^T + b          (residual, Sec. 3.2)      */
  FD_EPI_GELU = 2,  /* out bf16 [M][N]  = GELU_erf(A W^T + b) (MLP, R7; head, Sec. 3.4) */
  FD_EPI_TUP = 3,   /* out fp32 [(N / tup_hidden) M][tup_hidden]: column tau*D + d of row
                       l goes to row tau*M + l, column d (Eq. temporal_upsample)          */
  FD_EPI_SWIGLU = 4 /* out bf16 [M][N/2]: gated SiLU MLP (XL layout). W and bias rows come in
                       blocks of 64: rows 64j..64j+31 gate and 64j+32..64j+63 up of hidden
                       units 32j..32j+31; out[m][32j+i] = SiLU(g + bg) * (u + bu)          */
} fd_epilogue;

/* Linear layer on the tensor cores (tcgen05, bf16 in, fp32 accumulate).
 * A bf16 [M][K] row-major; W bf16 [N][K] row-major (nn.Linear); bias fp32 [N].
 * Requires N % 32 == 0 (N % 64 == 0 for FD_EPI_GELU, N % 128 == 0 for FD_EPI_SWIGLU),
 * K % 8 == 0, 16-byte aligned A / W / out / bias. bn = output tile width (64, 96, 128, 192
 * or 256; 96 only for the fp32 epilogues, 128 or 256 for FD_EPI_SWIGLU; 0 = library choice). */
fd_status fd_op_linear(int epilogue, int M, int N, int K, const void* A, const void* W,
                       const float* bias, void* out, int tup_hidden, int bn, int* err_dev,
                       void* stream);

/* The same with the launch shape chosen by the caller: bn as above (0 = library choice of
 * everything), pair = 1 for 128-row tiles on single CTAs, 2 for 256-row tiles on CTA pairs
 * (tcgen05 cta_group::2: each CTA of the pair holds its 128 rows of A and half of W's bn rows,
 * the even CTA issues the pair's MMAs; bn 96 / 128 / 192 / 256), 0 = library choice. Results
 * do not depend on the shape. fd_op_linear runs an explicit bn on single CTAs. */
fd_status fd_op_linear_tiled(int epilogue, int M, int N, int K, const void* A, const void* W,
                             const float* bias, void* out, int tup_hidden, int bn, int pair,
                             int* err_dev, void* stream);

/* Temporal 3D-RoPE table of chunk t (Sec. 3.2, reading of Algorithm 1's "RoPE offset"):
 * table[tau][i] = (cos, sin)((t * frames_per_chunk + tau) * rope_base^(-2i/24)) for the
 * frames_per_chunk frames of the chunk and the 12 temporal pairs (fp32 values of an fp64
 * evaluation). table: device float [frames_per_chunk][12][2]. */
fd_status fd_op_rope_table(int t, int frames_per_chunk, float rope_base, float* table,
                           void* stream);

/* Fused QKV projection of one attention block (Sec. 3.2, Sec. 3.3 step (2)):
 *   [Q | K | V] = A Wqkv^T + b   (Wqkv rows: heads*64 query, groups*64 key, groups*64 value)
 *   K, V <- RMSNorm over the 64 head dims with gains knorm_g / norm2_g (KV-norm), or with
 *           qk_norm = 1: Q, K <- RMSNorm with gains norm2_g / knorm_g (QK-norm), V as is
 *   Q, K <- 3D-RoPE at temporal index t*frames_per_chunk + row / tokens (cos / sin from
 *           rope_t, the fd_op_rope_table of chunk t), row and column of token (row % tokens)
 *           in a grid of width grid_w (rope_base; bands 24/20/20 dims)
 *   q_out bf16 [M][heads*64];  K -> k_ring bf16 [groups][ring_pitch][64] rows
 *   (t mod window)*M + row;  V -> vt_ring fp16 [groups][64][ring_pitch] (transposed), same
 *   key index.  M = frames_per_chunk * tokens; ring_pitch % 128 == 0, >= window * M;
 *   bqkv, q_out and the rings 16-byte aligned. */
fd_status fd_op_qkv(int M, int K, const void* A, const void* Wqkv, const float* bqkv,
                    const float* knorm_g, const float* norm2_g, int qk_norm, int heads, int groups,
                    int tokens, int grid_w, int frames_per_chunk, int window, int t, float eps,
                    float rope_base, const float* rope_t, void* q_out, void* k_ring,
                    void* vt_ring, int ring_pitch, int bn, int* err_dev, void* stream);

/* Attention of Lq queries over the first n_keys keys of a ring (Sec. 3.3, Eq. kv_cache):
 *   out[r][n*64 + d] = sum_j softmax_j(q_n . k_j / 8) v_j[d],  KV group g = n / (heads/groups)
 * q bf16 [Lq][heads*64]; k_ring bf16 [groups][ring_pitch][64]; vt_ring fp16
 * [groups][64][ring_pitch]; out bf16 [Lq][heads*64]. 1 <= n_keys <= ring_pitch,
 * ring_pitch % 128 == 0. Ring entries past n_keys must hold finite values.
 * parts: CTAs of the launch (0 = library choice, one per SM; 1..4096). The launch is
 * persistent: the query rows of the heads of each KV group are packed into 128-row tiles, the
 * (tile pair x 128-key block) units are cut into `parts` equal runs, one per CTA, and a tile
 * pair whose keys fall into several runs is finished by combining partial results. With
 * parts > 1, `workspace` is a caller-owned device buffer of fd_attention_workspace_bytes(...)
 * bytes (16-byte aligned) that the call overwrites (its counters are cleared on `stream` first);
 * calls sharing it must not overlap. The combine order is fixed: results do not depend on
 * which CTA finishes first. */
size_t fd_attention_workspace_bytes(int Lq, int heads, int groups, int n_keys, int parts);
fd_status fd_op_attention(int Lq, int heads, int groups, const void* q, const void* k_ring,
                          const void* vt_ring, int ring_pitch, int n_keys, void* out,
                          int parts, void* workspace, int* err_dev, void* stream);

/* Allocation-free variant of fd_op_attention. The paper has no counterpart: this is a library
 * convenience for callers that cannot call cudaMalloc, for example plug-ins that must stay
 * inside a device-memory budget handed to them by a host framework (which owns every
 * allocation), and real-time loops that cannot afford the device synchronisation an allocation
 * may cause. Such callers can pass their own inputs and outputs but have no way to provide the
 * partial-result workspace.
 * This call takes that workspace from one array in the library's static device memory,
 * FD_STATIC_ATTN_SCRATCH_BYTES (32 MiB) on every GPU that loads the library, held until the
 * process exits. It allocates nothing: no cudaMalloc, cudaFree or allocating library routine.
 *   - Arguments and results are those of fd_op_attention without `workspace`. parts = 0 lets
 *     the library choose (one CTA per SM: about 135 KB per SM). If
 *     fd_attention_workspace_bytes(..., parts) would exceed the static size, the call returns
 *     FD_ERR_INVALID_ARG and launches nothing (pass fewer parts; parts = 1 uses no workspace).
 *   - The 32 MiB are reserved on a device when the library's device code is loaded there,
 *     which with CUDA's lazy module loading may be this call's first use on that device.
 *   - The first call in a CUDA context (per device, and again after a device reset, which
 *     makes a new context) looks up the array's device address with that context current
 *     (cudaGetSymbolAddress); make that first call before any stream capture begins.
 *   - Every call shares the one array; it clears the array's counters on `stream` (a memset,
 *     not an allocation) and writes every other entry it later reads. Calls whose kernels
 *     overlap on the GPU (unordered streams) race on the array and may return wrong results. */
#define FD_STATIC_ATTN_SCRATCH_BYTES (32u << 20)
fd_status fd_op_attention_static(int Lq, int heads, int groups, const void* q,
                                 const void* k_ring, const void* vt_ring, int ring_pitch,
                                 int n_keys, void* out, int parts, int* err_dev, void* stream);

/* Rolling-cache append (Algorithm 1, cache update): fp32 k, v [groups][rows][64] rounded to
 * nearest even into ring slot s = t mod window: k_ring[g][s*rows + r][d] (bf16) and
 * vt_ring[g][d][s*rows + r] (fp16). The oldest chunk's slot is overwritten (eviction). */
fd_status fd_op_kv_append(const float* k, const float* v, int groups, int rows, int window,
                          int t, int ring_pitch, void* k_ring, void* vt_ring, void* stream);

/* u bf16 [M][D] = h / sqrt(mean(h^2) + eps) * g   (RMSNorm, Sec. 3.2); D % 128 == 0. */
fd_status fd_op_rmsnorm(const float* h, const float* g, int M, int D, float eps, void* u,
                        void* stream);

/* The same with e4m3 output (the input of an FP8 MLP, Sec. 4.6):
 * u e4m3 [M][D] = e4m3(h / sqrt(mean(h^2) + eps) * g * out_scale), round to nearest even,
 * saturating at +-448. */
fd_status fd_op_rmsnorm_e4m3(const float* h, const float* g, int M, int D, float eps,
                             float out_scale, void* u, void* stream);

/* FP8 linear layer (the MLP products of the FP8 option, Sec. 4.6): A e4m3 [M][K], W e4m3
 * [N][K] (nn.Linear layout), col_scale fp32 [N] (the dequantisation s_A * s_W[n]), bias fp32
 * [N]; acc = sum_k A[m][k] W[n][k], exact e4m3 products accumulated in fp32 (tcgen05
 * kind::f8f6f4):
 *   FD_EPI_F32    out fp32 [M][N]  = acc * col_scale + bias
 *   FD_EPI_RESID  out fp32 [M][N] += acc * col_scale + bias
 *   FD_EPI_GELU   out e4m3 [M][N]  = e4m3(GELU(acc * col_scale + bias) * out_scale)
 *   FD_EPI_SWIGLU out e4m3 [M][N/2] = e4m3(SiLU(g) u * out_scale), g / u = acc * col_scale +
 *                 bias of the gate / up rows, interleaved in blocks of 32 as for fd_op_linear
 *                 (the FP8 gated MLP layer 1); N % 256 == 0
 * K % 16 == 0, N % 32 == 0 (N % 128 == 0 for FD_EPI_GELU), 16-byte aligned A / W / out /
 * bias / col_scale.
 * bn = output tile width (96 / 128 / 192 / 256, 128 or 256 for FD_EPI_GELU; 0 = choice). */
fd_status fd_op_linear_e4m3(int epilogue, int M, int N, int K, const void* A, const void* W,
                            const float* col_scale, const float* bias, void* out,
                            float out_scale, int bn, int* err_dev, void* stream);

/* PixelUnshuffle(p) of a latent frame z fp32 [C][H][W] into tokens x0 bf16 [(H/p)(W/p)][C p^2]
 * (Sec. 4.3; raster token order of Eq. projection). */
fd_status fd_op_unshuffle(const float* z, int C, int H, int W, int p, void* x0, void* stream);

/* Pixel head (Sec. 3.4 Step 3): F fp32 [frames * gh * gw][C rs^2] -> pixels
 * [C][frames][gh rs][gw rs], pix = clamp(F[tau*L + y/rs*gw + x/rs][c rs^2 + (y%rs) rs + x%rs],
 * -1, 1), as fp32 or uint8 code round_half_even((pix + 1) * 127.5) (NaN -> 0). rs % 4 == 0. */
fd_status fd_op_pixel_head(const float* F, int frames, int grid_h, int grid_w, int channels,
                           int rs, int out_dtype, void* pixels, void* stream);

/* Head layer 2 with the pixel shuffle folded into the product's epilogue (Sec. 3.4 Step 3;
 * the decoder's last product, run this way by fd_decode_chunk): in one launch, the pixels that
 * fd_op_pixel_head gives from fd_op_linear's F = A W^T + b, bit for bit, without storing F.
 * A bf16 [M][K], the rows of frame tau's tokens at tau L .. tau L + L - 1 (L = grid_h grid_w);
 * W bf16 [channels rs^2][K]; bias fp32 [channels rs^2]. The first `frames` frames (frames L <=
 * M) are written: pixels [channels][frames][grid_h rs][grid_w rs], fp32 clamped to [-1, 1]
 * (out_dtype FD_DTYPE_F32) or uint8 codes (FD_DTYPE_U8). 128 x 256 tiles on single CTAs. rs % 4 == 0, 32 % rs == 0,
 * K % 8 == 0, (channels rs^2) % 32 == 0; 16-byte aligned A / W / bias / pixels.
 * Errors: FD_ERR_INVALID_ARG, FD_ERR_CUDA; err_dev as for fd_op_linear. */
fd_status fd_op_linear_pixel(int M, int K, const void* A, const void* W, const float* bias,
                             int frames, int grid_h, int grid_w, int channels, int rs,
                             int out_dtype, void* pixels, int* err_dev, void* stream);

/* ---- single kernels of the training step (fd_train_step), for per-kernel checks ---- */

/* The attention's scores backward in one launch (the training step's, Sec. 3.3 attention with
 * its softmax derivative): S = Q K^T and dP = dO V^T on the tensor cores (never stored), then
 *   P = exp(S / sqrt(64) - lse[r]), dS = P (dP - delta[r]) / sqrt(64)
 * with P = 0 on padding query rows (r mod Pc mod Lp >= L) and padding keys (c mod Lp >= L),
 * written as dS bf16 [M][N], dS^T and P^T bf16 [N][M]. Q, dO bf16 [M][64]; K, V bf16 [N][64];
 * lse, delta fp32 [M]. N % 32 == 0, Pc % Lp == 0, 0 < L <= Lp; 16-byte aligned.
 * Errors: FD_ERR_INVALID_ARG, FD_ERR_CUDA; err_dev as for fd_op_linear. */
fd_status fd_op_scores_bwd(int M, int N, const void* Q, const void* dO, const void* K,
                           const void* V, const float* lse, const float* delta, int Pc, int Lp,
                           int L, void* dS, void* dST, void* PT, int* err_dev, void* stream);

/* RMSNorm backward (the derivative of y = x r g, r = (mean(x^2) + eps)^(-1/2), Sec. 3.2):
 * dx = r (dy g) - x r^3 sum_j(dy_j g_j x_j) / D and dg = sum over rows of dy x r.
 * x, dy, dx fp32 [M][D]; g, dg fp32 [D]; work: fp32 [M][D] scratch of the caller. */
fd_status fd_op_rmsnorm_bwd(const float* x, const float* g, const float* dy, int M, int D,
                            float eps, float* dx, float* dg, float* work, void* stream);

/* GELU backward, exact form: dz = da (Phi(z) + z phi(z)); fp32 z, da, dz and a bf16 copy of dz
 * (the operand of the next products), n elements each. */
fd_status fd_op_gelu_bwd(const float* z, const float* da, int64_t n, float* dz, void* dz_bf16,
                         void* stream);

/* The L1 term of one chunk's pixels through the pixel shuffle (Sec. 3.4 Step 3, Sec. 3.5 Eq.
 * loss): F fp32 [frames grid_h grid_w][channels rs^2] (refined token tau L + l), target fp32
 * [channels][frames][grid_h rs][grid_w rs]; loss = mean |PixelShuffle(F) - target| (one fp32)
 * and dF = sign(F - target) / (pixel count) in F's layout. work: fp32 scratch of
 * ceil(frames L channels rs^2 / 256) elements. */
fd_status fd_op_l1_pixel_bwd(const float* F, const float* target, int frames, int grid_h,
                             int grid_w, int channels, int rs, float* dF, float* loss,
                             float* work, void* stream);

/* ---- rotary positions ---- */

/* How a head's leading rot_dim elements are paired: pair i is elements (2i, 2i + 1) or
 * (i, i + rot_dim / 2). */
typedef enum { FD_ROTARY_INTERLEAVED = 0, FD_ROTARY_HALF = 1 } fd_rotary_layout;

/* How the frequencies f = base^(-2i/d) of an axis of d elements are stretched to contexts
 * `factor` times longer than those trained on:
 *   LINEAR  f / factor (positions interpolated)
 *   BASE    base * factor^(d / (d - 2)) for base: the slowest pair of the axis is slowed by
 *           `factor`, the fastest not at all (axes of 2 elements keep their one frequency)
 *   BLEND   g f + (1 - g) f / factor with g = clamp((n - slow_turns) / (fast_turns -
 *           slow_turns), 0, 1) and n = trained_len f / (2 pi), the pair's turns over the
 *           trained context: fast pairs as they are, slow ones interpolated */
typedef enum {
  FD_ROTARY_SCALE_NONE = 0,
  FD_ROTARY_SCALE_LINEAR = 1,
  FD_ROTARY_SCALE_BASE = 2,
  FD_ROTARY_SCALE_BLEND = 3
} fd_rotary_scaling;

typedef struct {
  int32_t head_dim;      /* elements of a head, 2..256                                      */
  int32_t rot_dim;       /* leading elements that are turned, even, 2..head_dim             */
  int32_t layout;        /* fd_rotary_layout                                                */
  int32_t axes;          /* position axes, 1..3 (time, row, column for video tokens)        */
  int32_t axis_dims[3];  /* elements turned by each axis, even, >= 2, their sum is rot_dim  */
  int32_t scaling;       /* fd_rotary_scaling                                               */
  float base;            /* > 0                                                             */
  float factor;          /* > 0; used unless scaling is NONE                                */
  int32_t trained_len;   /* >= 1; BLEND                                                     */
  float fast_turns;      /* > slow_turns; BLEND                                             */
  float slow_turns;
  float amplitude;       /* turned elements are multiplied by it, finite (1: a rotation)    */
} fd_rotary_config;

/* The frequencies of one configuration. A host object: it holds no device memory, any number of
 * calls on any streams and devices may use it at once. */
typedef struct fd_rotary_s* fd_rotary;
fd_status fd_rotary_create(const fd_rotary_config* cfg, fd_rotary* out);
fd_status fd_rotary_destroy(fd_rotary plan);

/* Turns queries and keys by their positions, in one launch: for pair (a, b) of axis x at
 * frequency f and angle t = positions[token][x] f
 *   a' = amplitude (a cos t - b sin t),  b' = amplitude (a sin t + b cos t)
 * and with backward = 1 the gradient (the transposed turn: t negated), from the gradients of
 * the outputs to those of the inputs. Elements past rot_dim are copied. A position's phase
 * is an integer product modulo one turn, so no int32 position, negative ones too, loses its
 * angle to rounding.
 * dtype FD_DTYPE_F32 / BF16 / F16 of q, k and the outputs; positions int32 [tokens][axes].
 * Element (token, head, i) of q is at q[token q_token_stride + head q_head_stride + i], of q_out
 * with the out strides (in elements, any values that keep the heads apart), k likewise; k with 0 heads is
 * left out (pointers may be NULL). An output may be its input (same pointer and strides), no
 * other overlap is allowed. tokens may be 0. */
fd_status fd_op_rotary(fd_rotary plan, int backward, int dtype, int tokens,
                       const int32_t* positions, int q_heads, const void* q,
                       int64_t q_token_stride, int64_t q_head_stride, void* q_out,
                       int64_t q_out_token_stride, int64_t q_out_head_stride, int k_heads,
                       const void* k, int64_t k_token_stride, int64_t k_head_stride, void* k_out,
                       int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream);

/* ---- a cache of bounded size that keeps what attention uses ----
 *
 * For streams that are not served by the last W chunks alone: every (stream, KV group) has
 * `capacity` slots, each holding a key, a value, the position that they belong to and the
 * attention weight that the entry has gathered so far. Slots are in no order. New tokens take
 * the slots of the entries with the least weight (fd_op_cache_insert), attention reads the
 * slots and adds to their weights (fd_op_cache_attention), a long first pass is cut down once
 * (fd_op_cache_compact). An empty slot has a negative position; the caller sets all positions to
 * -1 before the first insert. Whatever an empty slot's key, value and weight hold (NaN too) has
 * no effect. Entries that are in use have finite keys and values. */
typedef struct {
  int32_t streams, groups, capacity;  /* >= 0, >= 1, 0..1,048,576                            */
  int32_t head_dim;                   /* 64 or 128                                          */
  int32_t dtype;                      /* FD_DTYPE_BF16 or FD_DTYPE_F16                      */
  int32_t reserved;                   /* 0                                                  */
  void* k;                            /* element i of slot j: k[stream stream_stride + group */
  void* v;                            /*   group_stride + j slot_stride + i]; v the same     */
  int64_t stream_stride, group_stride, slot_stride; /* elements, multiples of 8, >= head_dim (>= 0
                                         of one stream or group); k and v 16-byte aligned   */
  int32_t* pos;                       /* [streams][groups][capacity]                        */
  float* weight;                      /* [streams][groups][capacity]                        */
} fd_cache;

/* Attention of n_q queries a stream over the first `used` slots of its cache, and the weights
 * that they give to each slot:
 *   p[t][h][j] = softmax over the visible slots j of scale q[t][h] . k[j];  KV group h / (heads / groups)
 *   out[t][h]  = sum_j p[t][h][j] v[j]
 *   weight_out[j] = decay weight[j] + sum over the queries t and the group's heads h of p[t][h][j]
 * Slot j is visible to query t if 0 <= pos[j] <= q_pos[t] (one position for all tokens of a
 * chunk lets each see the whole chunk). A query that sees no slot gives zeros and adds nothing.
 * q, out of the cache's type: element (stream, t, h, i) of q at q[stream q_stream_stride + t
 * q_token_stride + h q_head_stride + i], of out with the out strides (elements; 16-byte
 * aligned; strides multiples of 8, and >= head_dim where there is more than one entry). out
 * shares no memory with q, which is read again for the weights, or with the cache. q_pos int32
 * [streams][n_q]. scale > 0, finite; decay finite;
 * heads / groups <= 128, streams groups <= 65,535, n_q heads / groups <= 1,048,560. weight_out fp32
 * [streams][groups][capacity], entries past `used` are not written; it may be cache->weight;
 * NULL: the weights are not gathered. Softmax, sums and weights are in fp32, P is rounded to the
 * cache's type for its product with V. The order of every sum is fixed: equal calls give equal
 * bits. workspace: fd_cache_attention_workspace_bytes(...) bytes of device memory (16-byte
 * aligned) that the call overwrites; calls that may overlap need one each. err_dev as for
 * fd_op_linear. streams, n_q and used may be 0 (with used = 0 out is zeros). */
size_t fd_cache_attention_workspace_bytes(const fd_cache* cache, int used, int heads, int n_q);
fd_status fd_op_cache_attention(const fd_cache* cache, int used, int heads, int n_q,
                                const void* q, int64_t q_stream_stride, int64_t q_token_stride,
                                int64_t q_head_stride, const int32_t* q_pos, float scale,
                                float decay, void* out, int64_t out_stream_stride,
                                int64_t out_token_stride, int64_t out_head_stride,
                                float* weight_out, void* workspace, int* err_dev, void* stream);

/* Failure-path check: the waits of the attention's kernels for many rows give up after 2 s; here one of
 * them (0 a thread's, 1 a thread's for copies in flight, 2 a warp's, 3 a polling loop) waits on a
 * barrier that nothing arrives at, with a limit of 1 ms, and sets bit 32 of *err_dev when it gives up.
 * (All but 1 give up early where *err_dev is not 0 already.) The kernel ends by itself. */
fd_status fd_debug_cache_wait_timeout(int which, int* err_dev, void* stream);

/* New tokens into the cache, evicting what they displace. For each (stream, group), the slots
 * are ranked by (class, weight, slot index): class 0 empty slots (weights ignored), class 1
 * entries that nothing protects, class 2 protected ones (pos < sinks, or pos >= new_pos[0] -
 * recent of the stream). The first n_new in this order are given up, so ties go to the lowest
 * index, -0 ranks as +0 and NaN above every number, and the n_new new tokens take them in the order
 * of their slot index. slots int32 [streams][groups][n_new]: the slots taken, ascending.
 * The new entries' positions are new_pos int32 [streams][n_new] (>= 0) and their weight is 0.
 * k_new, v_new of the cache's type: element (stream, t, group, i) at k_new[stream
 * new_stream_stride + t new_token_stride + group new_group_stride + i] (elements; 16-byte
 * aligned, strides multiples of 8). pos_out, weight_out: [streams][groups][capacity] arrays
 * that receive all positions and weights; they may be cache->pos and cache->weight. Keys and
 * values are written in place. 0 <= n_new <= capacity <= 1,048,576; sinks, recent >= 0. */
fd_status fd_op_cache_insert(const fd_cache* cache, int n_new, const void* k_new,
                             const void* v_new, int64_t new_stream_stride,
                             int64_t new_token_stride, int64_t new_group_stride,
                             const int32_t* new_pos, int sinks, int recent, int32_t* pos_out,
                             float* weight_out, int32_t* slots, void* stream);

/* Cuts a cache down: for each (stream, group), of the first `used` slots of src the
 * dst->capacity that rank last in the order of fd_op_cache_insert (recency counts from
 * now[stream], int32) are copied to dst with their positions and weights, in the order of their
 * slots; where src has fewer entries, the slots at dst's end are empty (position -1, weight 0,
 * key and value zero). src_slots int32 [streams][groups][dst->capacity]: the slot that each came
 * from, -1 for an empty one. src and dst have the same streams, groups, head_dim and dtype and
 * share no memory. 0 <= used <= src->capacity, dst->capacity <= used <= 1,048,576. */
fd_status fd_op_cache_compact(const fd_cache* src, int used, const fd_cache* dst,
                              const int32_t* now, int sinks, int recent, int32_t* src_slots,
                              void* stream);

/* ---- attention in which every query sees a span of keys, and its gradient ----
 *
 * n_q queries of `heads` heads and n_k keys of `groups` KV heads (head h reads group h / (heads /
 * groups)); query t sees the keys j with spans[t][0] <= j < spans[t][1] (spans int32 [n_q][2], 8-byte
 * aligned; bounds outside of [0, n_k) are cut off, an empty span sees nothing). Sequences packed one
 * behind another, causal masks, the decoder's chunks with their window and new tokens after a past
 * are all such spans.
 * Element (token, head, i) of a matrix is at its token_stride token + head_stride head + i (elements;
 * multiples of 8, >= head_dim where there is more than one; 16-byte aligned pointers).
 * What no query sees, and the rows of queries that see nothing, have no effect whatever they hold
 * (NaN too). Keys and values that some query sees, and the queries (and their gradients) that see some,
 * are finite. */
typedef struct {
  int32_t n_q, n_k;         /* 0..16,777,216; n_q heads, n_k groups <= 2^36                   */
  int32_t heads, groups;    /* heads % groups == 0, heads / groups <= 128, heads <= 65,535    */
  int32_t head_dim;         /* 64 or 128                                                      */
  int32_t dtype;            /* FD_DTYPE_BF16 or FD_DTYPE_F16                                  */
  float scale;              /* of the scores, > 0, finite                                     */
} fd_span_attention;

/* Workspace of the call below (backward = 0) or of its gradient (1), bytes of device memory, 16-byte
 * aligned, that a call overwrites; calls that may overlap need one each. */
size_t fd_span_attention_workspace_bytes(const fd_span_attention* attn, int backward);

/* out[t][h] = sum_j exp(s_j - lse) v_j,  s_j = scale q[t][h] . k_j,  lse[h][t] = log sum_j exp(s_j)
 * (fp32, natural logarithm). A query that sees nothing gets zeros and -inf. Softmax and sums are in fp32, the
 * probabilities are rounded to dtype for their product with V (fp16: times a power of two that keeps its digits
 * down to 2^-25 of the row's largest; smaller ones are off by 2^-36 of that each). The order of every sum is
 * fixed: equal calls give equal bits. out shares no memory with the inputs. err_dev as for fd_op_linear. */
fd_status fd_op_span_attention(const fd_span_attention* attn, const void* q, int64_t q_token_stride,
                               int64_t q_head_stride, const void* k, int64_t k_token_stride,
                               int64_t k_head_stride, const void* v, int64_t v_token_stride,
                               int64_t v_head_stride, const int32_t* spans, void* out,
                               int64_t out_token_stride, int64_t out_head_stride, float* lse,
                               void* workspace, int* err_dev, void* stream);

/* The gradient, from dout like out, with out and lse as the forward call left them:
 *   P = exp(s - lse),  dS = P (dout . v_j - dout . out)
 *   dq[t][h] = scale sum_j dS k_j;  dk[j] = scale sum dS q[t][h];  dv[j] = sum P dout[t][h]
 * (dk, dv over the queries and the group's heads). The probabilities are computed again and never
 * stored. Sums are in fp32 and a fixed order: equal calls give equal bits; P and dS are rounded to dtype for
 * their products. (fp16: scaled by powers of two, so that P keeps its digits down to 2^-28, and dS down to 2^-28 of
 * its bound, the largest sum_i |dout_i| (max |v_i| + max |out_i|): for dq that of its query over the keys that it
 * sees, for dk that of its key over the queries and heads that see it. Smaller ones are off by 2^-39 each, or by
 * that of the bound.)
 * Queries that see nothing and keys that nothing sees get zeros; a query that sees one key (P = 1 whatever
 * the scores) gets dq = 0 and adds nothing to dk. dq like q, dk and dv like k, each with
 * strides of its own;
 * they share no memory with the inputs or each other. spans, err_dev as above; workspace of
 * fd_span_attention_workspace_bytes(attn, 1). */
fd_status fd_op_span_attention_bwd(
    const fd_span_attention* attn, const void* q, int64_t q_token_stride, int64_t q_head_stride,
    const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
    int64_t v_token_stride, int64_t v_head_stride, const int32_t* spans, const void* out,
    int64_t out_token_stride, int64_t out_head_stride, const float* lse, const void* dout,
    int64_t dout_token_stride, int64_t dout_head_stride, void* dq, int64_t dq_token_stride,
    int64_t dq_head_stride, void* dk, int64_t dk_token_stride, int64_t dk_head_stride, void* dv,
    int64_t dv_token_stride, int64_t dv_head_stride, void* workspace, int* err_dev, void* stream);

/* ---- checkpoints: activations kept in 8 bits for the backward pass ----
 *
 * Blocks of 32 neighbouring elements of a row share a power of two 2^E, the smallest with E >= -126
 * that lets the block's largest magnitude fit into 127 steps; an element is the code
 * rint(x 2^-E), ties to even, and stands for code 2^E: at most half a step, 2^(E - 1), off, which is
 * at most 1/127 of the block's largest magnitude. codes int8 [rows][width], exps uint8
 * [rows][ceil(width / 32)] holding E + 127. A block that holds an infinity or a NaN has the byte 255 and
 * codes 0, and is restored as NaN. (What rounds past the largest finite number of the type stays
 * at the last step, or at the largest fp16 number, before it.) */

/* x of dtype FD_DTYPE_F32 / BF16 / F16, element (row, i) at x[row x_stride + i], into codes and exps.
 * width % 8 == 0, 8..1,048,576; x 16-byte aligned, x_stride % 8 == 0; codes 8-byte aligned. rows
 * 0..2^30. */
fd_status fd_op_checkpoint_save(int dtype, int rows, int width, const void* x, int64_t x_stride,
                                int8_t* codes, uint8_t* exps, void* stream);

/* The values back, rounded to dtype (exact in fp32 and bf16). transposed = 0: element (row, i) at
 * x[row x_stride + i], x 16-byte aligned, x_stride % 8 == 0 and >= width. transposed = 1, the operand of a
 * weight gradient: element (row, i) at x[i x_stride + row], x_stride >= rows, any alignment of whole
 * elements. */
fd_status fd_op_checkpoint_load(int dtype, int transposed, int rows, int width,
                                const int8_t* codes, const uint8_t* exps, void* x,
                                int64_t x_stride, void* stream);

/* ---- the join between two residual blocks ----
 *
 * The norm after a block, its gate and residual scale, the residual sum and the norm before the
 * next block, for `rows` tokens of `width` elements in one pass:
 *   n = b r_post,  r_post = (mean(b^2) + eps)^(-1/2)      (post_gain NULL: n = b, a gain of ones)
 *   y = h + scale gate n post_gain                        (gate NULL: ones)
 *   u = y r_pre pre_gain,  r_pre = (mean(y^2) + eps)^(-1/2)   (pre_gain NULL: no u)
 * in fp32; the norm before is that of y before it is rounded. */
typedef struct {
  int32_t rows, width;      /* rows 0..2^30; width % 8 == 0, 8..8192                          */
  int32_t dtype;            /* of b, u, du and db: FD_DTYPE_BF16 or FD_DTYPE_F16              */
  int32_t stream_dtype;     /* of h, y, dy and dh: FD_DTYPE_F32 or dtype                      */
  const float* post_gain;   /* [width] or NULL                                                */
  const float* pre_gain;    /* [width] or NULL                                                */
  const float* gate;        /* [ceil(rows / gate_rows)][width] or NULL; token t has the gate of row
                               t / gate_rows (one gate for all: gate_rows >= rows; a token's own: 1) */
  int32_t gate_rows;        /* >= 1 with a gate                                               */
  float scale;              /* finite                                                         */
} fd_block_join;

/* Forward. Rows of h, b, y, u are their strides apart (elements, multiples of 8, >= width where there
 * is more than one row); pointers 16-byte aligned. y may be h and u may be b (same pointer and strides), no other
 * overlap is allowed. u is NULL without a pre_gain. r_post, r_pre [rows] receive the norms' factors,
 * which the gradient needs (NULL: not wanted). h_codes, h_exps and b_codes, b_exps (both NULL: not
 * wanted) receive h and b as fd_op_checkpoint_save gives them. eps >= 0. */
fd_status fd_op_block_join(const fd_block_join* join, const void* h, int64_t h_stride,
                           const void* b, int64_t b_stride, float eps, void* y, int64_t y_stride,
                           void* u, int64_t u_stride, float* r_post, float* r_pre,
                           int8_t* h_codes, uint8_t* h_exps, int8_t* b_codes, uint8_t* b_exps,
                           void* stream);

/* Gradient, from those of y (dy; NULL: zero, with a pre_gain only) and u (du; NULL without a pre_gain):
 * with m = y r_pre, g = du pre_gain and y = h + scale gate n post_gain computed again,
 *   d = dy + r_pre (g - m mean(g m));  dh = d;  w = scale d
 *   d_gate = sum w n post_gain;  d_post = sum w gate n;  d_pre = sum du m
 *   e = w gate post_gain;  db = r_post (e - n mean(e n))
 * (without the norms: d = dy, db = w gate). h_exps not NULL: h points to codes of rows of `width` (h_stride =
 * width), their exponents at h_exps; b the same. h is not read without a pre_gain. dh may be dy, db may
 * be du or a b that is not in codes (same pointer and strides); dh, db, d_post, d_pre, d_gate may be NULL: not
 * wanted. Sums over tokens are in a fixed order: equal calls give equal bits. workspace: fd_block_join_bwd_workspace_bytes(...) bytes of device
 * memory (16-byte aligned) that the call overwrites; calls that may overlap need one each. With rows
 * = 0 d_post and d_pre are zeros. */
size_t fd_block_join_bwd_workspace_bytes(int rows, int width);
fd_status fd_op_block_join_bwd(const fd_block_join* join, const void* dy, int64_t dy_stride,
                               const void* du, int64_t du_stride, const void* h, int64_t h_stride,
                               const uint8_t* h_exps, const void* b, int64_t b_stride,
                               const uint8_t* b_exps, const float* r_post, const float* r_pre,
                               void* dh, int64_t dh_stride, void* db, int64_t db_stride,
                               float* d_post, float* d_pre, float* d_gate, void* workspace,
                               void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLASHDEC_OPS_H */
