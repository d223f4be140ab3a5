/*
 * spinq.h -- C ABI of the GB300 (sm_103a) rotated W4A4 hot path of SpinQuant
 * (arXiv 2405.16406).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Pointers.  Every data pointer is a DEVICE pointer owned by the caller; the
 *   library never allocates, frees or keeps a pointer after the call returns.
 *   One exception: spinq_w4a4_gemm_noalloc keeps its workspace in a fixed
 *   device array of SPINQ_NOALLOC_SCRATCH_BYTES that the library owns (held
 *   by every GPU that loads the library until the process exits) and caches
 *   that array's device address per CUDA context.
 *   `stream` is a cudaStream_t (NULL = the legacy default stream).  Every
 *   call is asynchronous: it validates its arguments on the host, enqueues
 *   kernels on `stream` and returns; it never synchronizes.
 * Layouts.  Row-major, the reduction dimension K (or head_dim D) contiguous.
 *   4-bit codes are packed two per byte, the even index in the LOW nibble.
 *   Symmetric codes are two's complement nibbles in [-8, 7]; asymmetric codes
 *   are unsigned nibbles in [0, 15].  Scales and zeros are fp32.
 * Rotation.  A Hadamard spec {n_small, n_pow2} names R = (H_s (x) H_P)/sqrt(K)
 *   with K = n_small * n_pow2, H_P the natural-order Sylvester matrix of order
 *   n_pow2 and H_s the small factor of order n_small: [1] for n_small = 1, else
 *   the Paley I matrix of order n_small (n_small - 1 = q, a prime power with
 *   q = 3 mod 4; GF(q) = integers mod q for prime q, GF(27) =
 *   GF(3)[t]/(t^3 + 2t + 1) with element i = c0 + 3 c1 + 9 c2 <-> c0 + c1 t +
 *   c2 t^2; H_s = I + S, S = [[0, 1..1], [-1.., Q]], Q[i][j] = chi(a_i - a_j)).
 *   The small factor acts on the slow index (element k = i * n_pow2 + j) and
 *   activations are rotated as row vectors: x' = x R (Sec. 3.1, R3 and R4;
 *   Sec. 2.2 footnote for the Hadamard scaling).
 * Quantizer.  Eq. 1 (Sec. 2): symmetric alpha = clip * max|x| / (2^(N-1)-1),
 *   beta = 0, q = clamp(rint(x/alpha), -2^(N-1), 2^(N-1)-1); asymmetric
 *   alpha = clip * (max x - min x) / (2^N - 1), beta = clip * min x,
 *   u = clamp(rint((x - beta)/alpha), 0, 2^N - 1); a zero range stores
 *   alpha = 0 and codes 0.  rint is round-half-to-even.  The clipping ratio
 *   follows the appendix "Quantization choice".  Only N = 4 has kernels.
 * Errors.  Invalid arguments return SPINQ_EINVAL before any launch (NULL
 *   required pointer, non-positive or inconsistent size, K not even, a
 *   pointer not 16-byte aligned where noted, clip_ratio outside (0, 1]).
 *   A valid request with no compiled kernel (bits != 4, an unsupported
 *   Hadamard order or granularity) returns SPINQ_EUNSUPPORTED.  A failed
 *   launch returns SPINQ_ECUDA.  Device-side waits in the GEMM are bounded;
 *   a wait that gives up records SPINQ_ETIMEOUT in a device status word that
 *   spinq_device_status() reads back.
 */
#ifndef SPINQ_H_
#define SPINQ_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SPINQ_OK = 0,
  SPINQ_EINVAL = 1,
  SPINQ_EUNSUPPORTED = 2,
  SPINQ_ECUDA = 3,
  SPINQ_ETIMEOUT = 4,
  SPINQ_ESCRATCH = 5  /* spinq_w4a4_gemm_noalloc: the request needs more
                         workspace than its fixed array holds */
} spinq_status;

typedef enum {
  SPINQ_PER_TOKEN = 0,   /* one (alpha, beta) per row of activations      */
  SPINQ_PER_CHANNEL = 1, /* one scale per output channel (row) of weights */
  SPINQ_PER_GROUP = 2    /* one (alpha, beta) per group of group_size     */
} spinq_gran;

/* Quantizer of Eq. 1: bit width N, symmetric (1) or asymmetric (0),
 * granularity, group size (PER_GROUP only) and clipping ratio in (0, 1]. */
typedef struct {
  int32_t bits;
  int32_t symmetric;
  int32_t granularity;
  int32_t group_size;
  float clip_ratio;
} spinq_quant_cfg;

/* Online Hadamard of size n_small * n_pow2 (Sec. 3.1, R3/R4). */
typedef struct {
  int32_t n_small; /* 1, 12, 20 or 28 */
  int32_t n_pow2;  /* power of two, 1 .. 16384 */
} spinq_had_cfg;

/*
 * spinq_rotate_quant_act -- online rotation R4 fused with per-token 4-bit
 * activation quantization (Sec. 3.1 "Additional unabsorbed rotations" and
 * Eq. 1).  For each row m: x'_m = x_m R (skipped when had == NULL), then
 * Eq. 1 over the K values of x'_m with one (alpha_m, beta_m).  x' is kept in
 * fp32 and never stored.
 *   x_f16  [M][ldx] fp16, row m starts at x_f16 + m*ldx elements; 16-byte
 *          aligned rows (ldx % 8 == 0, pointer 16-byte aligned).
 *   had    NULL or a spec with n_small * n_pow2 == K.
 *   q      bits = 4, granularity = SPINQ_PER_TOKEN.
 *   codes  [M][K/2] packed codes (16-byte aligned).
 *   scale  [M] alpha_m.   zero [M] beta_m (asymmetric) or NULL (symmetric).
 * Supported K: 32 <= K <= 32768, K % 32 == 0 (with had: the spec's sizes).
 */
spinq_status spinq_rotate_quant_act(const void* x_f16, int64_t M, int64_t K, int64_t ldx,
                                    const spinq_had_cfg* had, const spinq_quant_cfg* q,
                                    uint8_t* codes, float* scale, float* zero, void* stream);

/*
 * spinq_quant_weight -- offline weight preparation: merge the rotation into
 * the weight (Sec. 3.1 rotational invariance: x' W'^T = x R R^T W^T = x W^T
 * with W' = W R, i.e. every output row rotated like an activation row), then
 * symmetric Eq. 1 per output channel (round-to-nearest, the RTN weight
 * quantizer of the appendix RTN-vs-GPTQ ablation), plus the integer row sum
 * of the codes that the GEMM epilogue needs.
 *   w_f16  [N][K] fp16 (16-byte aligned).   had NULL = no merge.
 *   q      bits = 4, symmetric = 1, granularity = SPINQ_PER_CHANNEL.
 *   codes  [N][K/2], scale [N] (s_n), rowsum [N] (sum_k q_nk).
 */
spinq_status spinq_quant_weight(const void* w_f16, int64_t N, int64_t K, const spinq_had_cfg* had,
                                const spinq_quant_cfg* q, uint8_t* codes, float* scale,
                                int32_t* rowsum, void* stream);

/*
 * Random-sign rotation (Sec. 2.2 footnote: a Hadamard matrix multiplied by a
 * random +-1 diagonal S is again a rotation, a "random Hadamard matrix"):
 * R = S (H_s (x) H_P) / sqrt(K), the signs acting on the input index k:
 * x' = (x S) (H_s (x) H_P) / sqrt(K), and W' = W S H / sqrt(K) for the merged
 * weights, so that x' W'^T = x W^T still holds.
 *   signs  device bit mask [K/8] bytes: bit (k % 8) of byte k / 8 set means
 *          s_k = -1.  Requires a Hadamard spec (had != NULL).
 * Other arguments as spinq_rotate_quant_act / spinq_quant_weight.
 */
spinq_status spinq_rotate_quant_act_signed(const void* x_f16, int64_t M, int64_t K, int64_t ldx,
                                           const spinq_had_cfg* had, const uint8_t* signs,
                                           const spinq_quant_cfg* q, uint8_t* codes, float* scale, float* zero,
                                           void* stream);
spinq_status spinq_quant_weight_signed(const void* w_f16, int64_t N, int64_t K, const spinq_had_cfg* had,
                                       const uint8_t* signs, const spinq_quant_cfg* q, uint8_t* codes,
                                       float* scale, int32_t* rowsum, void* stream);

/*
 * spinq_w4a4_gemm -- the W4A4 linear on Eq. 1 codes with an exact integer
 * accumulator and a fused per-token x per-channel dequantization epilogue.
 *   acc[m][n] = sum_k a_mk * q_nk, a = q (symmetric activations) or u - 8
 *               (asymmetric activations), exact in 32-bit integers;
 *   y[m][n]   = fp16( s_n * (alpha_m * acc[m][n] + beta'_m * rowsum_n) ),
 *               beta'_m = beta_m + 8 alpha_m (asymmetric) or 0 (symmetric),
 *   which equals sum_k (alpha_m c_mk + beta_m)(s_n q_nk), the product of the
 *   two dequantized operands of Eq. 1.
 *   a_codes [M][K/2], a_scale [M], a_zero [M] or NULL (symmetric);
 *   w_codes [N][K/2] symmetric, w_scale [N], w_rowsum [N];
 *   y_f16 [M][N] fp16; acc_out [M][N] int32 or NULL (debug output).
 *   Requirements: K % 128 == 0, N % 16 == 0, K <= 65536; code, output,
 *   w_scale and w_rowsum pointers 16-byte aligned.
 */
spinq_status spinq_w4a4_gemm(const uint8_t* a_codes, const float* a_scale, const float* a_zero,
                             const uint8_t* w_codes, const float* w_scale,
                             const int32_t* w_rowsum, int64_t M, int64_t N, int64_t K,
                             void* y_f16, int32_t* acc_out, void* stream);

/*
 * spinq_w4a4_gemm_workspace_bytes -- device workspace, in bytes, that
 * spinq_w4a4_gemm_splitk needs for an M x N x K call on the current CUDA
 * device: M*N*4 + 4*ceil(N/128) for the calls whose K range it splits across
 * CTAs (spinq_w4a4_gemm_splitk_plan), and 0 otherwise (those calls need no
 * workspace and may pass NULL).
 */
int64_t spinq_w4a4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);

/*
 * spinq_w4a4_gemm_splitk -- the same operation and outputs as
 * spinq_w4a4_gemm, for small M (decode, M <= 256), where the GEMM is bound by
 * streaming the weights from HBM.  Up to 4 tokens (M * K <= 160 KiB) it runs
 * the GEMV kernel: each warp owns whole output channels, streams their packed
 * weights from global memory and takes exact integer dot products (no
 * workspace).  Otherwise a cost model fitted on GB300 picks between the
 * split-K kernel and the kernels of spinq_w4a4_gemm.  In the split-K kernel
 * each CTA owns 128 output channels and a slice of K, so every SM streams a
 * disjoint part of the weights; the slices' exact integer partial
 * accumulators are summed in `workspace` and the last slice of each
 * 128-channel tile applies the epilogue (with a single slice the CTA writes
 * the outputs itself and no workspace is used).  For M > 256 the call runs
 * the same kernel as spinq_w4a4_gemm and does not touch `workspace`.
 *   workspace       device buffer of spinq_w4a4_gemm_workspace_bytes(M, N, K)
 *                   bytes, 16-byte aligned, all zero before the first call;
 *                   each completed call leaves it zero again.  Calls that may
 *                   overlap on the GPU need distinct workspaces.  After a call
 *                   that recorded SPINQ_ETIMEOUT, clear it again.
 *   workspace_bytes its size (SPINQ_EINVAL if smaller than required).
 * Other arguments and requirements as spinq_w4a4_gemm.
 */
spinq_status spinq_w4a4_gemm_splitk(const uint8_t* a_codes, const float* a_scale, const float* a_zero,
                                    const uint8_t* w_codes, const float* w_scale,
                                    const int32_t* w_rowsum, int64_t M, int64_t N, int64_t K,
                                    void* y_f16, int32_t* acc_out, void* workspace,
                                    int64_t workspace_bytes, void* stream);

/* Size of the fixed device array spinq_w4a4_gemm_noalloc works in (8 MiB). */
#define SPINQ_NOALLOC_SCRATCH_BYTES (8ll << 20)

/*
 * spinq_w4a4_gemm_noalloc -- spinq_w4a4_gemm_splitk for callers that cannot
 * allocate device memory where they run the layer: a serving runtime that
 * reserves its whole memory budget at start-up and forbids later
 * allocations, a thread that must not call into an allocator while other
 * streams are being captured into CUDA graphs, an embedder with no device
 * allocator of its own to hand a workspace from.  The paper has no
 * counterpart: this is an interface convenience, not part of the method.
 *   Same arguments, outputs and requirements as spinq_w4a4_gemm; no workspace
 *   argument.  The workspace lives in a fixed device array of
 *   SPINQ_NOALLOC_SCRATCH_BYTES owned by the library, which every GPU that
 *   loads the library holds until the process exits.
 *   A request whose plan needs more workspace than that
 *   (spinq_w4a4_gemm_workspace_bytes(M, N, K) > SPINQ_NOALLOC_SCRATCH_BYTES,
 *   e.g. split-K decode plans with M * N * 4 above 8 MiB) is refused with
 *   SPINQ_ESCRATCH before anything is enqueued; split the tokens into smaller
 *   calls.  Requests whose plan needs no workspace (the GEMV, the prefill
 *   kernels, unsliced tiles) always run.
 *   The call itself allocates nothing: no cudaMalloc/cudaFree and no
 *   allocating library routine.  It clears the part of the array it uses
 *   (cudaMemsetAsync on `stream`) before the kernel, since the array keeps
 *   the previous call's contents.
 *   The first call in each CUDA context looks up the array's device address
 *   (cudaGetSymbolAddress, with that device current) and caches it for that
 *   context; make that first call outside any stream capture.
 *   Every call shares the one array per device: calls that may overlap on the
 *   GPU (different streams without ordering between them) race on it.
 */
spinq_status spinq_w4a4_gemm_noalloc(const uint8_t* a_codes, const float* a_scale, const float* a_zero,
                                     const uint8_t* w_codes, const float* w_scale,
                                     const int32_t* w_rowsum, int64_t M, int64_t N, int64_t K,
                                     void* y_f16, int32_t* acc_out, void* stream);

/*
 * spinq_rotated_linear -- the down_proj of Sec. 3.1 in one call: the online
 * rotation R4 (optionally with random signs, as spinq_rotate_quant_act_signed)
 * fused with the per-token Eq. 1 quantizer, then the W4A4 GEMM on those codes
 * against weights merged with the same rotation (spinq_quant_weight[_signed]).
 * The two kernels run back to back on `stream` (the GEMM's prologue overlaps
 * the quantizer's tail) and hand the codes over in `workspace`, which stays
 * in L2 between them (14.7 MB for 2048 tokens of K = 14336).
 *   x_f16 [M][ldx], had, signs (NULL = none), q (activation quantizer, 4
 *   bits, per token) as spinq_rotate_quant_act(_signed); w_codes [N][K/2],
 *   w_scale [N], w_rowsum [N], y_f16 [M][N] as spinq_w4a4_gemm.
 *   workspace  device buffer of spinq_rotated_linear_workspace_bytes(M, K)
 *              bytes, 16-byte aligned: the codes and scales in flight.
 */
int64_t spinq_rotated_linear_workspace_bytes(int64_t M, int64_t K);
spinq_status spinq_rotated_linear(const void* x_f16, int64_t M, int64_t K, int64_t ldx, const spinq_had_cfg* had,
                                  const uint8_t* signs, const spinq_quant_cfg* q, const uint8_t* w_codes,
                                  const float* w_scale, const int32_t* w_rowsum, int64_t N, void* y_f16,
                                  void* workspace, int64_t workspace_bytes, void* stream);

/*
 * spinq_rotate_quant_kv -- R3 on Q and K over head_dim, then the 4-bit
 * KV-cache quantizer (Sec. 3.1: R3 is an online Hadamard inserted for low-bit
 * KV-cache quantization; appendix "Quantization choice": asymmetric).
 * R2 is assumed merged into W_v / W_o, so V is quantized without rotation.
 *   q_in  [B][S][Hq][D] fp16 -> q_out (same layout; may equal q_in):
 *         q_out = fp16(q_in R).
 *   k_in, v_in [B][S][Hkv][D] fp16.
 *   K' = k_in R; K' and V quantized with kvq (bits = 4, symmetric = 0,
 *         granularity = SPINQ_PER_GROUP, group_size = D) into
 *   k_codes, v_codes [B][S][Hkv][D/2]; k_scale, k_zero, v_scale, v_zero
 *         [B][S][Hkv] fp32.
 *   had   {1, D}.  Supported D: 64 or 128.  All pointers 16-byte aligned.
 */
spinq_status spinq_rotate_quant_kv(const void* q_in, void* q_out, const void* k_in,
                                   const void* v_in, int64_t B, int64_t S, int64_t Hq,
                                   int64_t Hkv, int64_t D, const spinq_had_cfg* had,
                                   const spinq_quant_cfg* kvq, uint8_t* k_codes, float* k_scale,
                                   float* k_zero, uint8_t* v_codes, float* v_scale,
                                   float* v_zero, void* stream);

/*
 * spinq_gemm_select_kernel -- which kernel spinq_w4a4_gemm (and
 * spinq_w4a4_gemm_splitk / _noalloc for M > 256) runs, process-wide:
 *   SPINQ_GEMM_AUTO     the built-in cost model picks (the default);
 *   SPINQ_GEMM_TILE128  one CTA per 128 x 256 output tile;
 *   SPINQ_GEMM_TILE256  one CTA per 256 x 256 output tile;
 *   SPINQ_GEMM_PAIR     two CTAs (an SM pair) per 256 x 256 tile; calls it
 *                       cannot serve (M <= 128, no pair resident) use AUTO;
 *   SPINQ_GEMM_GEMV     (M <= 4 with M * K <= 160 KiB; AUTO picks it there
 *                       unless SPINQ_GEMM_TCGEMV takes the tokens, on the
 *                       _splitk / _noalloc entry points too) each warp
 *                       owns whole output channels and streams their packed
 *                       weights; calls it cannot serve use AUTO;
 *   SPINQ_GEMM_SPLITK   the split-K kernel on the _splitk / _noalloc entry
 *                       points for every M <= 256 (GEMV and prefill kernels
 *                       excluded); spinq_w4a4_gemm treats it as AUTO;
 *   SPINQ_GEMM_TCGEMV   (M <= 16, on every entry point; AUTO picks it for 3 to
 *                       16 tokens when K / 128 = NKW W with NKW in {1, 2, 4,
 *                       8} and W <= 16, else for 5 to 8 tokens) the products
 *                       on the tensor core (fp16 m16n8k16 on the exact codes),
 *                       no workspace: for such K, one CTA per SM whose W
 *                       warps split K and stream the packed weights straight
 *                       into registers; else a CTA per 16 output channels
 *                       that stages them through shared memory; calls it
 *                       cannot serve use AUTO.
 * All kernels compute bit-identical outputs; this is a tuning and testing
 * control.  Returns the previous selection, or -1 (and changes nothing) for
 * an unknown value.  Not synchronized with GEMM calls in other threads.
 */
typedef enum {
  SPINQ_GEMM_AUTO = 0,
  SPINQ_GEMM_TILE128 = 1,
  SPINQ_GEMM_TILE256 = 2,
  SPINQ_GEMM_PAIR = 3,
  SPINQ_GEMM_GEMV = 4,
  SPINQ_GEMM_SPLITK = 5,
  SPINQ_GEMM_TCGEMV = 6
} spinq_gemm_kernel;

int spinq_gemm_select_kernel(int kernel);

/*
 * spinq_gemm_split_k -- process-wide number of K slices per 128-channel tile
 * of the split-K kernel: 1..64 fixes it (at most K / 128), 0 lets the cost
 * model pick (the default).  A tuning and testing control like
 * spinq_gemm_select_kernel; spinq_w4a4_gemm_workspace_bytes and
 * spinq_w4a4_gemm_splitk_plan follow it.  Returns the previous value, or -1
 * (and changes nothing) for a value out of range.
 */
int spinq_gemm_split_k(int n);

/*
 * spinq_w4a4_gemm_plan -- the kernel (SPINQ_GEMM_TILE128, _TILE256, _PAIR,
 * _GEMV or _TCGEMV) that spinq_w4a4_gemm runs for an M x N x K call on the current CUDA
 * device under the current selection; -1 for shapes the call rejects.
 * Launches nothing.
 */
int spinq_w4a4_gemm_plan(int64_t M, int64_t N, int64_t K);

/*
 * spinq_w4a4_gemm_splitk_plan -- the kernel that spinq_w4a4_gemm_splitk runs
 * for an M x N x K call given a workspace of spinq_w4a4_gemm_workspace_bytes
 * bytes: SPINQ_GEMM_SPLITK, with *nsplit (may be NULL) set to its number of K
 * slices per 128-channel tile (1: no slicing, no workspace), or the kernel
 * spinq_w4a4_gemm would run (*nsplit = 0).  -1 for shapes the call rejects.
 * Launches nothing.
 */
int spinq_w4a4_gemm_splitk_plan(int64_t M, int64_t N, int64_t K, int* nsplit);

/*
 * spinq_rope_rotate_quant_kv -- spinq_rotate_quant_kv with the rotary
 * position embedding applied to Q and K first, in the same kernel: for each
 * token at position p and i < D/2, with (cos, sin) of angle p theta_i taken
 * from the caller's table,
 *   x_i <- x_i cos - x_{i+D/2} sin,   x_{i+D/2} <- x_i sin + x_{i+D/2} cos
 * (the rotate-half form), computed in fp32 and rounded to fp16 like the
 * model's activations; then R3 (Sec. 3.1, the online Hadamard that follows
 * RoPE on Q and K) and the KV quantizer exactly as spinq_rotate_quant_kv.
 *   positions [B][S] int32, each in [0, max_pos) (others are clamped).
 *   cos_sin   [max_pos][D/2] pairs (cos, sin) as fp32, 16-byte aligned; the
 *             caller computes angle p theta_i, theta_i = base^(-2i/D),
 *             accurately (e.g. in double) once.
 * Other arguments, layouts and requirements as spinq_rotate_quant_kv.
 */
spinq_status spinq_rope_rotate_quant_kv(const void* q_in, void* q_out, const void* k_in, const void* v_in,
                                        const int32_t* positions, const float* cos_sin, int64_t max_pos, int64_t B,
                                        int64_t S, int64_t Hq, int64_t Hkv, int64_t D, const spinq_had_cfg* had,
                                        const spinq_quant_cfg* kvq, uint8_t* k_codes, float* k_scale,
                                        float* k_zero, uint8_t* v_codes, float* v_scale, float* v_zero,
                                        void* stream);

/*
 * spinq_decode_attention_kv4 -- attention of one decode query per (batch,
 * query head) over the 4-bit KV cache written by spinq_rotate_quant_kv (or
 * its RoPE form), the consumer of R3 (Sec. 3.1: R3 rotates Q and K over
 * head_dim so that Q K^T is unchanged while K quantizes to 4 bits):
 *   s_t = softmax_scale * q . k_t,  k_t = k_scale * u_t + k_zero,
 *   o   = sum_t softmax_t(s) v_t,     v_t = v_scale * u'_t + v_zero,
 * over t < lens[b]; query head h reads kv head h / (Hq / Hkv).
 *   q        [B][Hq][D] fp16, already rotated by R3 (the q_out of the call
 *            above for the decode token).
 *   k_codes, v_codes [B][S][Hkv][D/2], 16-byte aligned; k_scale, k_zero,
 *            v_scale, v_zero [B][S][Hkv] fp32 (S is the cache capacity: the
 *            row stride).
 *   lens     [B] int32 in [1, S] (device), or NULL for S everywhere.
 *   out      [B][Hq][D] fp16.
 *   workspace device buffer of spinq_decode_attention_workspace_bytes(B, S,
 *            Hq, Hkv, D) bytes, 16-byte aligned (the per-chunk partial
 *            results; no zeroing needed).
 *   Supported: D = 64 or 128, Hq / Hkv in {1, 2, 4, 8}, S * Hkv * D / 2 <
 *   2^31 (one batch's codes within 2 GiB).  Both products run
 *   on the tensor core with fp32 accumulation: q . u on the fp16 query and
 *   the exact codes, the value sum on the codes and fp16 weights
 *   p * v_scale / max(v_scale) (relative rounding 2^-11 per weight); the
 *   softmax and the scales in fp32.  Two kernels on `stream` (the chunks,
 *   then their merge).
 */
int64_t spinq_decode_attention_workspace_bytes(int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t D);
spinq_status spinq_decode_attention_kv4(const void* q, const uint8_t* k_codes, const float* k_scale,
                                        const float* k_zero, const uint8_t* v_codes, const float* v_scale,
                                        const float* v_zero, const int32_t* lens, int64_t B, int64_t S, int64_t Hq,
                                        int64_t Hkv, int64_t D, float softmax_scale, void* out, void* workspace,
                                        int64_t workspace_bytes, void* stream);

/*
 * The paged 4-bit cache.  K and V of a token lie in one slot of a page; a
 * page holds page_size tokens of every kv head, and a sequence is the list
 * of its pages (a row of a page table), in any order:
 *   k_codes, v_codes [num_pages][kv_heads][page_size][head_dim/2] packed Eq. 1
 *            codes, 16-byte aligned (K rotated by R3, as spinq_rotate_quant_kv
 *            stores it);
 *   scales   [num_pages][kv_heads][page_size][4] fp32, 16-byte aligned:
 *            (K alpha, K beta, V alpha, V beta) of the token and head, alpha >= 0
 *            (Eq. 1's step; a V alpha below 2^-40 counts as 2^-40 in attention).
 * Slot number s of the cache is slot s % page_size of page s / page_size.
 * page_size: 16, 32, 64, 128 or 256.  head_dim: 64 or 128.  A slot that no
 * call has written may hold anything (also values that are not finite): no
 * call's result depends on slots past a sequence's length.  A page number
 * outside [0, num_pages) reads no memory out of range; the values of its
 * tokens are undefined.
 */
typedef struct {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* scales;
  int64_t num_pages;
  int32_t page_size;
  int32_t kv_heads;
  int32_t head_dim;
} spinq_kv4_pages;

/* Rotary embedding of the first rotary_dim values of a head (Sec. 3.1: RoPE
 * precedes R3).  rotary_dim: 0 (none), D/4, D/2, 3D/4 or D.  Value pair i <
 * rotary_dim/2 turns by the angle of table entry [position][i]: values
 * (i, i + rotary_dim/2) (interleaved = 0) or (2i, 2i + 1) (interleaved = 1).
 *   positions [T] int32 in [0, max_pos) (others are clamped);
 *   cos_sin   [max_pos][rotary_dim/2] pairs (cos, sin) fp32, 16-byte aligned:
 *             scaling for long contexts is in the caller's table. */
typedef struct {
  int32_t rotary_dim;
  int32_t interleaved;
  const int32_t* positions;
  const float* cos_sin;
  int64_t max_pos;
} spinq_rope_cfg;

/*
 * spinq_kv4_append -- T new tokens on their way into attention, in one pass:
 * the norm of each query and key head, the rotary embedding, R3 and the 4-bit
 * quantizer (Sec. 3.1; Eq. 1), K and V written into their slots of the pages:
 *   x <- x w / sqrt(mean(x^2) + eps)  (queries with q_weight, keys with k_weight),
 *   x <- rotary embedding (rope != NULL),  x' = x H_D / sqrt(D)  (queries, keys),
 *   q_out = fp16(x'),  K codes = Eq. 1 of x',  V codes = Eq. 1 of v.
 * All of it in fp32 from the fp16 input to the code.
 *   q [T][Hq][D], k, v [T][kv_heads][D] fp16: a token's heads are contiguous,
 *          tokens ldq, ldk, ldv elements apart (parts of one projection's
 *          output, for instance), 16-byte aligned, ld % 8 == 0.
 *   q_out  [T][Hq][D] fp16 (may equal q when ldq = Hq D).  Hq may be 0.
 *   q_weight, k_weight  [D] fp16, 16-byte aligned, or NULL (no norm); eps >= 0.
 *   kvq    bits = 4, symmetric = 0, granularity = SPINQ_PER_GROUP, group_size = D.
 *   slots  [T] int64 slot numbers, distinct; a token whose number is outside
 *          the cache (e.g. -1, padding) is not written, its q_out is.
 *   A row with a value that is not a number is cached with NaN scales.  Codes are
 *   Eq. 1 in fp32; at the middle of two they may differ by one from those
 *   that spinq_rotate_quant_kv writes.
 *   Supported: T times the larger head count below 2^31.
 */
spinq_status spinq_kv4_append(const void* q, int64_t ldq, void* q_out, const void* k, int64_t ldk, const void* v,
                              int64_t ldv, int64_t T, int64_t Hq, const void* q_weight, const void* k_weight,
                              float eps, const spinq_rope_cfg* rope, const spinq_quant_cfg* kvq,
                              const spinq_kv4_pages* cache, const int64_t* slots, void* stream);

/*
 * spinq_kv4_read -- cached tokens expanded to fp16, packed: tokens starts[b],
 * starts[b] + 1, ... of sequence b at rows cu_tokens[b] .. cu_tokens[b+1] - 1 of
 *   k, v [total][kv_heads][D] fp16 = fp16(alpha u + beta)  (K still rotated by
 *        R3, as the rotated queries want it: what spinq_prompt_attention takes
 *        for the context of a prompt that arrives in chunks).
 *   page_table [batch][table_width] int32;  starts [batch] int32 or NULL (0);
 *   cu_tokens [batch + 1] int32 ascending from 0, cu_tokens[batch] = total.
 *   Tokens past the page table read as zeros.  total * kv_heads < 2^31.
 */
spinq_status spinq_kv4_read(const spinq_kv4_pages* cache, const int32_t* page_table, int64_t batch,
                            int64_t table_width, const int32_t* starts, const int32_t* cu_tokens, int64_t total,
                            void* k, void* v, void* stream);

/*
 * spinq_prompt_attention -- attention over whole prompts, packed, grouped heads:
 *   o_i = sum_j softmax_j(softmax_scale q_i . k_j) v_j
 * for query i of a sequence of lq queries and lk >= 0 keys; with causal = 1
 * over j <= i + lk - lq (the queries are the sequence's last positions), else
 * over all.  A query that sees no key gives zeros.  Query head h reads kv head
 * h / (Hq / Hkv).
 *   q [total_q][Hq][D], k, v [total_k][Hkv][D] fp16, tokens ldq, ldk, ldv
 *          elements apart as in spinq_kv4_append;  out [total_q][Hq][D] fp16,
 *          not overlapping the inputs.
 *   cu_q, cu_k [batch + 1] int32 (device), ascending from 0: sequence b has
 *          rows cu[b] .. cu[b+1] - 1 (rows of out after the last are not written;
 *          offsets outside [0, total] are clamped).
 *   max_q, max_k  no less than any sequence's lq and lk (host numbers; the
 *          launch is planned with max_q, max_k is only checked).
 *   workspace  spinq_prompt_attention_workspace_bytes(...) bytes: 0 for every
 *          argument, so that it may be NULL; what is given is not used.
 *   Keys and values of a sequence must be finite; rows of other sequences
 *   and rows outside every sequence never reach a result.
 *   Supported: D = 64 or 128, Hq / Hkv whole and at most 128.  Scores and sums
 *   in fp32, the softmax weights in fp16 for the product with V.
 */
int64_t spinq_prompt_attention_workspace_bytes(int64_t batch, int64_t max_q, int64_t max_k, int64_t Hq, int64_t Hkv,
                                               int64_t D);
spinq_status spinq_prompt_attention(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                    const int32_t* cu_q, const int32_t* cu_k, int64_t batch, int64_t total_q,
                                    int64_t total_k, int64_t max_q, int64_t max_k, int64_t Hq, int64_t Hkv, int64_t D,
                                    int32_t causal, float softmax_scale, void* out, void* workspace,
                                    int64_t workspace_bytes, void* stream);

/*
 * spinq_prefix_attention_kv4 -- attention of one decode query per (sequence,
 * query head) over the paged 4-bit cache, where the sequences share a prefix
 * (an instruction text, a document) that is read and multiplied once for all:
 * softmax over the prefix_len tokens of prefix_table, then the sequence's own
 * lens[b] tokens of page_table[b], K and V as in spinq_decode_attention_kv4.
 * A sequence without any token gives zeros; prefix_len may be 0.
 *   q, out [B][Hq][D] fp16, q rotated by R3 (spinq_kv4_append's q_out);
 *   prefix_table [ceil(prefix_len / page_size)] int32;
 *   page_table [B][table_width] int32, lens [B] int32 (device), each in
 *          [0, table_width * page_size] (others are clamped).
 *   workspace  spinq_prefix_attention_workspace_bytes(...) bytes, 16-byte
 *          aligned (no zeroing needed); 0 where the call refuses the sizes.
 *   Supported: Hq / kv_heads whole and at most 128, Hq and B at most 65535.
 *   Scores and sums in fp32.  For the product with V's codes the weights p
 *   alpha are fp16: one number for the prefix of more than floor(128 / (Hq /
 *   kv_heads)) sequences, two parts (2^-22) else and for the own tokens.  That
 *   limit and the parts that the prefix is split into depend on B, so a sequence's
 *   output may change in its last bits when the batch does.
 */
int64_t spinq_prefix_attention_workspace_bytes(int64_t B, int64_t prefix_len, int64_t table_width, int32_t page_size,
                                               int64_t Hq, int64_t Hkv, int64_t D);
spinq_status spinq_prefix_attention_kv4(const void* q, const spinq_kv4_pages* cache, const int32_t* prefix_table,
                                        int64_t prefix_len, const int32_t* page_table, int64_t table_width,
                                        const int32_t* lens, int64_t B, int64_t Hq, float softmax_scale, void* out,
                                        void* workspace, int64_t workspace_bytes, void* stream);

/*
 * spinq_kv4_plan -- the bookkeeping of one step of the paged cache, from the
 * requests' lengths: sequence b drops its last drop[b] tokens (all of them, where
 * it has no more), then add[b] tokens are to come behind the rest.  Pages that no
 * token is left on go back to the free pages, new tokens get theirs from there:
 *   start = max(lens[b] - drop[b], 0);  lens[b] <- start + add[b];
 *   token i of the sequence: row t = cu_tokens[b] + i, position
 *   start + i + position_offset, slot of token start + i of its row of page_table.
 * The free pages are a stack, free_pages[0 .. *free_count - 1], freed pages on
 * top in such order that a sequence which drops and adds gets its own back.
 * Sequences are served in their order; where the pages run out, the first that is
 * not to be had in full and every later one that needs a page are refused, as is one
 * longer than its row of page_table, one whose rows end past `total`, or one whose
 * new tokens would begin in a page that was given back (below): lens[b] <- start, its
 * slots are -1 (spinq_kv4_append passes over them), granted[b] = 0.  What later calls
 * of the step give for its rows means nothing, and none of its tokens is to be kept
 * (a count of 0 for spinq_kv4_keep).
 *   lens       [batch] int32, in and out (clamped to the row's capacity);
 *   drop, add  [batch] int32, or NULL (none); below 0 counts as 0;
 *   page_table [batch][table_width] int32, in and out: entries past a sequence's
 *              pages are left as they are.  Of its first ceil(lens[b] / page_size)
 *              entries one below 0 is no page: the program has given it back (put it on
 *              the list itself) after a window passed it, and nothing comes of it when its
 *              tokens are dropped.  Every other one is a page that neither the list nor
 *              another entry holds: what was given back must not stay in the table;
 *   free_pages [free_capacity] int32, free_count [1] int32, in and out; pages that
 *              the list has no room for are lost (no list as long as the cache is full);
 *   depths     [total] int32 or NULL: position start + depths[t] + position_offset
 *              in place of i (a drafted tree's nodes);
 *   cu_tokens  [batch + 1] int32 (at most total);  positions [total] int32, slots
 *              [total] int64: 0 and -1 in rows behind the last token;
 *   granted    [batch] int32 or NULL.
 *   All of it stays on the GPU, so a captured step replays with new lengths.
 *   Arrays must not overlap.  page_size 16, 32, 64, 128 or 256; batch at most 4096.
 */
spinq_status spinq_kv4_plan(int32_t* lens, const int32_t* drop, const int32_t* add, int64_t batch,
                            int32_t* page_table, int64_t table_width, int32_t page_size, int32_t* free_pages,
                            int32_t* free_count, int64_t free_capacity, const int32_t* depths,
                            int64_t position_offset, int64_t total, int32_t* cu_tokens, int32_t* positions,
                            int64_t* slots, int32_t* granted, void* stream);

/*
 * spinq_kv4_keep -- the accepted path of each drafted tree moves together: token
 * starts[b] + path[b][i] of sequence b is moved to starts[b] + i, i < counts[b],
 * codes and scales of K and V as they are (a node's rotation is that of its depth,
 * which is its place on the path).
 *   page_table [batch][table_width], starts, counts [batch], path
 *          [batch][path_width] int32 (device); counts are clamped to [0, path_width].
 *   A path ascends (path[b][i] >= i, each larger than the one before: a parent comes
 *   before its node); where one does not, which of its tokens arrive is not
 *   specified.  A token outside the page table or the cache is not moved.
 *   Supported: batch * kv_heads < 2^31.
 */
spinq_status spinq_kv4_keep(const spinq_kv4_pages* cache, const int32_t* page_table, int64_t batch,
                            int64_t table_width, const int32_t* starts, const int32_t* path, int64_t path_width,
                            const int32_t* counts, void* stream);

/*
 * spinq_window_prompt_attention -- spinq_prompt_attention (causal) where a query
 * sees the last positions and a few first tokens only: key j of a query at position
 * p = i + lk - lq is seen if j <= p and (p - j < window or j < sinks).
 *   window >= 1, sinks >= 0.  Other arguments, layouts and limits as
 *   spinq_prompt_attention (keys and values of a sequence are finite, those that no query
 *   sees among them).  A work item, two tiles of 128 rows (query x head of the group), reads
 *   the sinks in whole groups of 32 and the keys from the first that a window of its queries
 *   reaches.
 */
spinq_status spinq_window_prompt_attention(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                                           int64_t ldv, const int32_t* cu_q, const int32_t* cu_k, int64_t batch,
                                           int64_t total_q, int64_t total_k, int64_t max_q, int64_t max_k, int64_t Hq,
                                           int64_t Hkv, int64_t D, int64_t window, int64_t sinks, float softmax_scale,
                                           void* out, void* stream);

/*
 * spinq_tree_attention_kv4 -- attention of the last tokens of each sequence, a
 * drafted tree that is to be verified, over the paged 4-bit cache.  Sequence b has
 * lens[b] tokens in the cache, the last nq = cu_q[b+1] - cu_q[b] of them its
 * queries' own (appended before the call).  Query i sees the context (the tokens
 * before those nq), its ancestors, and itself:
 *   o_i = sum_j softmax_j(softmax_scale q_i . k_j) v_j,
 * K and V as in spinq_decode_attention_kv4.  With window >= 1 it sees only those of
 * them that are less than `window` positions before its own or below position
 * `sinks`; a context token's position is its place, a query's the context's length plus
 * its depth.  A query that sees no key (lens[b] below nq) gives zeros.
 *   q, out  [total_q][Hq][D] fp16, q rotated by R3 (spinq_kv4_append's q_out);
 *           rows of out behind the last sequence are not written;
 *   page_table [B][table_width] int32, lens [B] int32 (device), each in
 *           [0, table_width * page_size] (others are clamped); entries of pages that
 *           no query sees may be anything here (pages given back; for spinq_kv4_plan they
 *           are below 0);
 *   cu_q    [B + 1] int32 (device) ascending from 0;
 *   max_q   no less than any sequence's number of queries, at most 128;
 *   parents [total_q] int32: the number, within the sequence, of the query's parent,
 *           which comes before it; -1 (or any other number) for one that follows the
 *           context.  NULL: each query's parent is the one before it (a chain).
 *   window  0: none.
 *   workspace  spinq_tree_attention_workspace_bytes(...) bytes, 16-byte aligned (no
 *           zeroing needed); 0 where the call refuses the sizes.
 *   Supported: Hq / kv_heads whole and at most 128, Hq and B at most 65535.
 *   Scores and sums in fp32, the weights p alpha in two fp16 parts (2^-22).  How the
 *   keys are split over the GPU depends on max_q and the lengths of the whole batch, so a
 *   sequence's output may change in its last bits when those do; the same call gives the same
 *   bits every time.
 */
int64_t spinq_tree_attention_workspace_bytes(int64_t B, int64_t max_q, int64_t table_width, int32_t page_size,
                                             int64_t Hq, int64_t Hkv, int64_t D);
spinq_status spinq_tree_attention_kv4(const void* q, const spinq_kv4_pages* cache, const int32_t* page_table,
                                      int64_t table_width, const int32_t* lens, const int32_t* cu_q,
                                      const int32_t* parents, int64_t B, int64_t total_q, int64_t max_q, int64_t Hq,
                                      int64_t window, int64_t sinks, float softmax_scale, void* out, void* workspace,
                                      int64_t workspace_bytes, void* stream);

/*
 * spinq_window_attention_kv4 -- decode attention of one query per (sequence, query
 * head), the sequence's last token, over the last `window` of its lens[b] tokens and
 * the first `sinks` of the paged 4-bit cache (window 0: all of them).
 *   q, out  [B][Hq][D] fp16, q rotated by R3.  A sequence without tokens gives zeros.
 *   workspace  spinq_tree_attention_workspace_bytes(B, 1, ...) bytes.
 *   Other arguments, limits and arithmetic as spinq_tree_attention_kv4.
 */
spinq_status spinq_window_attention_kv4(const void* q, const spinq_kv4_pages* cache, const int32_t* page_table,
                                        int64_t table_width, const int32_t* lens, int64_t B, int64_t Hq,
                                        int64_t window, int64_t sinks, float softmax_scale, void* out,
                                        void* workspace, int64_t workspace_bytes, void* stream);

/*
 * 8-bit variants (main results table, W4A8 rows "4-8-x"; appendix "Latency
 * measurement on GPU": W-fp8-A-fp8 with the dequantization fused into the
 * GEMM epilogue).  They share the rotation convention above and run on the
 * E4M3 tensor-core pipe without unpacking.
 *
 * Code formats:
 *   SPINQ_FMT_INT8_PLANES  Eq. 1 with N = 8 per token: the code c = q
 *       (symmetric, [-128, 127]) or u - 128 (asymmetric, u in [0, 255]) is
 *       stored as two E4M3 planes, row [2K] bytes: byte k = E4M3(16 (c >> 4)),
 *       byte K + k = E4M3(c & 15) (both exact), so c = dec(k) + dec(K + k).
 *   SPINQ_FMT_E4M3         per-row FP8: alpha = clip max|x'| / 448, code =
 *       E4M3(x' / alpha), round to nearest even, saturating at +-448
 *       (E4M3: 1 sign, 4 exponent bits with bias 7, 3 mantissa bits, no
 *       infinities), [K] bytes per row.
 *   SPINQ_FMT_INT4_BYTES   (weights of the W4A8 linear) Eq. 1 with N = 4,
 *       symmetric per output channel, each code q in [-8, 7] stored as the
 *       E4M3 byte of q, [K] bytes per row, plus rowsum = sum_k q.
 */
typedef enum {
  SPINQ_FMT_INT8_PLANES = 1,
  SPINQ_FMT_E4M3 = 2,
  SPINQ_FMT_INT4_BYTES = 3
} spinq_code_format;

/*
 * spinq_rotate_quant_act8 -- online rotation (as spinq_rotate_quant_act)
 * then the 8-bit per-token quantizer `format`:
 *   SPINQ_FMT_INT8_PLANES  q: bits = 8, symmetric or asymmetric; codes
 *                          [M][2K]; scale [M]; zero [M] (asymmetric) or NULL.
 *   SPINQ_FMT_E4M3         q: bits = 8, symmetric = 1; codes [M][K]; scale [M].
 *   q->granularity = SPINQ_PER_TOKEN.  K % 128 == 0, K <= 32768, x rows and
 *   codes 16-byte aligned.  Other formats return SPINQ_EINVAL.
 */
spinq_status spinq_rotate_quant_act8(const void* x_f16, int64_t M, int64_t K, int64_t ldx,
                                     const spinq_had_cfg* had, const spinq_quant_cfg* q, int32_t format,
                                     uint8_t* codes, float* scale, float* zero, void* stream);

/*
 * spinq_quant_weight8 -- offline weight preparation of the 8-bit linears:
 * W' = W R (when had != NULL), then per output channel
 *   SPINQ_FMT_E4M3        q: bits = 8, symmetric; codes [N][K]; scale [N];
 *                         rowsum unused (may be NULL);
 *   SPINQ_FMT_INT4_BYTES  q: bits = 4, symmetric; codes [N][K]; scale [N];
 *                         rowsum [N].
 *   q->granularity = SPINQ_PER_CHANNEL; sizes as spinq_rotate_quant_act8.
 */
spinq_status spinq_quant_weight8(const void* w_f16, int64_t N, int64_t K, const spinq_had_cfg* had,
                                 const spinq_quant_cfg* q, int32_t format, uint8_t* codes, float* scale,
                                 int32_t* rowsum, void* stream);

/*
 * spinq_fp8_gemm -- W-fp8-A-fp8 linear:
 *   y[m][n] = fp16(alpha_m s_n sum_k a_mk w_nk), a, w decoded E4M3 codes,
 * products exact and summed in fp32 on the tensor core.
 *   a_codes [M][K] (SPINQ_FMT_E4M3), a_scale [M]; w_codes [N][K], w_scale [N].
 *   K % 128 == 0, K <= 65536, N % 16 == 0; code and output pointers 16-byte
 *   aligned.
 */
spinq_status spinq_fp8_gemm(const uint8_t* a_codes, const float* a_scale, const uint8_t* w_codes,
                            const float* w_scale, int64_t M, int64_t N, int64_t K, void* y_f16, void* stream);

/*
 * spinq_w4a8_gemm -- W4A8 linear on Eq. 1 codes, exact integer accumulator:
 *   acc[m][n] = sum_k c_mk q_nk (c = q or u - 128, exact in fp32: every
 *               partial sum is an integer of magnitude <= 1024 K <= 2^24);
 *   y[m][n]   = fp16(s_n (alpha_m acc + beta'_m rowsum_n)),
 *               beta'_m = beta_m + 128 alpha_m (asymmetric) or 0,
 *   the dequantized product of the two Eq. 1 operands.
 *   a_planes [M][2K] (SPINQ_FMT_INT8_PLANES), a_scale [M], a_zero [M] or NULL;
 *   w_codes [N][K] (SPINQ_FMT_INT4_BYTES), w_scale [N], w_rowsum [N];
 *   acc_out [M][N] int32 or NULL (debug).
 *   K % 128 == 0, K <= 16384, N % 16 == 0; code and output pointers 16-byte
 *   aligned.
 */
spinq_status spinq_w4a8_gemm(const uint8_t* a_planes, const float* a_scale, const float* a_zero,
                             const uint8_t* w_codes, const float* w_scale, const int32_t* w_rowsum, int64_t M,
                             int64_t N, int64_t K, void* y_f16, int32_t* acc_out, void* stream);

/*
 * spinq_cayley_step -- one Cayley SGD update of a batch of rotations
 * (Sec. 3.2, the R' update and its Y / G_hat definitions), for learning R2
 * (head_dim x head_dim, one per layer) with the weights frozen:
 *   G_hat = G R^T - 1/2 R R^T G R^T,   Y = G_hat - G_hat^T,
 *   R'    = (I - alpha/2 Y)^-1 (I + alpha/2 Y) R,
 * computed, as the paper does, by the fixed-point iteration of Cayley SGD:
 *   R'_0 = R + alpha Y R,   R'_{k+1} = R + (alpha/2) Y (R + R'_k),
 *   k = 0 .. iters-1 (it converges to R' when |alpha Y / 2| < 1).
 * G is the NEGATIVE of the loss gradient `grad` passed here: the objective
 * is an argmin and the cited Cayley SGD forms G_hat from the negative
 * gradient (with G = +grad the printed update would climb the loss).
 *   R      [batch][n][n] fp32 row-major, each orthonormal (device).
 *   grad   [batch][n][n] fp32, dL/dR (device).
 *   alpha  learning rate (finite); iters in 0 .. 64.
 *   R_out  [batch][n][n] fp32; may be R itself (in-place update), must not
 *          overlap R or grad otherwise.
 *   Y_out  [batch][n][n] fp32 or NULL: the skew-symmetric Y of each update.
 *   Supported n: 16, 32, 64, 128.  Pointers 16-byte aligned.  Arithmetic in
 *   fp32 (the oracle works in double).
 */
spinq_status spinq_cayley_step(const float* R, const float* grad, int64_t batch, int64_t n, float alpha,
                               int32_t iters, float* R_out, float* Y_out, void* stream);

/*
 * Testing controls of the failure paths (the paper has no counterpart).
 * spinq_debug_set_wait_limit_ns -- time limit of the ordinary bounded waits
 *   of the Paley rotate+quant, W4A4, FP8 GEMM and prompt and prefix attention
 *   kernels on the current device (2e9 ns by default; the drains of copies and MMAs in flight keep
 *   their full limit).  A test lowers it so that those waits give up, checks
 *   SPINQ_ETIMEOUT through spinq_device_status and sets it back.  Outputs of
 *   a call that gave up are undefined.  SPINQ_EINVAL for ns <= 0.
 * spinq_debug_stall_launches -- the next n launches of the Paley rotate+quant,
 *   the W4A4 prefill (128- and 256-row tiles), the FP8 GEMM and the prompt
 *   and prefix attention kernels issue no input copies, so the waits of their consumers run out of time (a
 *   barrier that nothing completes): SPINQ_ETIMEOUT is recorded, every role
 *   leaves its loop, MMAs in flight are drained and tensor memory is freed.
 *   Lower the wait limit first so that this takes a millisecond, not 2 s.
 *   Outputs of such a call are undefined.  Returns the previous count, or -1
 *   for n < 0.
 * spinq_debug_fail_launches -- the next n kernel launches of the library are
 *   refused on the host (the call returns SPINQ_ECUDA; nothing reaches the
 *   GPU).  Returns the previous count, or -1 for n < 0.
 */
spinq_status spinq_debug_set_wait_limit_ns(int64_t ns);
int spinq_debug_stall_launches(int n);
int spinq_debug_fail_launches(int n);

/* Human-readable name of a status code (static storage). */
const char* spinq_status_string(spinq_status s);

/*
 * spinq_device_status -- read and clear the device status word that bounded
 * waits in the kernels write when they give up (SPINQ_ETIMEOUT), for the
 * current CUDA device.  Synchronizes the device.  Returns SPINQ_OK when no
 * kernel recorded an error since the last call, SPINQ_ECUDA if the read
 * itself failed.  `detail` (may be NULL) receives the recorded site code.
 */
spinq_status spinq_device_status(int32_t* detail);

/* Library build identifier (static storage). */
const char* spinq_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SPINQ_H_ */
