/*
 * scope.h -- C ABI of the SCOPE sparse self-attention layer for video DiTs,
 * for AMD Instinct MI355X (gfx950).
 *
 * The layer (one attention head at a fixed layer and denoising step; heads
 * are independent and batched) takes post-3D-RoPE queries and keys Q, K and
 * values V, each N x d, and computes
 *   1. a k-means clustering of the queries in the full d-dim space   (Sec. 3.2, Eq. 2)
 *   2. a k-means clustering of each RoPE key subspace T, H, W and the
 *      composite code of every key                                   (Sec. 3.3, Eq. 3-4)
 *   3. score tables P_m = Qbar^m (U^m)^T and lookup-and-sum proxy
 *      logits for every (query cluster, key)                         (Eq. 5-6, Alg. 2)
 *   4. hybrid Top-p / fixed Top-k counts, the online per-head Top-k
 *      and each cluster's final key set                              (Eq. 7-10, Alg. 3)
 *   5. exact attention of each query cluster over its key set        (Eq. 11, Alg. 1)
 * Calls 1-5 below map one-to-one onto these stages.
 *
 * Conventions shared by every call
 * --------------------------------
 *  - Every array argument is a DEVICE pointer owned by the caller.  Scalars
 *    and the shape/size structs are host values.  The library allocates and
 *    frees nothing.  Its only global state belongs to the no-allocation
 *    attention call (5n): a fixed device array per GPU and a host table of
 *    their addresses.
 *  - Every call is asynchronous: it validates its arguments on the host,
 *    enqueues its kernels on `stream` (a hipStream_t; NULL = the default
 *    stream) and returns.  No call synchronises or copies to the host.
 *  - Layout: Q, K, V, O are [heads][n][d], d contiguous, in the dtype of the
 *    shape (fp32 or bf16); calls 9 to 11 take strides of heads and rows.  All
 *    other arrays are dense, row-major, with the shapes given per argument,
 *    heads outermost.
 *  - Workspace: calls that need scratch take `workspace` (256-byte aligned)
 *    of at least scope_workspace_size() bytes, calls 6 and 7 of at least
 *    scope_training_workspace_size(), calls 10 and 11 of at least
 *    scope_packed_workspace_size().  One workspace serves every call, but
 *    two calls that may run concurrently (replays of captured graphs among
 *    them) need two workspaces.  Nothing in it outlives its call.
 *  - Errors: argument checks run before any GPU work and return
 *    SCOPE_ERR_INVALID_ARGUMENT (bad value), SCOPE_ERR_UNSUPPORTED (valid but
 *    outside what the kernels implement) or SCOPE_ERR_WORKSPACE; nothing is
 *    enqueued then.  A failed kernel launch returns SCOPE_ERR_HIP.  Faults
 *    that depend on data are OR-ed into the optional device word
 *    `dev_status` (bit 0: non-finite input; bit 1: |x| >= 2^e with
 *    e = min(22, 39 - ceil(log2 n)), outside the range in which the int64
 *    fixed-point sums of the k-means means are exact (2^22 for n <= 2^17,
 *    2^15 at n = 2^24), also set for non-finite input; bit 2: an initial
 *    row index out of range, replaced by the default row; bit 3: a key set
 *    that is not strictly ascending in [0, n), call 7; bit 4: offsets or
 *    lengths of sequences that fall or leave their array, calls 10 and 11).
 *    The inputs are checked in the first update pass of calls 1 and 2.
 *    Nothing aborts or prints.
 *  - Determinism: every output is bitwise reproducible run to run and
 *    independent of launch geometry (calls 6, 7, 10, 11: see there); calls 1-4 are
 *    bit-exact with respect to the canonical arithmetic defined under each call.
 */
#ifndef SCOPE_H
#define SCOPE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SCOPE_ABI_VERSION 2

typedef enum {
  SCOPE_OK = 0,
  SCOPE_ERR_INVALID_ARGUMENT = 1,
  SCOPE_ERR_UNSUPPORTED = 2,
  SCOPE_ERR_WORKSPACE = 3,
  SCOPE_ERR_HIP = 4,
  SCOPE_ERR_SCRATCH_LIMIT = 5 /* beyond the no-allocation entry point's list */
} scope_status;

typedef enum { SCOPE_F32 = 0, SCOPE_BF16 = 1 } scope_dtype;

/* Selection policies (call 4b): the online per-head Top-k of Eq. 9-10, and
 * the two variants it is compared with in Fig. 6. */
typedef enum {
  SCOPE_POLICY_ONLINE = 0, /* r_c = max(b_c, k_head)              (Eq. 10) */
  SCOPE_POLICY_FIXED = 1,  /* r_c = b_c = max(t_c, k_fix), no top-up      */
  SCOPE_POLICY_TOPP = 2    /* r_c = t_c, pure Top-p                       */
} scope_policy;

/* Problem shape.  The three RoPE channel ranges I_T, I_H, I_W (Sec. 3.3;
 * App. A: disjoint, covering all d channels) are given as (offset, length)
 * in T, H, W order.  Supported: 1 <= heads <= 65535, 1 <= n <= 2^24, 2 <= d <= 128
 * for clustering/scoring/selection, d in {64, 128} for attention.         */
typedef struct {
  int32_t heads;
  int32_t n;
  int32_t d;
  int32_t dtype; /* scope_dtype of Q, K, V and O */
  int32_t range_off[3];
  int32_t range_len[3];
} scope_shape;

/* A general key partition (App. B; the partition ablation of Table 3): the
 * d channels split into M disjoint sets I_1 .. I_M that together cover all
 * of them, subspace m clustered into c[m] centroids.  `channels` lists I_1,
 * then I_2, ... (len[0] + ... + len[M-1] = d entries), each set in strictly
 * ascending channel order; entries past d are ignored.  The three RoPE
 * ranges in T, H, W order give exactly the results of calls 2-4.
 * Supported: 1 <= M <= 8, 1 <= c[m] <= min(n, 1024), c[0] + ... + c[M-1]
 * <= 3072 (one table row of a cluster is staged on chip during selection). */
#define SCOPE_MAX_SUBSPACES 8
#define SCOPE_MAX_D 128
typedef struct {
  int32_t m;
  int32_t c[SCOPE_MAX_SUBSPACES];
  int32_t len[SCOPE_MAX_SUBSPACES];
  int32_t channels[SCOPE_MAX_D];
} scope_partition;

int32_t scope_abi_version(void);
const char *scope_status_string(int32_t status);

/* Workspace bytes that suffice for every call below with these sizes.     */
int32_t scope_workspace_size(const scope_shape *shape, int32_t c_q,
                             const int32_t c_m[3], size_t *bytes);

/* 1. Query clustering (Sec. 3.2, Eq. 2; Alg. 1 first step).
 * Lloyd k-means of each head's n query rows into c_q clusters, `iters`
 * iterations of (assign, update), starting from rows init_idx[h][0..c_q)
 * (distinct rows in [0, n); NULL selects row floor((2r+1) n / (2 c_q))).
 * Canonical arithmetic: assign = argmin_r fl(||u_r||^2 - 2<x,u_r>) with
 * every dot product an fp32 fma chain in ascending channel order and ties
 * to the lowest r; update = exact int64 sums of rint(x * 2^24) over the
 * members, one fp64 division by count * 2^24, rounded to fp32; an empty
 * cluster keeps its centroid.  The iteration ends on an update, so each
 * returned centroid is the mean of its returned members (Eq. 2).
 * Outputs: q_centroids [heads][c_q][d] fp32; assign g [heads][n];
 * counts n_c [heads][c_q]; offsets [heads][c_q+1] (exclusive prefix sum of
 * counts); perm [heads][n] = the members of each cluster in ascending token
 * order, cluster after cluster (the query permutation of Alg. 1).
 * Requires 1 <= c_q <= min(n, 1024), 1 <= iters.                           */
int32_t scope_cluster_queries(const scope_shape *shape, const void *q,
                              int32_t c_q, int32_t iters,
                              const int32_t *init_idx, float *q_centroids,
                              int32_t *assign, int32_t *counts,
                              int32_t *offsets, int32_t *perm,
                              void *workspace, size_t ws_bytes,
                              int32_t *dev_status, void *stream);

/* 2. Key subspace clustering (Sec. 3.3, Eq. 3-4; Alg. 2 k-means step).
 * For m = T, H, W: k-means of K[:, I_m] into c_m[m] centroids with the same
 * canonical arithmetic as call 1, from rows init_idx[h][m][0..c_m[m])
 * (row stride init_stride >= max c_m; NULL = default rows), `iters`
 * iterations followed by one more assignment, so every code is the exact
 * argmin against the returned codebook (Eq. 3).
 * Outputs: k_centroids [heads][sum_m c_m*len_m] fp32, per head U^T, U^H,
 * U^W back to back, each [c_m][len_m]; codes [heads][n] composite code
 * z_T | z_H << 10 | z_W << 20 (Eq. 4).  Requires 1 <= c_m <= min(n, 1024). */
int32_t scope_cluster_key_subspaces(const scope_shape *shape, const void *k,
                                    const int32_t c_m[3], int32_t iters,
                                    const int32_t *init_idx,
                                    int32_t init_stride, float *k_centroids,
                                    uint32_t *codes, void *workspace,
                                    size_t ws_bytes, int32_t *dev_status,
                                    void *stream);

/* 1w, 2w. Warm starts across denoising steps (Sec. 4 setup: SCOPE runs at
 * every step after a dense prefix, and the query and key distributions of
 * one head change little from step to step).  As calls 1 and 2, but Lloyd's
 * iterations start from the centroids already in q_centroids (call 1w) or
 * k_centroids (call 2w), e.g. the previous step's results, instead of the
 * rows init_idx; those buffers are read, then overwritten with the result.
 * Arguments, layouts, outputs and errors otherwise as calls 1 and 2 (no
 * init_idx; the starting centroids must be finite).  With the centroids a
 * call returned, iters more iterations from them give exactly what a
 * single call with the total iteration count gives.                      */
int32_t scope_cluster_queries_warm(const scope_shape *shape, const void *q,
                                   int32_t c_q, int32_t iters,
                                   float *q_centroids, int32_t *assign,
                                   int32_t *counts, int32_t *offsets,
                                   int32_t *perm, void *workspace,
                                   size_t ws_bytes, int32_t *dev_status,
                                   void *stream);
int32_t scope_cluster_key_subspaces_warm(const scope_shape *shape,
                                         const void *k, const int32_t c_m[3],
                                         int32_t iters, float *k_centroids,
                                         uint32_t *codes, void *workspace,
                                         size_t ws_bytes, int32_t *dev_status,
                                         void *stream);

/* 3. Score tables and proxy logits (Eq. 5-6; Alg. 2 scoring steps).
 * tables [heads][c_q][C_T+C_H+C_W]: P_m[c][r] = <qbar_c[I_m], u_r^m> as an
 * fp32 fma chain over the subspace channels in ascending order, columns
 * T then H then W.  If `scores` is not NULL it receives the proxy logits
 * [heads][c_q][n]: s_cj = fl(fl(fl(P_T[c][zT] + P_H[c][zH]) + P_W[c][zW])
 * * fl32(1/sqrt(d))) + 0.0 (the + 0 maps -0 to +0).  scope_select computes
 * the same logits on the fly, so `scores` is only needed for inspection.   */
int32_t scope_proxy_scores(const scope_shape *shape, const float *q_centroids,
                           int32_t c_q, const float *k_centroids,
                           const int32_t c_m[3], const uint32_t *codes,
                           float *tables, float *scores, void *stream);

/* 4. Key selection (Eq. 7-10; Alg. 3).
 * Logits come from `scores` if not NULL, else from (tables, codes) exactly
 * as in call 3.  For each cluster c, with pi_c = keys by logit descending,
 * ties by ascending key index:
 *   t_c   = the shortest prefix of pi_c whose softmax mass reaches rho
 *           (Eq. 7), rho >= 1 keeps all n; the softmax mass of key j is
 *           E_j = fixexp(s_cj - max_j s_cj), an integer in units of 2^-32
 *           (z = y*fl32(log2 e); 0 below z = -40; 2^frac(z) by a degree-7
 *           Taylor polynomial in fp32), and the prefix must reach
 *           ceil(rho * sum_j E_j) computed exactly;
 *   b_c   = max(t_c, k_fix)                                         (Eq. 8)
 *   k_head= ceil(sum_c n_c b_c / sum_c n_c), exact integers         (Eq. 9)
 *   r_c   = max(b_c, k_head), S_c = the first r_c keys of pi_c      (Eq. 10)
 * Outputs: base_counts b [heads][c_q]; topp_counts t [heads][c_q] (may be
 * NULL); k_head [heads]; sel_counts r [heads][c_q]; sel_idx
 * [heads][c_q][n]: S_c in ascending key order in the first r_c entries
 * (the rest are left untouched).  counts are the n_c of call 1.
 * Requires 0 < rho <= 1 (finite) and 1 <= k_fix <= n.                      */
int32_t scope_select(const scope_shape *shape, int32_t c_q,
                     const int32_t c_m[3], const float *scores,
                     const float *tables, const uint32_t *codes,
                     const int32_t *counts, float rho, int32_t k_fix,
                     int32_t *base_counts, int32_t *topp_counts,
                     int32_t *k_head, int32_t *sel_counts, int32_t *sel_idx,
                     void *workspace, size_t ws_bytes, void *stream);

/* 4b. Selection under a named policy (the ablation of Fig. 6).  Arguments,
 * layouts, outputs and errors as call 4, plus `policy` (a scope_policy):
 * ONLINE is call 4; FIXED keeps b_c keys per cluster (Eq. 8) and TOPP the
 * t_c keys of Eq. 7, with no top-up to k_head.  k_head (Eq. 9) is written
 * for every policy.  An unknown policy is SCOPE_ERR_INVALID_ARGUMENT.     */
int32_t scope_select_policy(const scope_shape *shape, int32_t c_q,
                            const int32_t c_m[3], const float *scores,
                            const float *tables, const uint32_t *codes,
                            const int32_t *counts, float rho, int32_t k_fix,
                            int32_t *base_counts, int32_t *topp_counts,
                            int32_t *k_head, int32_t *sel_counts,
                            int32_t *sel_idx, void *workspace, size_t ws_bytes,
                            int32_t policy, void *stream);

/* 2p-4p. Calls 2-4 for a general key partition (App. B; Table 3).  The
 * shape's range fields are ignored (checked only by calls 2-4); `part`
 * (host memory) gives the sets and codebook sizes.  Errors as calls 2-4, and
 * SCOPE_ERR_INVALID_ARGUMENT for sets that are not a partition of the d
 * channels or not ascending, SCOPE_ERR_UNSUPPORTED beyond the limits above.
 *
 * Workspace bytes that suffice for the three partition calls and for calls 1
 * and 5 with these sizes.  When the sets are not the contiguous ranges
 * [0, len[0]), [len[0], len[0] + len[1]), ... this includes a channel-
 * reordered copy of K (heads * n * d elements).                            */
int32_t scope_partition_workspace_size(const scope_shape *shape, int32_t c_q,
                                       const scope_partition *part,
                                       size_t *bytes);

/* Key subspace clustering over the sets of `part`: for each m, k-means of
 * K[:, I_m] (the channels of I_m in ascending order) into c[m] centroids,
 * exactly as call 2 (same arithmetic, iterations plus one last assignment).
 * init_idx[(h * M + m) * init_stride + r] are the starting rows (NULL =
 * default rows), init_stride >= max c[m].
 * Outputs: k_centroids [heads][sum_m c[m] * len[m]] fp32, per head U^1 ..
 * U^M back to back, each [c[m]][len[m]] with column k on channel I_m[k];
 * codes [heads][M][n] uint16, z^m of key j at codes[(h * M + m) * n + j].  */
int32_t scope_cluster_key_partition(const scope_shape *shape, const void *k,
                                    const scope_partition *part, int32_t iters,
                                    const int32_t *init_idx,
                                    int32_t init_stride, float *k_centroids,
                                    uint16_t *codes, void *workspace,
                                    size_t ws_bytes, int32_t *dev_status,
                                    void *stream);

/* Tables and proxy logits over the sets of `part` (Eq. 5-6): tables
 * [heads][c_q][c[0] + ... + c[M-1]], P_m[c][r] = <qbar_c[I_m], u_r^m> as an
 * fp32 fma chain over I_m in ascending channel order; if `scores` is not
 * NULL, s_cj = fl(fl(...fl(P_1[z^1] + P_2[z^2]) ... + P_M[z^M]) *
 * fl32(1/sqrt(d))) + 0.0, summed left to right (M = 1: no addition).
 * Uses the workspace when the sets are not contiguous ranges in order.    */
int32_t scope_proxy_scores_partition(const scope_shape *shape,
                                     const float *q_centroids, int32_t c_q,
                                     const float *k_centroids,
                                     const scope_partition *part,
                                     const uint16_t *codes, float *tables,
                                     float *scores, void *workspace,
                                     size_t ws_bytes, void *stream);

/* Selection (call 4b) with the logits of `part`: from `scores` if not
 * NULL, else from (tables, codes) exactly as scope_proxy_scores_partition
 * computes them.  Arguments, outputs and errors otherwise as call 4b.  With
 * heads * n words more workspace than that call needs, which
 * scope_partition_workspace_size covers, codes of up to three subspaces are
 * packed first (the same results, faster).                                 */
int32_t scope_select_partition(const scope_shape *shape, int32_t c_q,
                               const scope_partition *part,
                               const float *scores, const float *tables,
                               const uint16_t *codes, const int32_t *counts,
                               float rho, int32_t k_fix, int32_t *base_counts,
                               int32_t *topp_counts, int32_t *k_head,
                               int32_t *sel_counts, int32_t *sel_idx,
                               void *workspace, size_t ws_bytes, int32_t policy,
                               void *stream);

/* 5. Sparse attention over the selected keys (Eq. 11; Alg. 1 last step).
 * For every cluster c and every query i in perm[offsets[c] .. offsets[c+1]):
 *   O[i] = softmax(q_i K[S_c]^T * scale) V[S_c],  S_c = sel_idx[c][0..r_c),
 * with the original Q, K, V rows (scale <= 0 selects 1/sqrt(d)).  Products
 * run on bf16 matrix cores with fp32 accumulation and an fp32 online
 * softmax; fp32 inputs are rounded to bf16 on load; O is written in the
 * input dtype, in original token order.  A cluster with r_c = 0 writes 0.
 * Dense attention (Eq. 1) is the special case of one cluster holding all
 * queries (c_q = 1, offsets = {0, n}, perm = identity) and all keys.
 * Bad indices cannot fault: index arrays are clamped to their valid
 * ranges on the device, or read through range-checked loads that return
 * 0 (the selected-key gather from bf16 K and V, copies among them).
 * Requires d in {64, 128}, 16-byte aligned q, k, v, o, and for bf16 inputs
 * n * d * 2 < 2^32 (n < 2^24 at d = 128), else SCOPE_ERR_UNSUPPORTED.
 * The call needs workspace for its work list only: heads * (ceil(n / 256) +
 * c_q) slots of 32 bytes, rounded up to 256.  With scope_workspace_size bytes
 * it also keeps bf16 copies of fp32 K and V and a block order, and is faster;
 * the results are the same bit for bit.                                    */
int32_t scope_sparse_attention(const scope_shape *shape, const void *q,
                               const void *k, const void *v, int32_t c_q,
                               const int32_t *offsets, const int32_t *perm,
                               const int32_t *sel_counts,
                               const int32_t *sel_idx, float scale, void *o,
                               void *workspace, size_t ws_bytes, void *stream);

/* 5n. Sparse attention without allocation or workspace, for callers that
 * cannot allocate device memory (code under HIP graph capture, serving loops
 * and harnesses that forbid it).  Arguments, outputs, layout and errors as
 * call 5 without `workspace`/`ws_bytes`: the call's work list (heads *
 * (ceil(n / 256) + c_q) slots of two 16-byte entries) lives in a fixed
 * device array of SCOPE_NOALLOC_MAX_WORK_ITEMS entries (1 MiB), one per GPU, held until
 * the process ends; larger problems return SCOPE_ERR_SCRATCH_LIMIT before
 * anything is enqueued.  The array's device address is looked up on the
 * first call on each device (the current device).  No call allocates or
 * frees memory.  Every call on a GPU shares that GPU's array and rewrites
 * the entries it reads, so calls that overlap on one GPU (two streams, or
 * two host threads) race; serialise them.                                 */
#define SCOPE_NOALLOC_MAX_WORK_ITEMS 65536
int32_t scope_sparse_attention_noalloc(const scope_shape *shape,
                                       const void *q, const void *k,
                                       const void *v, int32_t c_q,
                                       const int32_t *offsets,
                                       const int32_t *perm,
                                       const int32_t *sel_counts,
                                       const int32_t *sel_idx, float scale,
                                       void *o, void *stream);

/* Training through the layer: calls 1-4 decide index sets, which have no
 * gradient; the attention over them is differentiable in Q, K and V.
 *
 * Dropout, in the calls that take `dropout` and `rng`: each probability (or
 * element) is kept or dropped on its own and the kept ones are scaled by
 * 1 / (1 - p'), where p' = T / 65536, T = min(65535, rint(65536 * dropout)).
 * No mask is stored: `rng` (device, two uint64: seed and offset, read when the
 * kernels run, so a captured graph draws new masks when the caller writes new
 * values between replays) keys Philox4x32-10, and a backward call with the
 * same rng values repeats the forward's mask.  Calls that must not share a mask
 * (layers, steps, GPUs that hold other heads) need different seeds or offsets;
 * attention and scope_dropout draw from separate streams of one (seed, offset).
 *   pairs:    (a0, a1) = the first two words of Philox with key = seed and
 *             counter (i, 2^31 + 2h, offset low, offset high) for query token
 *             i of head h, (b0, b1) of (j, 2^31 + 2h + 1, offset low, offset
 *             high) for key token j; z = upper xor lower word of the 64-bit
 *             product (a0 xor b0) * ((a1 + b1) mod 2^32); kept if z >> 16 >= T
 *   elements: Philox of counter (e / 8 low, e / 8 high, offset low, offset
 *             high) gives element e's eight neighbours a 16-bit number each,
 *             low halves first; kept if it is >= T
 * 0 <= dropout < 1, else SCOPE_ERR_INVALID_ARGUMENT; rng is 8-byte aligned and
 * may be NULL where T = 0.
 *
 * Workspace bytes that suffice for calls 6 and 7 with these sizes (the ranges
 * of the shape are checked and not used).                                   */
int32_t scope_training_workspace_size(const scope_shape *shape, int32_t c_q,
                                      size_t *bytes);

/* 6. Attention for training.  As call 5, with the rows' statistics and dropout:
 *   lse_i = log sum_{j in S_c} exp(scale <q_i, k_j>)        (fp32, natural log)
 *   O_i   = sum_{j in S_c} exp(scale <q_i, k_j> - lse_i) m_ij v_j,
 * m_ij the dropout factor of the pair (0 or 1 / (1 - p')).  bf16 inputs run on
 * the bf16 matrix cores with the weights rounded to bf16; fp32 inputs are not
 * rounded (fp32 matrix products), unlike call 5's.  Sums and statistics are
 * fp32.  A cluster without keys gives O = 0 and lse = -inf.  Rows of queries in
 * no cluster are left as they were, in O and lse [heads][n].
 * S_c must be strictly ascending (as call 4 writes it): a key counts once; perm
 * must not hold a query twice.
 * Requirements and errors as call 5, and SCOPE_ERR_UNSUPPORTED for c_q > 1024,
 * rows of a head of 2^32 bytes or more, or so many heads and clusters that a
 * launch would need 2^32 threads; the outputs must not overlap the inputs or each
 * other (SCOPE_ERR_INVALID_ARGUMENT where O overlaps Q, K or V).
 * Calls 6 and 7 repeat bit for bit.  Long sums may be cut into parts, whose
 * number follows from heads, n, d, c_q and the dtype, so a head's last bits can
 * differ between calls of different sizes.                                  */
int32_t scope_sparse_attention_train(const scope_shape *shape, const void *q,
                                     const void *k, const void *v, int32_t c_q,
                                     const int32_t *offsets,
                                     const int32_t *perm,
                                     const int32_t *sel_counts,
                                     const int32_t *sel_idx, float scale,
                                     float dropout, const uint64_t *rng,
                                     void *o, float *lse, void *workspace,
                                     size_t ws_bytes, void *stream);

/* 7. Gradients of call 6.  From its inputs, its O and lse, and d_o, the
 * gradient of O (of the input dtype, [heads][n][d]), with the probabilities
 * recomputed from lse:
 *   p_ij = exp(scale <q_i, k_j> - lse_i), D_i = <d_o_i, O_i>
 *   ds_ij = p_ij (m_ij <d_o_i, v_j> - D_i)
 *   dQ_i = scale sum_j ds_ij k_j, dK_j = scale sum_i ds_ij q_i,
 *   dV_j = sum_i p_ij m_ij d_o_i,
 * j over S_c and i over the queries whose cluster keeps j.  Types as call 6:
 * for bf16 inputs p, and ds for dK, enter the matrix products rounded to bf16, ds
 * for dQ as two bf16 terms; every sum is fp32.  dK and dV are written for every
 * key (0 where no cluster keeps it), dQ for every query in a cluster (0 where its
 * cluster keeps no key); rows of queries in no cluster are left as they were and
 * give no gradient.  Bad sets
 * cannot fault: a set that is not strictly ascending in [0, n) sets bit 3 of
 * dev_status (may be NULL) and its gradients are unspecified.  Rows of K and V
 * that no set holds are not read into any result; a non-finite row of Q or d_o
 * may spread to dK and dV of keys that its cluster does not keep.  Requirements
 * and errors as call 6; no gradient may overlap an input or another one.     */
int32_t scope_sparse_attention_backward(
    const scope_shape *shape, const void *q, const void *k, const void *v,
    const void *o, const float *lse, const void *d_o, int32_t c_q,
    const int32_t *offsets, const int32_t *perm, const int32_t *sel_counts,
    const int32_t *sel_idx, float scale, float dropout, const uint64_t *rng,
    void *dq, void *dk, void *dv, void *workspace, size_t ws_bytes,
    int32_t *dev_status, void *stream);

/* 8. Dropout of a tensor of `count` elements (0 <= count <= 2^40) of a
 * scope_dtype, with an optional residual (NULL: none):
 *   y_e = x_e / (1 - p') where kept, else 0, plus residual_e,
 * computed in fp32 and rounded once.  A dropped element gives 0 whatever x_e is
 * (infinities and NaN among it).  The gradient of x is the same call on the
 * gradient of y with the same rng and no residual.  y may be x or the residual;
 * otherwise they must not overlap.  Pointers are aligned to their elements
 * (16-byte alignment of all is faster, the results are the same).           */
int32_t scope_dropout(int32_t dtype, int64_t count, const void *x,
                      const void *residual, float dropout, const uint64_t *rng,
                      void *y, void *stream);

/* Rows of a tensor [heads][rows][d] wherever they lie: element (h, i, c) is at
 * h * head + i * row + c, in elements.  A NULL pointer in place of strides is
 * the dense layout (row = d, head = rows * d).  Inputs may have any strides >= 0
 * (0: one row for all); rows of an output must not overlap one another.      */
typedef struct {
  int64_t row, head;
} scope_strides;

/* 9. Rotary positions: queries and keys turned by their tokens' positions (the
 * layer takes them after this), or their gradients turned back.  `axes` channel
 * ranges I_a = [range_off[a], range_off[a] + range_len[a]), disjoint, of even
 * length, hold range_len[a] / 2 pairs each: neighbours (2 i, 2 i + 1) of the range
 * for SCOPE_PAIRS (even offsets), (i, i + len / 2) for SCOPE_HALVES.  With t the
 * angle of the pair at the token's position p_a,
 *   y_a = factor (x_a cos t - x_b sin t), y_b = factor (x_a sin t + x_b cos t),
 * t replaced by -t where `inverse` (the gradient of x from that of y).  Channels
 * in no range are copied.  positions [axes][rows]; turns: for each pair, axis after
 * axis, the fraction of a whole turn per position in units of 2^-64, so that
 * t / (2 pi) = p * turns / 2^64 mod 1 is exact in integers at any position.
 * Sines and cosines are fp32 within 2^-22, products fp32, y rounded once.
 * A second tensor x2 -> y2 of heads[1] heads and the same positions (keys with
 * their queries) is turned by the same launch; heads[1] = 0: none.
 * y may be x, and y2 x2, with the same strides; otherwise an output must not overlap
 * an input, its own or the other tensor's, nor the other output.
 * Requires rows >= 0, 1 <= heads[0], 2 <= d <= 1024 even, 1 <= axes <= 3, a finite
 * factor; every size below 2^31.  Any alignment of whole elements is taken;
 * 16-byte alignment of pointers and strides, with d (and for halves ranges'
 * offsets and half lengths) multiples of 8, is faster.                       */
typedef enum { SCOPE_PAIRS = 0, SCOPE_HALVES = 1 } scope_rotary_layout;
typedef struct {
  int32_t rows, heads[2], d, dtype;
  int32_t axes, range_off[3], range_len[3];
  int32_t layout, inverse;
  float factor;
} scope_rotation;
int32_t scope_rotary(const scope_rotation *rotation, const int32_t *positions,
                     const uint64_t *turns, const void *x, const scope_strides *x_strides,
                     void *y, const scope_strides *y_strides, const void *x2,
                     const scope_strides *x2_strides, void *y2,
                     const scope_strides *y2_strides, void *stream);

/* Exact attention over sequences packed one after the other, with query heads in
 * groups that share a key head (heads a multiple of kv_heads; query head h reads key
 * head h / (heads / kv_heads)).  Sequence s has the query rows offsets_q[s] ..
 * offsets_q[s+1] and the key rows offsets_k[s] .. offsets_k[s+1], or with lengths_k
 * (call 10) the first lengths_k[s] of those, a cache with room for more.  Lengths may
 * differ and be 0.  With n queries and m keys of a sequence, query i sees every key,
 * or where `causal` the keys j <= i + m - n: the last query sees all, queries before
 * the first key see none.  Output rows in no sequence (before the first offset or
 * from the last on) are left as they were, or where `clear` set to 0, lse to -inf.
 * Supported: d in {64, 128}, 1 <= sequences <= 65536, 0 <= rows <= 2^24, heads * rows
 * < 2^31 each, fewer than 2^30 queries of one key head, so few items that a launch needs
 * less than 2^32 threads; 16-byte aligned rows (pointers and strides); 66 rows in a row,
 * of one key head or of all query heads that share it, within 2^32 bytes.     */
typedef struct {
  int32_t heads, kv_heads;
  int32_t rows_q, rows_k; /* rows of q, o; of k, v */
  int32_t sequences;
  int32_t d, dtype, causal;
  int32_t clear;          /* output rows in no sequence: 0 as they were, else set */
} scope_pack;

/* Workspace bytes that suffice for calls 10 and 11 with these sizes.        */
int32_t scope_packed_workspace_size(const scope_pack *pack, size_t *bytes);

/* 10. Forward, for prompts, chunks behind a cache and single tokens:
 *   lse_i = log sum_j exp(scale <q_i, k_j>)   (fp32, natural log; [heads][rows_q])
 *   O_i   = sum_j exp(scale <q_i, k_j> - lse_i) v_j,  j over the keys that i sees
 * (scale <= 0 selects 1/sqrt(d)).  A query that sees no key gives O = 0 and
 * lse = -inf.  Rows in no sequence are not read, those of O and lse as `clear` says.
 * Types as call 6 (fp32 inputs are not rounded, bf16 weights are); sums and
 * statistics are fp32.  A non-finite key row reaches only queries that see it; a
 * non-finite value row may also reach queries whose last key lies up to 94 before it.
 * Results repeat bit for bit.  Long sums may be cut into parts, whose number follows
 * from the sizes in `pack` alone.
 * Bad offsets cannot fault: each is taken as the largest so far within [0, rows] and
 * lengths are cut to their room; either sets bit 4 of dev_status (may be NULL).
 * lse and O must not overlap the inputs.                                      */
int32_t scope_packed_attention(const scope_pack *pack, const void *q,
                               const scope_strides *q_strides, const void *k,
                               const scope_strides *k_strides, const void *v,
                               const scope_strides *v_strides, const int32_t *offsets_q,
                               const int32_t *offsets_k, const int32_t *lengths_k,
                               float scale, void *o, const scope_strides *o_strides,
                               float *lse, void *workspace, size_t ws_bytes,
                               int32_t *dev_status, void *stream);

/* 11. Gradients of call 10 (without lengths_k), formulas and types as call 7
 * without dropout: dK and dV sum over the query heads that share the key head.  dK
 * and dV are 0 for keys of a sequence that no query sees, dQ for queries that see no
 * key; rows in no sequence as `clear` says.  A non-finite row of Q or d_o may
 * reach dK and dV of keys of its sequence that it does not see, a non-finite row of
 * K or V dQ of queries that do not see it.  No gradient may overlap an input or
 * another one.  Otherwise as call 10.                                        */
int32_t scope_packed_attention_backward(
    const scope_pack *pack, const void *q, const scope_strides *q_strides, const void *k,
    const scope_strides *k_strides, const void *v, const scope_strides *v_strides,
    const void *o, const scope_strides *o_strides, const float *lse, const void *d_o,
    const scope_strides *d_o_strides, const int32_t *offsets_q, const int32_t *offsets_k,
    float scale, void *dq, const scope_strides *dq_strides, void *dk,
    const scope_strides *dk_strides, void *dv, const scope_strides *dv_strides,
    void *workspace, size_t ws_bytes, int32_t *dev_status, void *stream);

/* Diagnostics: the measured peaks that roofline fractions are also quoted
 * against.  scope_debug_copy copies `bytes` (a multiple of 16; src and dst
 * 16-byte aligned, not overlapping) with a plain vector copy kernel, so its
 * time gives the achievable HBM bandwidth (2 * bytes moved).
 * scope_debug_mfma_loop launches `blocks` blocks of 256 threads whose waves
 * each issue iters * 8 independent bf16 32x32x16 matrix products from
 * registers (8 * 32768 * iters flops per wave) and write one float per
 * thread to out[blocks * 256]: the achievable bf16 MFMA rate.              */
int32_t scope_debug_copy(const void *src, void *dst, size_t bytes, void *stream);
int32_t scope_debug_mfma_loop(float *out, int32_t blocks, int32_t iters,
                              void *stream);

/* Diagnostic: the selection's fixed-point exponential (call 4) applied to
 * y[0..count) (y <= 0), results in out[0..count).                          */
int32_t scope_debug_fixexp(const float *y, uint64_t *out, int64_t count,
                           void *stream);

/* Diagnostic: the work list of call 5 for `heads` heads, as the sparse
 * attention builds it.  offsets [heads][c_q + 1] and sel_counts
 * [heads][c_q] (device) are as for scope_sparse_attention.  *items_per_head
 * (host) receives S, the slots per head; items (device, 16-byte aligned,
 * `capacity` int32 values, at least heads * S * 8) receives
 * [heads][S][2][4] int32: each slot holds two entries (cluster, first row,
 * rows, selected keys) run by one block, the second with rows = 0 when the
 * block runs one chunk, and slots with both entries empty after the used
 * ones.  pair != 0 lets two remainder chunks share a slot, as every kernel
 * but the one for fp32 inputs without room for bf16 copies does.  The list
 * is in cost order, as for a call without a block order of its own.
 * Returns SCOPE_ERR_INVALID_ARGUMENT on bad sizes or pointers, before any
 * launch.                                                                   */
int32_t scope_debug_attention_items(int32_t heads, int32_t n, int32_t c_q,
                                    int32_t pair, const int32_t *offsets,
                                    const int32_t *sel_counts, int32_t *items,
                                    int64_t capacity, int32_t *items_per_head,
                                    void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SCOPE_H */
