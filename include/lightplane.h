/*
 * lightplane.h — C ABI of the MI355X (gfx950) Lightplane Renderer library.
 *
 * The library computes the Renderer of "Lightplane" (arXiv 2404.19760): fused,
 * differentiable emission-absorption ray marching over a hybrid 3D representation
 * f = g o h (Section 3.2), where h is bi/tri-linear sampling of a triplane or voxel
 * feature grid and g a tiny MLP, with a backward pass that stores one scalar per ray
 * and recomputes everything else (Section 3.4).  Next to it: the Splatter, and for networks that work
 * on the structures a group norm with an activation, products with bias, activation and residual, the norms around a
 * residual block, the clipping of gradients by their norm and the orthogonalised update of weight matrices.
 *
 * General rules
 *   - Every pointer named "device" is a pointer to GPU memory owned by the caller
 *     (for example a torch tensor); the small structs themselves and the pointer
 *     arrays inside them live in HOST memory and are read during the call only.
 *   - Calls enqueue work on `stream` (a hipStream_t passed as void*, NULL = the
 *     default stream) and return without waiting.  The library allocates nothing
 *     and keeps no pointer after a call returns.
 *   - Every function returns an lp_status and never throws or aborts; a message
 *     for the last failure on the calling thread is available from lp_last_error().
 *   - All floating point is IEEE binary32 and tensors are dense and C-contiguous unless a call says
 *     otherwise.
 */
#ifndef LIGHTPLANE_H
#define LIGHTPLANE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LP_MAX_LAYERS 8    /* linear layers of a decoder MLP */
#define LP_MAX_FEATURES 16 /* rendered feature channels of the two-MLP decoder */

typedef enum {
    LP_OK = 0,
    LP_ERR_INVALID_ARG = 1, /* NULL required pointer, non-positive size, dims mismatch      */
    LP_ERR_UNSUPPORTED = 2, /* valid, but no kernel of this library covers the shape       */
    LP_ERR_HIP = 3,         /* the HIP runtime reported an error (launch, attribute query) */
    LP_ERR_WORKSPACE = 4    /* workspace missing or smaller than lp_bwd_workspace_bytes     */
} lp_status;

typedef enum { LP_GRID_VOXEL = 0, LP_GRID_TRIPLANE = 1, LP_GRID_HASH = 2, LP_GRID_HEXPLANE = 3 } lp_grid_kind;

/* Storage type of the values of a hash structure that is READ (Section 3.2 notes that the
   hashing scheme is where precision and layout can be traded).  Gradients and the Splatter's
   outputs are always fp32. */
typedef enum { LP_F32 = 0, LP_BF16 = 1, LP_F16 = 2 } lp_dtype;

/*
 * The 3D hash structure theta (Section 3.2), channel-last.
 *   voxel   : data[0] = [B][NX][NY][NZ][C]                       (data[1], data[2] ignored)
 *   triplane: data[0] = [B][NX][NY][C], data[1] = [B][NY][NZ][C], data[2] = [B][NZ][NX][C];
 *             a point (x,y,z) reads plane 0 at (x,y), plane 1 at (y,z), plane 2 at (z,x)
 *             bilinearly and SUMS the three feature vectors.
 *   hash    : data[0] = [B][hash_size][C], a hash table (Section 3.2 names hash tables among the
 *             structures; the paper defines none, this one is the single-resolution spatial hash
 *             of Teschner et al. 2003 that Instant-NGP uses): the point is interpolated
 *             trilinearly in a virtual NX x NY x NZ lattice as in a voxel grid, but lattice corner
 *             (ix, iy, iz) is stored in entry ((ix * 1) xor (iy * 2654435761) xor (iz * 805459861))
 *             mod hash_size (products and xor in 32-bit unsigned arithmetic); corners that collide
 *             share the entry and their gradients add.  The Splatter writes such tables too
 *             (colliding corners pool what is pushed into them).
 *             The matrix-core kernels take tables whose hash_size is a power of two (16 or 32
 *             channels, or 16 channels under the merged two-MLP decoder); every other table runs
 *             on the generic kernels.
 *   hexplane: a structure over space AND time (Section 3.2 names HexPlane among the structures;
 *             the definition is Cao & Johnson 2023's): data[0..2] as the triplane's planes, and
 *             data_t[p] = [B][N_c][NT][C] the space-time plane over (c, t), c being the spatial
 *             axis that plane p leaves out (z, x, y for p = 0, 1, 2).  A point (x,y,z) of a ray
 *             with time t reads both planes of a pair bilinearly, multiplies the two feature
 *             vectors channel by channel, and SUMS the three products.  Time t_min maps to index 0
 *             and t_max to index NT - 1 of the time axis, times outside are clamped; contract
 *             coordinates act on the spatial axes only.  The gradient has six tensors (d_grid[p]
 *             for data[p], d_grid[3 + p] for data_t[p]).  Renderer only (the Splatter refuses it).
 *             The matrix-core kernels take 16 or 32 channels (or 16 channels under the merged
 *             two-MLP decoder); every other shape runs on the generic kernels.
 * World coordinate aabb_min[a] maps to index 0 and aabb_max[a] to index N_a - 1 along axis
 * a; positions outside the box are clamped onto it.  B scenes share the MLP.
 * contract_a: 0 = off.  In (0, 2]: contract coordinates (appendix, "Experimental Details",
 * equation CC) with foreground scale a: every axis of a sample position is first mapped by
 * CC(x) = 0.5 a x for |x| <= 1 and 0.5 ((2 - a)(1 - 1/|x|) + a) sign(x) beyond (the paper
 * converts the axes independently), which sends the whole line into (-1, 1) and the unit
 * interval onto [-a/2, a/2]; the box mapping above then applies to the contracted position
 * (use the box [-1, 1]^3).  Sample spacing stays the world distance along the ray.
 */
typedef struct {
    int32_t kind; /* lp_grid_kind */
    int32_t B, C; /* scenes, feature channels (the paper's K) */
    int32_t NX, NY, NZ;
    const void* data[3]; /* device; elements of type `dtype` */
    float aabb_min[3], aabb_max[3];
    float contract_a;
    int32_t dtype; /* lp_dtype; LP_BF16 / LP_F16 halve the bytes a sample reads */
    int64_t hash_size; /* LP_GRID_HASH: entries of one scene's table, in [1, 2^31); else ignored */
    const void* data_t[3]; /* LP_GRID_HEXPLANE: device, the space-time planes; else ignored */
    int32_t NT;            /* LP_GRID_HEXPLANE: resolution of the time axis, >= 2 */
    float t_min, t_max;    /* LP_GRID_HEXPLANE: times of the first and last index, t_max > t_min */
} lp_grid;

/*
 * The tiny MLP g (Section 3.2): n_layers linear layers, ReLU after every layer but the
 * last.  dims[0] == C, dims[n_layers] == 4.  Output 0 through softplus is the density
 * sigma; outputs 1..3 through the logistic sigmoid are the colour.
 * W[l] = [dims[l+1]][dims[l]] row-major (out, in), b[l] = [dims[l+1]].
 */
typedef struct {
    int32_t n_layers;
    int32_t dims[LP_MAX_LAYERS + 1];
    const float* W[LP_MAX_LAYERS]; /* device */
    const float* b[LP_MAX_LAYERS]; /* device */
} lp_mlp;

/*
 * M rays with S samples each (the ray set of Section 3.3, whose R + 1 points per ray are read as S samples).  Sample j
 * (j = 1..S) sits at distance t_j = near + (j - 1/2) (far - near) / S from the origin along
 * the UNIT direction, so Delta = (far - near) / S is the world distance between samples.
 */
typedef struct {
    int64_t M;
    int32_t S;
    const float* origins; /* device [M][3] */
    const float* dirs;    /* device [M][3], unit length (not renormalised) */
    const float* near;    /* device [M] */
    const float* far;     /* device [M] */
    const int32_t* scene; /* device [M] scene index in [0,B), or NULL (all rays use scene 0) */
    const float* time;    /* device [M] time of every ray, or NULL (all rays at the grid's t_min);
                             read for LP_GRID_HEXPLANE only */
} lp_rays;

/* How the MLP contractions are evaluated by the matrix-core kernels. */
typedef enum {
    LP_MATH_DEFAULT = 0, /* the library's choice for the shape                            */
    LP_MATH_GENERIC = 1, /* scalar fp32 kernels for any layer widths (slow)               */
    LP_MATH_BF16X3 = 2   /* fp32 operands split into bf16 hi+lo, three MFMA products,
                            fp32 accumulation (matrix-core kernels; supported shapes only) */
} lp_math_mode;

/*
 * Forward (Eq. (1), Section 3.3).  With T_0 = 1, T_j = T_{j-1} exp(-sigma_j Delta),
 * w_j = T_{j-1} - T_j:
 *     rgb = sum_j w_j c_j + T_S bg,   alpha = 1 - T_S,   depth = sum_j w_j t_j.
 * Outputs (device, written, not accumulated): rgb [M][3], alpha [M], depth [M], and
 * ray_cache [M], the one scalar per ray the backward needs (Section 3.4; here the total
 * optical depth sum_j sigma_j Delta, opaque to the caller).  alpha, depth and ray_cache
 * may each be NULL if not wanted.  bg is a HOST array of 3 floats.  M == 0 is a no-op.
 */
lp_status lp_render_fwd(const lp_grid* grid, const lp_mlp* mlp, const lp_rays* rays,
                        const float bg[3], float* rgb, float* alpha, float* depth,
                        float* ray_cache, int32_t math_mode, void* stream);

/*
 * Backward (Eq. (2), Section 3.4): vector-Jacobian product of the forward for upstream
 * gradients d_rgb [M][3] (required), d_alpha [M], d_depth [M] (either may be NULL = zero),
 * all device.  Marches each ray in reverse, recomputes sampling and MLP, rebuilds the
 * transmittance from ray_cache (as written by lp_render_fwd for the SAME inputs), and
 * ACCUMULATES into (the caller zeroes or pre-loads them):
 *     d_grid[p] — same shape as grid->data[p] (device; triplane: all three required; HexPlane: six,
 *                 d_grid[3 + p] with the shape of grid->data_t[p]),
 *     dW[l], db[l] — same shapes as mlp->W[l], mlp->b[l] (device).
 * No gradient is produced for rays, near, far or bg.  `workspace` is device memory of at
 * least lp_bwd_workspace_bytes(...) bytes, 256-byte aligned, contents ignored on entry and
 * undefined on exit.  Grid gradients are summed with floating-point atomics, so they are
 * reproducible up to summation order only.
 */
lp_status lp_render_bwd(const lp_grid* grid, const lp_mlp* mlp, const lp_rays* rays,
                        const float bg[3], const float* d_rgb, const float* d_alpha,
                        const float* d_depth, const float* ray_cache, float* const d_grid[],
                        float* const dW[LP_MAX_LAYERS], float* const db[LP_MAX_LAYERS],
                        void* workspace, size_t workspace_bytes, int32_t math_mode,
                        void* stream);

/* Bytes of workspace lp_render_bwd needs for these shapes; independent of S and of M
   (it depends on the MLP size and the device's compute-unit count).  *bytes is written. */
lp_status lp_bwd_workspace_bytes(const lp_grid* grid, const lp_mlp* mlp, const lp_rays* rays,
                                 int32_t math_mode, size_t* bytes);

/*
 * lp_render_bwd for callers that cannot allocate device memory or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * results and error behaviour as lp_render_bwd without `workspace`: the per-wave partial-sum
 * records of the MLP gradients go to a static device array of LP_STATIC_SCRATCH_BYTES that the
 * library holds on every GPU it runs on until the process ends.  The call allocates nothing.
 * A shape whose records need more (an MLP of more than about 8 000 parameters on the
 * matrix-core kernels) is refused with LP_ERR_UNSUPPORTED and a message that names both sizes.
 * All calls on one GPU share that array: calls that overlap on one GPU (different streams or
 * threads) race; calls that are ordered on one stream do not (the records are fully rewritten
 * by every call before they are read, nothing needs clearing).
 */
#define LP_STATIC_SCRATCH_BYTES (32u * 1024u * 1024u)
lp_status lp_render_bwd_static(const lp_grid* grid, const lp_mlp* mlp, const lp_rays* rays,
                               const float bg[3], const float* d_rgb, const float* d_alpha,
                               const float* d_depth, const float* ray_cache, float* const d_grid[],
                               float* const dW[LP_MAX_LAYERS], float* const db[LP_MAX_LAYERS],
                               int32_t math_mode, void* stream);

/* 1 if the matrix-core (LP_MATH_BF16X3) kernels cover this grid kind / MLP shape, else 0. */
int32_t lp_has_fast_path(const lp_grid* grid, const lp_mlp* mlp);

/* ---- The Renderer with the paper's own decoder (Section 3.3, text below Eq. (1)) ----------
 *
 * Two MLPs instead of one: the opacity MLP g_sigma maps the sampled feature to the density
 * (one output, through softplus); the feature MLP g_v maps the sampled feature AND the
 * encoded view direction to the n_feat rendered features f_v ("e.g. colors"):
 *     sigma_j = softplus(g_sigma(h(x_j))),   f_j = act(g_v([h(x_j) ; enc(d)])),
 *     out = sum_j w_j f_j + T_S bg   (n_feat channels),   alpha, depth as in lp_render_fwd.
 * enc(d) = (d, sin(2^k pi d), cos(2^k pi d) for k = 0 .. n_freq-1), component by component:
 * 3 + 6 n_freq values (the paper does not give the form; n_freq = 0 is the raw direction).
 * act = logistic sigmoid (LP_FEAT_SIGMOID) or identity (LP_FEAT_IDENTITY).
 * opacity.dims[0] == C, last == 1; feature.dims[0] == C + 3 + 6 n_freq, last == n_feat;
 * both MLPs need at least one hidden layer (n_layers >= 2); 1 <= n_feat <= LP_MAX_FEATURES;
 * 0 <= n_freq <= 4.  No gradient is produced for the directions.
 */
typedef enum { LP_FEAT_SIGMOID = 0, LP_FEAT_IDENTITY = 1 } lp_feat_act;

typedef struct {
    lp_mlp opacity; /* g_sigma */
    lp_mlp feature; /* g_v */
    int32_t n_freq;
    int32_t n_feat;
    int32_t feat_act; /* lp_feat_act */
} lp_decoder;

/* Bytes of device workspace the two calls below need (either pointer may be NULL).
   Independent of S and M.  The workspace holds the two MLPs merged into one block-structured
   MLP (and, for the backward, its gradient and the partial-sum records). */
lp_status lp_dec_workspace_bytes(const lp_grid* grid, const lp_decoder* dec, const lp_rays* rays,
                                 int32_t math_mode, size_t* fwd_bytes, size_t* bwd_bytes);

/* Forward.  out [M][n_feat], alpha [M], depth [M], ray_cache [M] (device; the last three may
   be NULL); bg is a HOST array of n_feat floats; workspace: device, 256-byte aligned, at least
   the fwd_bytes of lp_dec_workspace_bytes, contents ignored on entry, undefined on exit. */
lp_status lp_render_dec_fwd(const lp_grid* grid, const lp_decoder* dec, const lp_rays* rays,
                            const float* bg, float* out, float* alpha, float* depth, float* ray_cache,
                            void* workspace, size_t workspace_bytes, int32_t math_mode, void* stream);

/* Backward: upstream gradients d_out [M][n_feat] (required), d_alpha, d_depth (may be NULL);
   ACCUMULATES into d_grid (as lp_render_bwd) and into dW_opacity[l], db_opacity[l],
   dW_feature[l], db_feature[l] (device, shapes of the decoder's weights and biases).
   workspace: at least the bwd_bytes of lp_dec_workspace_bytes. */
lp_status lp_render_dec_bwd(const lp_grid* grid, const lp_decoder* dec, const lp_rays* rays,
                            const float* bg, const float* d_out, const float* d_alpha,
                            const float* d_depth, const float* ray_cache, float* const d_grid[],
                            float* const dW_opacity[LP_MAX_LAYERS], float* const db_opacity[LP_MAX_LAYERS],
                            float* const dW_feature[LP_MAX_LAYERS], float* const db_feature[LP_MAX_LAYERS],
                            void* workspace, size_t workspace_bytes, int32_t math_mode, void* stream);

/* 1 if the matrix-core kernels cover this grid kind / decoder shape, else 0.  Covered, for
   three features (sigmoid or identity) on grids of any storage type: 16 grid channels with a merged hidden width (opacity +
   feature MLP, layer by layer) of 32 or 64, one or two hidden layers, at most 16 direction
   inputs; and 16 or 32 grid channels with two 3-layer MLPs of width 64 each (the paper's
   experimental size, any n_freq), which run as two chains. */
int32_t lp_dec_has_fast_path(const lp_grid* grid, const lp_decoder* dec);

/* ---- Splatter (Section 3.3 "Splatter"; appendix "Normalization Process in Splatter") ---------
 *
 * The dual of the Renderer: M pixels with feature vectors are expanded into rays of S points
 * (placed like the Renderer's samples); every point pushes a feature vector into the target
 * hash structure with the interpolation weights the Renderer reads that cell with, and each
 * cell is finally divided by the sum of the weights that landed on it:
 *     theta[corner] += weight * vt_ij,  theta_w[corner] += weight,  out = theta / theta_w
 * (0 where nothing landed).  Naive Splatter (mlp == NULL, n_in == target->C): vt_ij = v_i.
 * With the MLP g_s: vt_ij = g_s([v_i ; h_prior(x_ij) ; enc(d_i)]) with h_prior the prior
 * structure read at the point (prior == NULL: none) and enc the direction encoding of the
 * two-MLP decoder above (n_freq = -1: none); ReLU hidden layers, linear output;
 * mlp->dims[0] == n_in + prior->C + (3 + 6 n_freq), mlp->dims[last] == target->C.
 * The prior has the target's kind, scene count, box and contraction; its own resolution (and,
 * for hash tables, its own hash_size).  Targets: voxel grids, triplanes and hash tables (a
 * HexPlane target is refused with LP_ERR_UNSUPPORTED).
 */
typedef struct {
    int32_t n_in;         /* channels of the pixel features */
    int32_t n_freq;       /* octaves of the direction encoding fed to the MLP, -1: none */
    const float* feats;   /* device [M][n_in] */
    const lp_grid* prior; /* NULL: none */
    const lp_mlp* mlp;    /* NULL: naive Splatter */
} lp_splat;

/* Forward.  target gives kind, B, C, resolution, box and contraction of the structure to
   build (its data pointers are ignored).  theta[p] (shape of the target's tensors) and
   theta_w[p] (same without the channel axis) are device buffers that are WRITTEN: the
   normalised structure and the weight sums (the backward needs the latter). */
lp_status lp_splat_fwd(const lp_grid* target, const lp_rays* rays, const lp_splat* splat,
                       float* const theta[3], float* const theta_w[3], void* stream);

/* 1 if lp_splat_fwd (and, with an MLP, lp_splat_bwd) runs this target / splat on the
   kernels for 16 and 32 channels (a wavefront takes a patch of an image's pixels, a tile of four
   rays or one ray), else 0 (generic kernels, same results).  Covered: targets of 16 or
   32 channels, with or without contract coordinates (voxel grids, triplanes and, for the naive
   Splatter, hash tables whose size is a power of two); with an MLP, voxel grids and triplanes
   with a prior of the same channel count and contraction in fp32, one or two hidden layers of
   width 64, and at most 48 pixel-feature plus direction-encoding inputs.  Nothing behind the
   device pointers is read. */
int32_t lp_splat_has_fast_path(const lp_grid* target, const lp_splat* splat);

/* Backward for d_theta[p] = dL/d(out) (device).  The weights depend on the ray geometry only,
   so dL/dtheta = d_theta / theta_w; the gradient of a pushed feature is that field read at
   the point.  d_feats [M][n_in] is WRITTEN; d_prior[p] (shapes of the prior's tensors),
   dW[l], db[l] are ACCUMULATED into (NULL lists are allowed where there is no prior / MLP).
   workspace: device, 256-byte aligned, lp_splat_bwd_workspace_bytes bytes. */
lp_status lp_splat_bwd(const lp_grid* target, const lp_rays* rays, const lp_splat* splat,
                       const float* const theta_w[3], const float* const d_theta[3], float* d_feats,
                       float* const d_prior[3], float* const dW[LP_MAX_LAYERS],
                       float* const db[LP_MAX_LAYERS], void* workspace, size_t workspace_bytes,
                       void* stream);

lp_status lp_splat_bwd_workspace_bytes(const lp_grid* target, const lp_rays* rays, const lp_splat* splat,
                                       size_t* bytes);

/* ---- Group norm with an activation over channel-last grids --------------------------------------
 *
 * What networks that work on the library's structures (between a Splatter and a Renderer) put between
 * their layers.  x holds N samples (scenes, planes) of P positions with C channels each, channel last:
 * element (n, p, c) sits at ((n P + p) stride + c), so voxel grids are P = NX NY NZ positions and a
 * plane of a triplane P = NX NY, and a slice of the channels of a wider tensor has a stride beyond C.
 * The C / G channels of a group and the positions of a sample are normalised together,
 *     mean, var = of the sample's group (var without Bessel's correction), rstd = (var + eps)^(-1/2),
 *     xh = (x - mean) rstd,   y = act(gamma xh + beta).
 * occupancy [N][P] (the weight sums theta_w a Splatter writes are one): positions whose value is not
 * above zero do not take part: x and d_y are not used there (they may hold anything, NaN included),
 * y and d_x are 0.  A sample without any position that takes part has mean = rstd = 0.
 * Statistics, sums and gamma, beta and their gradients are fp32 or wider whatever the tensors hold.
 */
typedef enum { LP_ACT_NONE = 0, LP_ACT_RELU = 1, LP_ACT_SILU = 2, LP_ACT_GELU = 3 /* with the error function */ } lp_act;

typedef struct {
    int64_t N, P;
    int32_t C, G;             /* channels, groups; G divides C */
    int32_t act;              /* lp_act */
    float eps;                /* >= 0, finite */
    int32_t x_dtype;          /* lp_dtype of x and d_x */
    int32_t y_dtype;          /* lp_dtype of y and d_y: x_dtype, or a 16-bit type where x is fp32 */
    int64_t x_stride;         /* elements from position to position of x and d_x, >= C; 0: C */
    int64_t y_stride;         /* the same of y and d_y */
    const float* gamma;       /* device [C], NULL: 1 */
    const float* beta;        /* device [C], NULL: 0 */
    const float* occupancy;   /* device [N][P], NULL: every position takes part */
} lp_group_norm;

/* Bytes of device workspace of the two calls below (either pointer may be NULL); they depend on
   N, P, C, G and the device's compute-unit count, and may be 0 (then NULL will do). */
lp_status lp_group_norm_workspace_bytes(const lp_group_norm* norm, size_t* fwd_bytes, size_t* bwd_bytes);

/* Forward.  y is WRITTEN; stats [N][G][2] (device, fp32: mean, rstd; may be NULL) is written for the
   backward.  workspace: device, 256-byte aligned, contents ignored on entry, undefined on exit.
   y may be x itself where types and strides are alike.  N == 0 or P == 0 is a no-op. */
lp_status lp_group_norm_fwd(const lp_group_norm* norm, const void* x, void* y, float* stats, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Backward for the upstream gradient d_y, with x as the forward had it and the stats it wrote.  d_x is
   WRITTEN (NULL: not wanted); d_gamma [C], d_beta [C] are ACCUMULATED into (either may be NULL), in an
   order that does not change from call to call.  d_x may be d_y itself where types and strides are alike.
   Of a ReLU the gradient at 0 is 0. */
lp_status lp_group_norm_bwd(const lp_group_norm* norm, const void* x, const float* stats, const void* d_y, void* d_x,
                            float* d_gamma, float* d_beta, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Products with bias, activation and residual ------------------------------------------------
 *
 * The other half of a layer over the cells of a grid, or over tokens: x holds P positions of K channels, channel
 * last, element (p, k) at (p x_stride + k), and every position becomes N channels,
 *     z = x W^T + b,   y = act(z) + r,
 * with W [N][K] dense and r (the residual) of y's shape.  All tensors but b and the parameters' gradients are of one type;
 * products and sums are fp32 (16-bit types: exact products on the matrix cores), and each result is rounded once.
 * The backward, for the upstream gradient d_y and the z that the forward kept (`pre`, rounded to the tensors' type):
 *     d_z = d_y act'(z),   d_x = d_z W,   d_W += d_z^T x,   d_b += sum over the positions of d_z;   r's gradient is d_y.
 * In d_x a 16-bit d_z is rounded once more; in d_W a bf16 one is kept in three parts (24 bits), an fp16 one in two (19 bits; one that is infinite, or beyond the
 * type's largest number, leaves NaN), in d_b in fp32.
 */
typedef struct {
    int64_t P;             /* positions */
    int32_t K, N;          /* channels in and out, 1 .. 2^20 */
    int32_t act;           /* lp_act */
    int32_t dtype;         /* lp_dtype of weight, x, residual, y, pre, d_y and d_x */
    int64_t x_stride;      /* elements from position to position of x and d_x, >= K; 0: K */
    int64_t y_stride;      /* the same of y and d_y, >= N; 0: N */
    int64_t r_stride;      /* the same of the residual; 0: N */
    const void* weight;    /* device [N][K] */
    const float* bias;     /* device [N], NULL: 0 */
    const void* residual;  /* device, NULL: 0; not used by the backward */
} lp_linear;

/* Bytes of device workspace of the two calls below (either pointer may be NULL); they depend on P, K, N, act and dtype and on the
   device's compute-unit count, and may be 0 (then NULL will do). */
lp_status lp_linear_workspace_bytes(const lp_linear* linear, size_t* fwd_bytes, size_t* bwd_bytes);

/* Forward.  y is WRITTEN; pre [P][N] (dense; may be NULL) is written for the backward.  y may be the residual itself where the
   strides are alike, and must not overlap anything else.  workspace: device, 256-byte aligned, contents ignored on
   entry, undefined on exit.  P == 0 is a no-op. */
lp_status lp_linear_fwd(const lp_linear* linear, const void* x, void* y, void* pre, void* workspace, size_t workspace_bytes, void* stream);

/* Backward.  pre as the forward wrote it (not used, and may be NULL, where act is LP_ACT_NONE).  d_x is WRITTEN (NULL: not
   wanted); d_weight [N][K] and d_bias [N] are ACCUMULATED into (either may be NULL), in an order that does not change from call to
   call.  None of the three may overlap anything else that the call is given.  x is read for d_weight alone and the weight for d_x
   alone: either may be NULL where that is.  Of a ReLU the gradient at 0 is 0. */
lp_status lp_linear_bwd(const lp_linear* linear, const void* x, const void* pre, const void* d_y, void* d_x, float* d_weight,
                        float* d_bias, void* workspace, size_t workspace_bytes, void* stream);

/* ---- The norms around a residual block ----------------------------------------------------------
 *
 * What stands between two blocks of a network over cells or tokens, in one pass.  With h the sum over the blocks so far, f the
 * last block's result and norm(v) = (v - mean) / sqrt(var + eps) (LP_NORM_LAYER; var without Bessel's correction) or
 * v / sqrt(mean of v^2 + eps) (LP_NORM_RMS) over the C channels of a position,
 *     u = post_gamma norm(f) (post_norm) or f,   s = alpha h + gate u,   y = gamma norm(s) + beta:
 * s goes on to the next block's sum, y into the next block.  N samples of P positions each, element (n, p, c) at
 * (n P + p) stride + c; a gate may differ from sample to sample.  Norms and sums are fp32 whatever the tensors hold, and y
 * comes from s before s is rounded.
 */
typedef enum { LP_NORM_RMS = 0, LP_NORM_LAYER = 1 } lp_norm_kind;

#define LP_RESIDUAL_NORM_MAX_CHANNELS 8192

typedef struct {
    int64_t N, P;
    int32_t C;                /* channels, 1 .. LP_RESIDUAL_NORM_MAX_CHANNELS */
    int32_t kind;             /* lp_norm_kind of both norms */
    int32_t post_norm;        /* 0 or 1 */
    int32_t gate_per_sample;  /* gate is [C] (0) or [N][C] (1) */
    float alpha;              /* finite */
    float eps;                /* >= 0, finite */
    int32_t h_dtype;          /* lp_dtype of h, s and their gradients */
    int32_t f_dtype;          /* lp_dtype of f, y and their gradients: h_dtype, or a 16-bit type where that is fp32 */
    int64_t h_stride;         /* elements from position to position of h, s, d_s and d_h, >= C; 0: C */
    int64_t f_stride;         /* the same of f and d_f */
    int64_t y_stride;         /* the same of y and d_y */
    const float* post_gamma;  /* device [C], NULL: 1 */
    const float* gate;        /* device, NULL: 1 */
    const float* gamma;       /* device [C], NULL: 1 */
    const float* beta;        /* device [C], NULL: 0 */
} lp_residual_norm;

/* Bytes of device workspace of the backward; they depend on N, P, C, post_norm and gate_per_sample and on the device's compute-unit count. */
lp_status lp_residual_norm_workspace_bytes(const lp_residual_norm* norm, size_t* bwd_bytes);

/* Forward.  f may be NULL (the first norm of a network: s = alpha h); s and y are WRITTEN, either may be NULL.  s may be h
   itself, y may be f itself where the strides are alike; otherwise what is written must not overlap anything else.
   N == 0 or P == 0 is a no-op. */
lp_status lp_residual_norm_fwd(const lp_residual_norm* norm, const void* h, const void* f, void* s, void* y, void* stream);

/* Backward from the forward's inputs (it computes s again) for the upstream gradients d_s and d_y (either may be NULL: zero).  d_h
   and d_f are WRITTEN (NULL: not wanted); d_h may be d_s itself, d_f may be d_y itself where the strides are alike, otherwise they must
   not overlap anything else.  d_gamma [C], d_beta [C], d_post_gamma [C] and d_gate (the gate's shape) are ACCUMULATED into (NULL:
   not wanted), in an order that does not change from call to call, and must not overlap anything else.  workspace: device, 256-byte aligned, contents ignored on entry,
   undefined on exit. */
lp_status lp_residual_norm_bwd(const lp_residual_norm* norm, const void* h, const void* f, const void* d_s, const void* d_y, void* d_h,
                               void* d_f, float* d_gamma, float* d_beta, float* d_post_gamma, float* d_gate, void* workspace,
                               size_t workspace_bytes, void* stream);

/* ---- The norm of all gradients, and clipping ----------------------------------------------------
 *
 * Before the optimiser's step: norm = sqrt(sum of squares of all values of all tensors), and
 *     out = in min(1, max_norm / (norm + eps)).
 * Squares and their sum are fp64, so that no fp32 value is too large or too small for them; the factor is applied in fp32 (in
 * fp64 where it is below fp32's normal numbers) and the result rounded once.  `norm` is rounded to fp32: infinite beyond its largest
 * number, with results that are clipped as others are.  A norm that is not finite in fp64 is applied as it is (an infinite one makes the finite values 0 and the infinite
 * ones NaN, NaN makes all NaN): look at `norm` where that must not reach the weights.
 */
typedef struct {
    int64_t size;     /* values */
    const void* in;   /* device, elements of type `dtype`, aligned to their size */
    void* out;        /* device, the same type; may be `in`; not used by lp_grad_norm */
    int32_t dtype;    /* lp_dtype */
} lp_gradient;

/* norm (device, 1 float) is WRITTEN.  `grads` is a HOST array; n == 0 and tensors of size 0 are fine (a norm of 0).  workspace: device,
   256-byte aligned, contents ignored on entry, undefined on exit; both calls need the same, which may be 0 bytes (then NULL will do). */
lp_status lp_grad_norm(int32_t n, const lp_gradient* grads, float* norm, void* workspace, size_t workspace_bytes, void* stream);
/* max_norm and eps: finite, >= 0.  An out that overlaps another tensor of the call, `norm` or a part of its own in is refused. */
lp_status lp_clip_grad_norm(int32_t n, const lp_gradient* grads, float max_norm, float eps, float* norm, void* workspace,
                            size_t workspace_bytes, void* stream);
lp_status lp_grad_norm_workspace_bytes(int32_t n, const lp_gradient* grads, size_t* bytes);

/* ---- Orthogonalised updates of weight matrices --------------------------------------------------
 *
 * The step of the Muon optimiser (Jordan et al. 2024) for the weight matrices whose gradients the
 * backward calls above accumulate, and for those of networks around them.  A matrix G (rows x cols) is
 * replaced by what a few Newton-Schulz products make of it, which moves all its singular values towards 1:
 *     X_0 = G / (||G||_F + eps),   A = X X^T,   X <- a X + (b A + c A A) X,   `steps` times
 * (of a matrix with more rows than columns: on the transpose).  A matrix of zeros gives zeros.
 * Products are computed on the matrix cores with operands as fp16 hi + lo parts at a power-of-two scale (22
 * bits, three products, fp32 accumulation); against 64 bits the result's error is 0.7 to 1.14 times that of fp32 products.
 */
#define LP_ORTH_MAX_STEPS 16

typedef struct {
    int32_t steps;       /* 1 .. LP_ORTH_MAX_STEPS */
    const float* coeffs; /* HOST [steps][3]: a, b, c of every step; NULL: 3.4445, -4.775, 2.0315 in every step.
                            Coefficients under which a singular value in [0, 1] could leave [0, 1024] are refused. */
    float eps;           /* >= 0, finite */
} lp_orth;

/* `count` matrices of one shape, one behind the other: element (i, r, c) at (i rows + r) cols + c. */
typedef struct {
    int64_t count;
    int32_t rows, cols;
    const void* in; /* device, elements of type `dtype` */
    void* out;      /* device, elements of type `dtype`; may be `in` */
    int32_t dtype;  /* lp_dtype */
} lp_matrices;

/* Orthogonalises n lists of matrices.  `lists` is a HOST array; outputs are WRITTEN.  workspace: device,
   256-byte aligned, contents ignored on entry, undefined on exit.  n == 0 is a no-op, and so is a list with
   count, rows or cols 0.  Lists are worked on at the same time: an out that overlaps another list's in or out,
   or a part of its own in, is refused. */
lp_status lp_orthogonalize(int32_t n, const lp_matrices* lists, const lp_orth* orth, void* workspace,
                           size_t workspace_bytes, void* stream);
/* 0 where all matrices are at most 64 x 224 or 32 x 448, or their transposes (then NULL will do).
   The result of a matrix of at most 64 x 128, or its transpose, does not depend on what else the call holds;
   others' last bits may (the order of their sums follows the work of the whole call). */
lp_status lp_orthogonalize_workspace_bytes(int32_t n, const lp_matrices* lists, size_t* bytes);

/* How the step of a matrix is scaled. */
typedef enum {
    LP_MUON_SCALE_NONE = 0,
    LP_MUON_SCALE_ASPECT = 1, /* sqrt(max(1, rows / cols)) */
    LP_MUON_SCALE_RMS = 2     /* 0.2 sqrt(max(rows, cols)): steps as large as Adam's */
} lp_muon_scale;

typedef struct {
    float lr, momentum, weight_decay; /* finite */
    int32_t nesterov;                 /* 0 or 1 */
    int32_t scale;                    /* lp_muon_scale */
    lp_orth orth;
} lp_muon;

/* fp32 weights with their gradient and momentum, laid out as in lp_matrices. */
typedef struct {
    int64_t count;
    int32_t rows, cols;
    float* weight;     /* device, updated */
    const float* grad; /* device */
    float* momentum;   /* device, updated; zeros before the first step */
} lp_muon_weights;

/* One step over n lists of weights:
     M <- momentum M + G,   U = G + momentum M (nesterov) or M,
     W <- (1 - lr weight_decay) W - lr s orthogonalised(U).
   Lists may share a gradient; a weight or momentum that overlaps anything else of the call is refused. */
lp_status lp_muon_step(int32_t n, const lp_muon_weights* lists, const lp_muon* muon, void* workspace,
                       size_t workspace_bytes, void* stream);
lp_status lp_muon_workspace_bytes(int32_t n, const lp_muon_weights* lists, size_t* bytes);

/* Diagnostics, not part of the method: how one SIMD of this GPU overlaps matrix instructions
   (32x32x16 bf16 products, 32 cycles each) with vector instructions (4 cycles each); the split of
   the Renderer's backward into two waves per ray follows from it.  ns_per_iteration (host, 10
   floats) receives nanoseconds per loop iteration of
     [0..3]  one wave per SIMD issuing one product followed by 0, 4, 8, 12 independent vector
             multiply-adds (a sum 32 + 4 K cycles means no overlap inside a wave);
     [4..6]  two waves per SIMD, waves w and w + 4 of a workgroup paired: the first issues 8 products
             per iteration, the second 64 multiply-adds; only the first works, only the second, both;
     [7..9]  the same with waves w and w + 1 paired.
   Allocates and frees a small device buffer; synchronises the stream. */
lp_status lp_diag_coexecution(float* ns_per_iteration, void* stream);

/* Diagnostics, not part of the method: the rate at which this GPU retires fp32 atomic adds that cover
   whole 64-byte lines (16 lanes per line), the unit the gradient scatter of the backward works in
   (Section 3.4: the backward adds every sample's feature gradient into the structure).
   lines_per_second (host, 6 floats): lines drawn at random from 256 MiB with 4, 2, 1 lines per
   instruction [0..2]; from 256 KiB with 4 lines per instruction [3]; neighbouring lines (a walk) in
   256 MiB and in 256 KiB [4..5].  Allocates and frees 256 MiB of device memory; synchronises the
   stream. */
lp_status lp_diag_atomic_rate(float* lines_per_second, void* stream);

/* Diagnostics of a MEASUREMENT build (the library compiled with -DLP_WS_PHASES; an ordinary build
   returns LP_ERR_UNSUPPORTED): cycles the two roles of the two-wave backward have spent in the
   phases of their steps since the last call, summed over all waves.  cycles (host, 32 values):
   [0..10] chain wave (step start, sampling issue, forward, hand-over of h1 and h2, Eq. (2), hand-over
   of the output gradients, first link of the input-gradient chain, hand-over of dZ2, second link,
   hand-over of the features, records and dZ1, interpolation of the next step's features),
   [16..26] weights wave (step start, h2 taken and transposed, wait for the output gradients, dWo, h1
   transposed, wait for dZ2, dW2, features taken and transposed, wait for dZ1, feature gradient and
   dW1, walk).  The sums are cleared by the call. */
lp_status lp_diag_ws_phases(unsigned long long* cycles);

/* Message of the last failure on this thread ("" if none).  Owned by the library. */
const char* lp_last_error(void);

/* Library version, major * 1000 + minor. */
int32_t lp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LIGHTPLANE_H */
