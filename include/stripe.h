/*
 * stripe.h -- C ABI of the MI355X (gfx950) executor for one Stripe block.
 *
 * A Stripe block (paper, Section 3.2) is a parallel polyhedral block
 * (Section 3.1.2, Definition 2): a list of indexes with one range each, a
 * list of affine constraints "expr >= 0", a single statement list, and the
 * buffers it reads and writes, each with an aggregation operation.  Blocks
 * nest (Section 3.1.3): a statement may be another block, which sees its
 * parent's buffers only through refinements -- offset, sized and strided
 * views -- and its parent's indexes only as explicitly passed affine values
 * (Figure 5b).  This library evaluates such a nest whose leaf statement list
 * is  load, [load, mul|add,] store  on one GPU.
 *
 * All descriptor memory is HOST memory owned by the caller; create() copies
 * what it needs, so the descriptor may be freed right after it returns.
 * Buffers handed to run() are DEVICE pointers owned by the caller.  No
 * function throws or aborts; every failure is a status code, with detail in
 * stripe_last_error().  Apart from that thread-local string the library keeps
 * no global state; handles are independent of each other.
 */
#ifndef STRIPE_H
#define STRIPE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STRIPE_OK = 0,
  STRIPE_ERR_NULL = 1,            /* a required pointer argument is NULL */
  STRIPE_ERR_INVALID_DESC = 2,    /* malformed descriptor (counts, ranges, shapes, type mix) */
  STRIPE_ERR_UNSUPPORTED = 3,     /* a legal block this library cannot run (yet) */
  STRIPE_ERR_OUT_OF_BOUNDS = 4,   /* an access inside the polyhedron may leave its buffer or view */
  STRIPE_ERR_ASSIGN_CONFLICT = 5, /* 'assign' level whose iterations are not provably disjoint */
  STRIPE_ERR_HIP = 6,             /* a HIP runtime call failed */
  STRIPE_ERR_NOMEM = 7,           /* out of host or device memory, or a workspace / the static scratch is too small */
  STRIPE_ERR_MISALIGNED = 8       /* a buffer pointer lacks the 16-byte alignment the planned kernel family needs */
} stripe_status_t;

typedef enum { STRIPE_I8 = 0, STRIPE_I32 = 1, STRIPE_BF16 = 2, STRIPE_F32 = 3 } stripe_dtype_t;

/* Aggregation operations (Section 2.1 last sentence; Section 3.2: 'assign'
 * declares that no two iterations write the same element). */
typedef enum {
  STRIPE_AGG_ASSIGN = 0, STRIPE_AGG_ADD = 1, STRIPE_AGG_MAX = 2, STRIPE_AGG_MIN = 3,
  STRIPE_AGG_MUL = 4   /* product; integer products wrap in int32 like any int32 arithmetic here */
} stripe_agg_t;

/* Leaf statement lists (Section 3.2 "intrinsics"; Figure 5, the four statements of the inner block):
 *   MUL : $a = load(in0); $b = load(in1); $o = mul($a,$b); out = store($o)
 *   ADD : the same with add
 *   COPY: $a = load(in0); out = store($a)
 *   ADD_RELU: $a = load(in0); $b = load(in1); $o = relu(add($a,$b)); out = store($o)   (relu(v) = max(v, 0)) */
typedef enum { STRIPE_INTR_MUL = 0, STRIPE_INTR_COPY = 1, STRIPE_INTR_ADD = 2, STRIPE_INTR_ADD_RELU = 3 } stripe_intrinsic_t;

/* TEMP: only at the root of a block with several statements: a buffer the library owns, written by one statement
 * and read by later ones.  The caller passes no pointer for it. */
typedef enum { STRIPE_IN = 0, STRIPE_OUT = 1, STRIPE_TEMP = 2 } stripe_dir_t;

/* Which kernel family runs the block (reported by stripe_block_query). */
typedef enum {
  STRIPE_PATH_AUTO = 0,      /* create: let the planner choose */
  STRIPE_PATH_GENERIC = 1,   /* affine-index contraction, any legal block */
  STRIPE_PATH_MFMA_GEMM = 2, /* nested-tile dense contraction on matrix cores */
  STRIPE_PATH_MFMA_CONV = 3, /* nested-tile convolution-shaped contraction on matrix cores */
  STRIPE_PATH_POOL = 4       /* max aggregation over a window of one input */
} stripe_path_t;

/*
 * One refinement (Section 3.2, "refinements"; Figure 5 "in I[3*x - 1, 4*y - 1, 0]
 * i8(5, 6, 8):(128, 8, 1)"): a buffer as one nesting level sees it.
 *   access_coeff [ndim][n_vars] row-major, access_const [ndim]:
 *       per dimension the affine origin of the view, in this level's variables
 *       (own indexes first, then passed values), measured from the origin of
 *       the view the level itself received.  The absolute coordinate of a
 *       leaf access is the sum over all levels.
 *   sizes [ndim]: extent of the view handed to this level's statements
 *       (root level: the extent of the buffer itself; leaf: all 1).  A view
 *       may hang over the edge of its parent (halo tiles); only accesses that
 *       are executed must fall inside every enclosing view and the buffer.
 *   strides [ndim]: in elements, non-negative, identical at every level.
 *   agg: aggregation of the output at this level; each level carries the
 *       nest's single operation or ASSIGN.  Ignored for inputs.
 */
typedef struct {
  stripe_dir_t dir;
  stripe_dtype_t dtype;
  stripe_agg_t agg;
  int32_t ndim;                /* 1..8 */
  const int64_t* access_coeff;
  const int64_t* access_const;
  const int64_t* sizes;
  const int64_t* strides;
} stripe_refinement_t;

/*
 * One nesting level (Section 3.2 first paragraph; Figure 5).
 * The outermost descriptor is the declaring root block ("block []:1"):
 * n_idx = n_passed = n_constraints = 0, its refinements give the buffers'
 * extents, strides and element types, access_const is the element offset of
 * the origin (normally 0) and access_coeff is unused.  Below it come 1..6
 * block levels; the last one (child == NULL) holds the intrinsic.
 * Every level lists the same buffers in the same order: inputs first (one for
 * COPY, two for MUL/ADD), the single output last.
 * Element types: inputs i8/i32 with an i32 output, or bf16/f32 with an f32
 * or bf16 output (rounded to nearest even on store).  Integer arithmetic is exact two's-complement int32 (operands
 * sign-extended before the multiply); float blocks accumulate in fp32.
 */
typedef struct stripe_block_desc {
  int32_t n_idx;
  const int64_t* ranges;        /* [n_idx]; index j takes 0 .. ranges[j]-1; 0 = empty block */
  int32_t n_passed;
  const int64_t* passed_coeff;  /* [n_passed][parent n_vars]: value = row . parent vars + const */
  const int64_t* passed_const;  /* [n_passed] */
  int32_t n_constraints;
  const int64_t* cons_coeff;    /* [n_constraints][n_vars]: row . vars + const >= 0 */
  const int64_t* cons_const;    /* [n_constraints] */
  int32_t n_refs;
  const stripe_refinement_t* refs;
  stripe_intrinsic_t intrinsic; /* leaf only */
  const struct stripe_block_desc* child;
  /* Statement lists (Section 3.2: a block may hold several statements, executed as if in serial).  Supported
   * at the root only: root->child is the first statement, ->next the following ones (NULL ends the list).
   * A statement of a list names the root refinements it uses, inputs first and its output last, in
   * parent_refs[n_refs]; with a single statement parent_refs may be NULL (same positions).  Root refinements
   * then come in the order: the caller's inputs, temporaries (STRIPE_TEMP), the single output last. */
  const struct stripe_block_desc* next;
  const int32_t* parent_refs;
} stripe_block_desc_t;          /* n_vars of a level = n_idx + n_passed */

typedef struct stripe_block stripe_block_t; /* opaque handle */

/* What the planner decided; algorithmic figures count in-polyhedron points only. */
typedef struct {
  int32_t path;               /* stripe_path_t actually used */
  int32_t n_idx;              /* indexes after flattening and merging */
  int32_t n_out_idx;          /* indexes the output address depends on */
  int32_t n_red_idx;          /* reduction indexes */
  int64_t hull_points;        /* product of the flattened ranges */
  int64_t work_points;        /* points meeting all constraints; -1 if not counted */
  int64_t output_elements;    /* distinct output elements the hull can write */
  int64_t algorithmic_bytes;  /* each input and output element once */
  int32_t tile_m, tile_n, tile_k;   /* workgroup tile of the nested-tile paths, else 0 */
  int32_t frag_m, frag_n, frag_k;   /* matrix-core fragment, else 0 */
  int32_t lds_bytes;
  int32_t workgroup_size;
  int64_t grid;               /* workgroups per launch */
  char kernel[96];            /* name of the kernel variant */
  int64_t workspace_bytes;    /* device workspace the handle's launches use (see stripe_block_set_workspace); 0 = none */
} stripe_block_info_t;

/*
 * Validate, flatten and plan a block (host only, no GPU call).
 * Flattening composes refinement offsets down the nest and substitutes passed
 * values (Section 3.1.3), so a tiled nest and its un-tiled form plan alike.
 * Every access is proven to stay inside its buffer and views for all points
 * of the polyhedron, otherwise STRIPE_ERR_OUT_OF_BOUNDS.
 * On success *out receives a handle the caller must release with
 * stripe_block_destroy().
 */
stripe_status_t stripe_block_create(const stripe_block_desc_t* desc, stripe_block_t** out);

/* As stripe_block_create, but forces a kernel family (STRIPE_PATH_AUTO = planner's
 * choice).  STRIPE_ERR_UNSUPPORTED if the block does not have that family's shape. */
stripe_status_t stripe_block_create_for_path(const stripe_block_desc_t* desc, stripe_path_t path,
                                             stripe_block_t** out);

/*
 * Launch the block on `hip_stream` (a hipStream_t; NULL = the default stream)
 * of the current device.  inputs[i] is the DEVICE pointer of the i-th input
 * refinement's buffer origin, output that of the output buffer; element types
 * and extents as declared at the root.  Output elements no iteration writes
 * keep their contents; written elements are overwritten (prior contents do
 * not enter the aggregation).  A block whose output elements are shared
 * between index tuples through different output indexes (O[x + i]) is run as
 * two launches: the aggregation's identity to every reached element, then an
 * atomic combine; sums of products over O[s*x + i] with x of one input and i of
 * the other are rewritten to one owner per element instead, one launch that
 * stores each element once.  A statement list runs its statements in order on
 * the stream.
 * Workspace: temporaries of a statement list that are not fused away, and
 * the partial sums of a dense contraction whose reduction index is split
 * over workgroups (Section 2.1: aggregations are associative and commutative,
 * so a reduction may be regrouped; chosen at create for products with few
 * output tiles and a long reduction), live in a device workspace of
 * stripe_block_workspace_size() bytes.  If the caller has handed one over
 * with stripe_block_set_workspace(), run() uses it and never allocates;
 * otherwise the handle allocates it on its first run on a device (the only
 * allocation run() ever makes; that first call then is not purely
 * asynchronous) and frees it on destroy.  A first run under graph capture
 * cannot allocate: products with at most 32 rows are then recorded on a kernel
 * that needs no workspace, anything else is to be run once before.  Either way two overlapping runs of
 * one handle race on the workspace.  Handles that report 0 bytes never
 * allocate.
 * Alignment: the specialised kernel families move 16 bytes per lane.
 * Whether a block's strides and origins keep that alignment is decided at
 * create (a block that does not runs on the generic kernels, which take
 * any element-aligned pointer); the buffer POINTERS are only seen here, and a
 * pointer that is not 16-byte aligned, handed to a handle planned for a
 * specialised family (path != STRIPE_PATH_GENERIC in stripe_block_query),
 * is refused with STRIPE_ERR_MISALIGNED before anything is launched.
 * Non-finite inputs are outside the contract of the specialised families:
 * they realise constraints by feeding zeros for removed points (0 * Inf is
 * NaN where the definition skips the point) and use IEEE maxNum/minNum for
 * max/min (a NaN operand is ignored).
 * Asynchronous: returns after enqueueing; only launch errors are reported.
 * Calls on different handles may overlap; two overlapping calls that write
 * the same output buffer race.
 */
stripe_status_t stripe_block_run(stripe_block_t* blk, const void* const* inputs, void* output,
                                 void* hip_stream);

/*
 * stripe_block_run for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same launches, but the handle's workspace (temporaries of a
 * statement list, partial sums of a split reduction) lives in a fixed array of STRIPE_STATIC_SCRATCH_BYTES that
 * is part of the library's code object (each GPU the library runs on holds its own copy until the process
 * ends) instead of memory the handle allocates on its first run; a workspace set with
 * stripe_block_set_workspace is not used by this call.
 * The call makes no hipMalloc / hipFree and calls no allocating library routine; the caller still passes inputs
 * and output.  If stripe_block_workspace_size() exceeds STRIPE_STATIC_SCRATCH_BYTES the call returns
 * STRIPE_ERR_NOMEM and launches nothing (use stripe_block_run then), unless the part beyond it is the partial sums of
 * products with at most 32 rows, which this call then runs on a kernel that needs none.  Handles that need no workspace
 * use no scratch at all.
 * Every call on a GPU shares that GPU's array, which keeps the previous call's contents; nothing in it needs to
 * start at zero (every element of a temporary or of a partial-sum image is written before it is read).  Two
 * calls that overlap on one GPU (different streams, or different host threads) and both need a workspace RACE
 * on the array: serialise them on one stream.  The array's device address is looked up on the first call on
 * each device.
 */
#define STRIPE_STATIC_SCRATCH_BYTES (8u << 20)
stripe_status_t stripe_block_run_static(stripe_block_t* blk, const void* const* inputs, void* output, void* hip_stream);

/*
 * The device workspace of a handle (see stripe_block_run).  workspace_size: bytes the handle's launches need, 0
 * if none.  set_workspace: `device_ptr` (256-byte aligned DEVICE memory of at least that many bytes, owned by
 * the caller, valid until replaced or the handle is destroyed) becomes the workspace of every later
 * stripe_block_run, which then never allocates; NULL returns to handle-owned memory.  STRIPE_ERR_NOMEM if
 * `bytes` is too small, STRIPE_ERR_INVALID_DESC if misaligned.  Host only.
 */
stripe_status_t stripe_block_workspace_size(const stripe_block_t* blk, size_t* bytes);
stripe_status_t stripe_block_set_workspace(stripe_block_t* blk, void* device_ptr, size_t bytes);

stripe_status_t stripe_block_query(const stripe_block_t* blk, stripe_block_info_t* info);

void stripe_block_destroy(stripe_block_t* blk);

const char* stripe_status_string(stripe_status_t status);

/* Detail of the last failure on the calling thread ("" if none).  The pointer
 * stays valid until the next failing call on this thread. */
const char* stripe_last_error(void);

/*
 * Bandwidth yardstick: copies n_bytes (a multiple of 16, both pointers
 * 16-byte aligned DEVICE memory) with a plain grid-stride 16-byte-per-lane
 * kernel on `hip_stream`.  Used to scale hardware traffic counters and to
 * state the achievable HBM rate next to the pooling kernels.
 */
stripe_status_t stripe_device_copy(const void* src, void* dst, size_t n_bytes, void* hip_stream);

/*
 * Streaming yardsticks with a chosen read : write mix: `reads` input streams (0, 1, 2 or 4) of n_vectors 16-byte
 * vectors each, laid one after the other from `src`, are added into one output stream of n_vectors vectors at
 * `dst` (write != 0), or only read (write == 0; dst then points at 4 spare bytes).  Streaming loads and stores, four
 * independent vectors per lane and trip, `grid` workgroups of 256 lanes.  DEVICE pointers, 16-byte aligned.  They
 * state what a perfectly regular kernel with the window kernels' 4 : 1 mix reaches on this chip.
 */
stripe_status_t stripe_device_stream(const void* src, void* dst, size_t n_vectors, int reads, int write, int grid, void* hip_stream);

/*
 * Matrix-core yardstick: every wavefront of `grid` workgroups of 256 lanes runs `iters` (even) passes over a
 * 4 x 4 tile of 32 x 32 x 16 bf16 matrix instructions whose operand fragments stay in registers (no LDS or global
 * traffic inside the loop): iters * 16 instructions = iters * 524,288 flop per wavefront, 4 wavefronts per
 * workgroup.  `operands`: DEVICE, 16-byte aligned, 16 * 256 vectors of 8 bf16 (64 KB): vector (s * 8 + f) * 256 + lane
 * is fragment f (0-3: A, 4-7: B) of operand set s (0, 1; the sets alternate from pass to pass) for lane `lane` of
 * the workgroup.  `out`: DEVICE, grid * 256 floats; each receives the sum of its lane's 256 accumulator elements.
 * from_lds != 0: the fragments are parked in LDS and fetched again before every pass (eight 16-byte reads per lane
 * for sixteen instructions, the contraction kernels' ratio) instead of staying in registers.
 * It states what the chip sustains for the contraction kernels' instruction on given operand values, apart from
 * the memory system (Section 3.3's roofline speaks of the compute roof; this measures it).
 */
stripe_status_t stripe_device_mfma(const void* operands, void* out, int iters, int from_lds, int grid, void* hip_stream);

/* ------------------------------------------------------------------------
 * Layers: the operators of a transformer's feed-forward block that are no
 * single Stripe block -- the linear layer with its epilogue, the same over
 * rows sorted by expert (a data-dependent, hence not affine, index space), the
 * layer norm, the gated unit, the cross entropy of a linear head -- each with its
 * gradients, and the step of the optimizer, AdamW.  Handles work like those of blocks:
 * create() validates and plans on the host, run() / backward() enqueue on
 * `hip_stream` of the current device and return, the workspace is the caller's
 * (set_workspace) or the handle's.
 *
 * Common to all of them:
 *  - buffers are DEVICE pointers, aligned to their element type; a pointer that
 *    is not is refused (STRIPE_ERR_MISALIGNED).  16-byte aligned pointers,
 *    strides and feature counts run faster kernels, nothing else depends on them;
 *  - sums, statistics and totals are fp32 (or wider); a bf16 result is rounded to
 *    nearest even once, on store; zeros, infinities and NaN go the way the formula sends them.  A bf16 linear layer's
 *    dz is rounded to bf16 before dx and dW are computed from it (db adds it up unrounded);
 *  - values of an activation that are smaller than 2^-118 may be 0;
 *  - a linear layer's fp32 products may be computed as three bf16 parts per value (large ones are: the kernels' names
 *    in stripe_linear_info_t then say "parts"), which hold all
 *    24 bits down to 2^-110; of smaller values they lose what lies below 2^-133;
 *  - a layer norm's squared distances are fp32: a row where their sum passes fp32's largest value has s = 0;
 *  - outputs must not overlap inputs or one another, except where stated (the same
 *    address is refused with STRIPE_ERR_INVALID_DESC, other overlaps are not looked for);
 *  - the same call on the same inputs gives the same bits (no atomics);
 *  - a bf16 gated unit and cross entropy round their dz as the linear layer does;
 *  - a call that needs a workspace and has none of the caller's allocates it, once per
 *    device, and keeps it until the handle is destroyed; under graph capture such a first call
 *    is refused with STRIPE_ERR_NOMEM before anything is launched.  Calls (or
 *    graph replays) of one handle that overlap race on the workspace unless each was
 *    recorded with a workspace of its own; calls that need none may overlap.
 */
typedef enum {
  STRIPE_ACT_NONE = 0,       /* z */
  STRIPE_ACT_RELU = 1,       /* max(z, 0); its derivative at 0 is 0 */
  STRIPE_ACT_GELU = 2,       /* z Phi(z), Phi the normal distribution function */
  STRIPE_ACT_GELU_TANH = 3,  /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
  STRIPE_ACT_SILU = 4        /* z / (1 + exp(-z)) */
} stripe_activation_t;

/*
 * Linear layer:  z = x W^T + b,  y = act(z) + r,  and its gradients for a given dy
 *   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum of dz over the rows      (dr = dy).
 * x [rows][in_features], W [out_features][in_features], y and r [rows][out_features], b [out_features] in fp32.
 * groups > 0: rows sorted by expert.  W [groups][out_features][in_features], b [groups][out_features], and `offsets`,
 * groups + 1 int32 values on the DEVICE: rows offsets[g] .. offsets[g+1] - 1 meet W[g] and b[g].  Rows outside
 * every group keep what y, pre and dx hold there; a group without rows gets dW[g] = 0, db[g] = 0.  Values
 * are read as their running maximum, limited to 0 .. rows, so that no sequence of them leads outside the buffers.
 */
typedef struct {
  int64_t rows;                        /* 0 .. 2^28 */
  int64_t in_features, out_features;   /* 1 .. 2^24 */
  int32_t groups;                      /* 0: one matrix for all rows; else 1 .. 4096 matrices */
  stripe_dtype_t dtype;                /* of x, W, r, y, pre, dy, dx, dW: STRIPE_BF16 or STRIPE_F32 */
  stripe_activation_t activation;
  /* Strides in elements, 0 = dense.  x_row: rows of x and dx; w_row, w_group: rows and matrices of W and dW;
   * y_row: rows of y, r, pre and dy. */
  int64_t x_row, w_row, w_group, y_row;
} stripe_linear_desc_t;

typedef struct stripe_linear stripe_linear_t;

typedef struct {
  char forward[96], input_grad[96], weight_grad[96];   /* kernels that 16-byte aligned buffers run on */
  int64_t workspace_bytes;
} stripe_linear_info_t;

stripe_status_t stripe_linear_create(const stripe_linear_desc_t* desc, stripe_linear_t** out);

/* bias, residual, pre may be NULL (no b, no r, z not stored); pre receives z in `dtype`, for a later backward pass.
 * offsets: NULL without groups.  residual may be y itself. */
stripe_status_t stripe_linear_run(stripe_linear_t* lin, const void* x, const void* w, const float* bias, const void* residual, const int32_t* offsets,
                                  void* y, void* pre, void* hip_stream);

/* dx, dw, dbias: any of them may be NULL (not computed), then x, w may be NULL where only that gradient reads them.
 * pre: z as run() stored it; NULL only with STRIPE_ACT_NONE. */
stripe_status_t stripe_linear_backward(stripe_linear_t* lin, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx,
                                       void* dw, float* dbias, void* hip_stream);

stripe_status_t stripe_linear_workspace_size(const stripe_linear_t* lin, size_t* bytes);
stripe_status_t stripe_linear_set_workspace(stripe_linear_t* lin, void* device_ptr, size_t bytes);   /* as stripe_block_set_workspace */
stripe_status_t stripe_linear_query(const stripe_linear_t* lin, stripe_linear_info_t* info);
void stripe_linear_destroy(stripe_linear_t* lin);

/*
 * Layer norm over the features of a row:  m = mean(x),  s = (mean((x - m)^2) + eps)^(-1/2),  h = (x - m) s,
 *   y = h gamma + beta;   with g = dy gamma:  dx = s (g - mean(g) - h mean(g h)),  dgamma = sum of dy h over the rows,
 *   dbeta = sum of dy.
 * gamma, beta, their gradients, m and s are fp32.
 */
typedef struct {
  int64_t rows;             /* 0 .. 2^30 */
  int64_t features;         /* 1 .. 2^24 */
  stripe_dtype_t dtype;     /* of x, y, dy, dx: STRIPE_BF16 or STRIPE_F32 */
  double eps;               /* >= 0 and finite */
  int64_t x_row, y_row;     /* strides in elements, 0 = dense: rows of x and dx, rows of y and dy */
} stripe_norm_desc_t;

typedef struct stripe_norm stripe_norm_t;

stripe_status_t stripe_norm_create(const stripe_norm_desc_t* desc, stripe_norm_t** out);

/* gamma, beta may be NULL (1, 0); mean, rstd [rows] may be NULL (not stored).  y may be x itself where the row strides agree. */
stripe_status_t stripe_norm_run(stripe_norm_t* norm, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                                void* hip_stream);

/* mean, rstd: as run() stored them.  dx, dgamma, dbeta: any of them may be NULL. */
stripe_status_t stripe_norm_backward(stripe_norm_t* norm, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                                     float* dgamma, float* dbeta, void* hip_stream);

stripe_status_t stripe_norm_workspace_size(const stripe_norm_t* norm, size_t* bytes);
stripe_status_t stripe_norm_set_workspace(stripe_norm_t* norm, void* device_ptr, size_t bytes);
void stripe_norm_destroy(stripe_norm_t* norm);

/*
 * Gated unit:  [g | u] = x W^T,  y = act(g) u,  and its gradients for a given dy
 *   dg = dy u act'(g),  du = dy act(g),  dz = [dg | du],  dx = dz W,  dW = dz^T x.
 * x [rows][in_features], y [rows][out_features]; W [2 out_features][in_features]: the gate's rows, then up's; pre = [g | u], [rows][2 out_features].
 * groups > 0: rows sorted by expert, W [groups][2 out_features][in_features] and `offsets` as for the linear layer.
 * y is computed from g and u as they were before pre's rounding; dz is rounded to the operands' type before its products.
 */
typedef struct {
  int64_t rows;                        /* 0 .. 2^28 */
  int64_t in_features, out_features;   /* 1 .. 2^24, 1 .. 2^23 */
  int32_t groups;                      /* 0: one matrix for all rows; else 1 .. 4096 matrices */
  stripe_dtype_t dtype;                /* of x, W, y, pre, dy, dx, dW: STRIPE_BF16 or STRIPE_F32 */
  stripe_activation_t activation;      /* STRIPE_ACT_NONE: y = g u */
  /* Strides in elements, 0 = dense.  x_row: rows of x and dx; w_row, w_group: rows and matrices of W and dW; y_row: rows of y and dy;
   * pre_row: rows of pre. */
  int64_t x_row, w_row, w_group, y_row, pre_row;
} stripe_gated_desc_t;

typedef struct stripe_gated stripe_gated_t;

stripe_status_t stripe_gated_create(const stripe_gated_desc_t* desc, stripe_gated_t** out);

/* offsets: NULL without groups.  pre may be NULL (not stored); it receives g and u in `dtype`, for a later backward pass. */
stripe_status_t stripe_gated_run(stripe_gated_t* gated, const void* x, const void* w, const int32_t* offsets, void* y, void* pre, void* hip_stream);

/* pre: as run() stored it.  dx, dw: either of them may be NULL (not computed), then w or x may be NULL. */
stripe_status_t stripe_gated_backward(stripe_gated_t* gated, const void* dy, const void* x, const void* w, const void* pre, const int32_t* offsets, void* dx,
                                      void* dw, void* hip_stream);

stripe_status_t stripe_gated_workspace_size(const stripe_gated_t* gated, size_t* bytes);
stripe_status_t stripe_gated_set_workspace(stripe_gated_t* gated, void* device_ptr, size_t bytes);
stripe_status_t stripe_gated_query(const stripe_gated_t* gated, stripe_linear_info_t* info);
void stripe_gated_destroy(stripe_gated_t* gated);

/*
 * Softmax cross entropy of a linear head, e.g. over a vocabulary, without keeping its logits:
 *   z = x W^T,  lse = log(sum of exp(z) over the classes),  loss = lse - z[target];
 *   dz = exp(z - lse) (dloss + dlse) - [class = target] dloss,  dx = dz W,  dW = dz^T x.
 * x [rows][in_features], W [classes][in_features]; targets [rows]: int32 on the DEVICE; loss, lse, dloss, dlse [rows]: fp32.
 * A row whose target is not one of 0 .. classes - 1 does not count: loss, lse and dx are 0, dW has nothing of it, and whatever x holds there
 * (NaN, too) changes no bit of any result.  Logits may be of any finite size: exponentials are taken of distances, as the hardware's one of base 2 of the
 * distance times log2 e, both in fp32 (f32 gradients: expf).  The backward pass computes z again, a piece of the vocabulary at a time (exp(z - lse) is
 * at most 1, whatever the two sums' roundings); a piece's dz is in the workspace, rounded to the operands' type.  In bf16 it is divided by the rows'
 * largest |dloss| or |dloss + dlse| before and multiplied by it in dx and dW: of rows whose weights are less than 2^-110 of that, digits may be
 * lost.  dx is added up in fp32 over the pieces.
 */
typedef struct {
  int64_t rows;             /* 0 .. 2^24 */
  int64_t in_features;      /* 1 .. 2^20 */
  int64_t classes;          /* 1 .. 2^24 */
  stripe_dtype_t dtype;     /* of x, W, dx, dW: STRIPE_BF16 or STRIPE_F32 */
  int64_t x_row, w_row;     /* strides in elements, 0 = dense: rows of x and dx, rows of W and dW */
} stripe_xent_desc_t;

typedef struct stripe_xent stripe_xent_t;

stripe_status_t stripe_xent_create(const stripe_xent_desc_t* desc, stripe_xent_t** out);

/* loss, lse: either of them may be NULL. */
stripe_status_t stripe_xent_run(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, float* loss, float* lse, void* hip_stream);

/* lse: as run() stored it for the same x, W and targets.  dloss: the gradient of every row's loss, NULL: ones; dlse: that of lse, NULL: zeros.
 * dx, dw: either of them may be NULL. */
stripe_status_t stripe_xent_backward(stripe_xent_t* xent, const void* x, const void* w, const int32_t* targets, const float* lse, const float* dloss,
                                     const float* dlse, void* dx, void* dw, void* hip_stream);

stripe_status_t stripe_xent_workspace_size(const stripe_xent_t* xent, size_t* bytes);
stripe_status_t stripe_xent_set_workspace(stripe_xent_t* xent, void* device_ptr, size_t bytes);
/* forward: the logits' kernel, which both passes run; input_grad, weight_grad: those of a piece of the vocabulary. */
stripe_status_t stripe_xent_query(const stripe_xent_t* xent, stripe_linear_info_t* info);
void stripe_xent_destroy(stripe_xent_t* xent);

/*
 * AdamW over many tensors:  with t = step and g = factor grad,
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
 * p, m, v are updated in place; `copy`, where a tensor has one, receives p in bf16.  All tensors are contiguous.
 * state_dtype STRIPE_F32: m, v fp32.  STRIPE_I8: blocks of 256 consecutive elements; m is m_scale[block] c |c| with c = m[i] in -127 .. 127 (int8), the square
 * root of v is v_scale[block] c^2 with c = v[i] in 0 .. 255 (uint8); m_scale, v_scale: fp32, ceil(elements / 256).  All zeros is the state before the first
 * step.  A value between two codes becomes one of them at random, such that its mean is kept (a square root of v that is not 0 does not become 0); the random
 * bits are a hash of (seed, the tensor's number, the element's modulo 2^32), so that the same call gives the same bits: give every step another seed.  A block whose
 * largest value is at most 1e-30 becomes 0, one that holds a value that is not finite becomes NaN as a whole.  p's update uses m and v
 * before they are coded.
 */
typedef struct {
  int32_t tensors;                  /* 0 .. 2^20 */
  const int64_t* elements;          /* [tensors], 0 .. 2^34 */
  const double* weight_decay;       /* [tensors] wd, or NULL: 0 */
  stripe_dtype_t grad_dtype;        /* STRIPE_BF16 or STRIPE_F32 */
  stripe_dtype_t state_dtype;       /* STRIPE_F32 or STRIPE_I8 */
  double beta1, beta2;              /* 0 <= b < 1 */
  double eps;                       /* 0, or at least 2^-126 and finite */
} stripe_adamw_desc_t;

typedef struct {
  float* p;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;         /* STRIPE_I8 only, else NULL */
  void* copy;                       /* bf16, or NULL */
} stripe_adamw_tensor_t;

typedef struct {
  double lr;
  int64_t step;                     /* t: 1 .. 2^53 */
  double factor;                    /* of the gradients, e.g. what limits their norm; 1: none */
  uint32_t seed;                    /* STRIPE_I8 */
  /* NULL, or five 4-byte values on the DEVICE that are read when the step runs, in place of the four above (which are then ignored): fp32 lr,
   * 1 / (1 - b1^t), 1 / sqrt(1 - b2^t), factor; uint32 seed.  For steps that are captured once and replayed. */
  const void* control;
} stripe_adamw_step_t;

typedef struct stripe_adamw stripe_adamw_t;

stripe_status_t stripe_adamw_create(const stripe_adamw_desc_t* desc, stripe_adamw_t** out);

/* The tensors that the steps update, desc.tensors of them (the pointers of one without elements are not looked at): kept until the next call of bind(),
 * which no step may overlap on the host.  A call checks every tensor: keep the buffers of gradients and bind once; a program whose gradients move binds before each step.  No buffer may be bound twice (the same address is refused), but two gradients may be one. */
stripe_status_t stripe_adamw_bind(stripe_adamw_t* adamw, const stripe_adamw_tensor_t* tensors);
stripe_status_t stripe_adamw_run(stripe_adamw_t* adamw, const stripe_adamw_step_t* step, void* hip_stream);

/* The values that bound states of STRIPE_I8 stand for: m[i], v[i] receive those of tensor i in fp32 (NULL, or NULL entries: not wanted). */
stripe_status_t stripe_adamw_read(stripe_adamw_t* adamw, float* const* m, float* const* v, void* hip_stream);
void stripe_adamw_destroy(stripe_adamw_t* adamw);

/* ------------------------------------------------------------------------
 * Autotiling (paper Section 3.3, Figures 4 and 5): host-only integer code.
 *
 * All three calls take the FLAT form of a block: the declaring root (no
 * indexes) whose child is the leaf.  A tile gives one size per leaf index,
 * 1 <= tile[j] <= ranges[j]; tile[j] == ranges[j] leaves index j whole.
 *
 * Cost model (Figure 4's caption): cache lines touched per unit of work.
 * For every counted refinement the tile's view is the box its accesses span
 * over one tile, overflow and halo included (constraints remove those
 * accesses at run time but the view still holds them).  Lines of a view =
 * product of its extents, the stride-1 dimension counted in whole lines
 * (views taken as line-aligned); footprint = product of its extents.
 *   cost = tiles * lines_per_tile / work,   tiles = prod ceil(range_j / tile_j),
 * work = product of the ranges of the indexes in `tiled_idx` (the figure
 * counts work in points of the tiled, spatial indexes: with 8 input
 * channels, 16 output channels, lines of 8 elements and a 512-element cap
 * this reproduces its 4.5 for the 3 x 4 tile and 4.666 for 6 x 2; dividing
 * by multiply-accumulates instead scales every cost of a block by one
 * constant).  A tile is inadmissible if its footprint exceeds the cap, or
 * if it violates `multiple_of` / `power_of_two` (Section 3.3: memory cap,
 * multiples of an earlier tensorisation, power-of-two pruning); a size equal
 * to the whole range is always allowed.
 */
typedef struct {
  int64_t line_elems;         /* cache line size in elements, >= 1 */
  int64_t mem_cap_elems;      /* cap on the summed footprints of the counted views, in elements; 0 = no cap */
  uint32_t counted_refs;      /* bit r: refinement r (descriptor order) counts toward lines and footprint */
  uint32_t tiled_idx;         /* bit j: index j may be tiled by the search and counts as work */
  int32_t power_of_two;       /* non-zero: the search tries power-of-two sizes only */
  const int64_t* multiple_of; /* [n_idx] or NULL: tile[j] must be a multiple of multiple_of[j] (entries < 1 = 1) */
} stripe_tile_model_t;

typedef struct {
  int64_t tiles;
  int64_t lines_per_tile;
  int64_t footprint_elems;
  int64_t work;
  double cost;
  int32_t admissible;
} stripe_tile_cost_t;

/* Cost of one given tile.  STRIPE_ERR_INVALID_DESC if root is not a flat form or a size is out of range. */
stripe_status_t stripe_tile_cost(const stripe_block_desc_t* root, const int64_t* tile, const stripe_tile_model_t* model,
                                 stripe_tile_cost_t* out);

/* Exhaustive search over the sizes of the indexes in model->tiled_idx (all others stay whole).
 * best_tile[n_idx] receives the admissible tile of least cost; ties go to fewer tiles, then to the
 * lexicographically larger tile.  STRIPE_ERR_UNSUPPORTED if no tile is admissible or the space
 * exceeds 2^22 candidates. */
stripe_status_t stripe_tile_search(const stripe_block_desc_t* root, const stripe_tile_model_t* model, int64_t* best_tile,
                                   stripe_tile_cost_t* best);

/*
 * The tiling rewrite (Section 3.3; Figure 5a -> 5b): returns a new nest
 * root -> outer block (ranges ceil(range_j / tile_j), refinements with the
 * tile's views: offsets scaled by the tile size, sizes including the halo) ->
 * inner block (ranges tile_j, accesses relative to the view, the original
 * constraints with every tiled index replaced by "passed outer value + inner
 * index", and one overflow constraint per index whose tile does not divide
 * its range).  The result is semantically the input block.  It is HOST
 * memory owned by the caller: release it with stripe_desc_free().
 */
stripe_status_t stripe_block_tile(const stripe_block_desc_t* root, const int64_t* tile, stripe_block_desc_t** out);
void stripe_desc_free(stripe_block_desc_t* desc);

#ifdef __cplusplus
}
#endif
#endif /* STRIPE_H */
