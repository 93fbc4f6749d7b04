/*
 * medverse_attn.h -- C ABI of the B200-native topology-aware (DAG) attention library.
 *
 * The library implements the attention of DAG-structured parallel decoding: every active
 * branch of a request's reasoning DAG (a Petri-net transition, Sec. 3.2) decodes at the same time
 * against one shared paged KV cache; a query token attends to the shared prefix, the nodes on its
 * own path and itself, never to a concurrently running sibling (Eq. 3), and its rotary position
 * continues from its fork or join point instead of the flattened sequence offset (Sec. 4.2,
 * "Adaptive Position Indices").
 *
 * Conventions for every call
 *   - extern "C", plain pointers and sizes.  "host" / "device" is stated per argument.
 *   - Ownership: the caller owns every device buffer (Q/K/V/O, page pools, workspace, the plan's
 *     device table buffer).  The library never allocates or frees device memory.  An mv_plan owns
 *     only host memory (its tables, kept in page-locked memory so that uploads are asynchronous).
 *   - Streams: `cuda_stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *     The three kernel calls and mv_plan_upload are asynchronous; they return the launch status only.
 *   - Errors: an mv_status is returned; argument errors are found on the host before any launch.
 *     Kernels never trap: every device-side wait is bounded; when one runs out the CTA issues nothing further, waits
 *     (again bounded) for its copies and products in flight, frees its tensor memory and returns, and
 *     mv_plan_read_status() then gives MV_ERR_TIMEOUT.  mv_status_string() names a status.
 *   - Layouts: q, k, v, q_rot, out are [tokens][heads][head_dim], row-major, element type
 *     mv_attn_geom.dtype.  The K and V page pools are separate buffers of the same element type, each
 *     [num_pages][n_kv_heads][head_dim / 64][page_size][64]: the block of one (page, KV head) is contiguous
 *     (4 KB for bf16, head_dim 128) and holds the head vectors of its 16 tokens split into 64-element column
 *     blocks, so that one bulk tensor copy with the 128-byte shared-memory swizzle moves the whole block.
 *     Element c of token t of (page p, head h) is at ((p * n_kv_heads + h) * (head_dim / 64) + c / 64) * 1024
 *     + t * 64 + c % 64.  Only mv_rope_write_kv writes the pools and only mv_dag_decode_attn reads them.
 *   - Order: "new tokens" (rows) are ordered (request, node index, token index) ascending.
 *   - Supported geometry: head_dim 64 or 128; n_q_heads a multiple of n_kv_heads; page_size 16.
 *     Anything else returns MV_ERR_UNSUPPORTED.  There is no CPU fallback.
 */
#ifndef MEDVERSE_ATTN_H_
#define MEDVERSE_ATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MV_OK = 0,
  MV_ERR_INVALID_ARG = 1,      /* null pointer, negative size, inconsistent offsets, bad enum          */
  MV_ERR_NOT_TOPOLOGICAL = 2,  /* a parent index is not smaller than its child's index (or a cycle)     */
  MV_ERR_PAGE_CAPACITY = 3,    /* a node's page list is too short for node_len + node_new tokens        */
  MV_ERR_UNSUPPORTED = 4,      /* head_dim / dtype / group size / batch shape the kernel does not take  */
  MV_ERR_WORKSPACE = 5,        /* workspace or table buffer missing, too small or misaligned            */
  MV_ERR_CUDA = 6,             /* a CUDA runtime call failed (launch error, copy error)                 */
  MV_ERR_TIMEOUT = 7           /* a bounded device-side wait ran out (read with mv_plan_read_status)    */
} mv_status;

/* Which nodes a token may attend to.  The paper states the mask twice, differently (Eq. 3 masks only
 * same-frontier siblings; Sec. 3.2 / 4.3 let a branch inherit the history of its own path only). */
typedef enum {
  MV_VIS_ANCESTORS = 0,  /* prefix + transitive ancestors + the node itself (Sec. 3.2, Sec. 4.3 Join) */
  MV_VIS_LAYERWISE = 1   /* Eq. 3 literally: every node of an earlier frontier layer + the node itself */
} mv_vis_mode;

/* Where a node's position indices start (Sec. 4.2). */
typedef enum {
  MV_POS_MAX_PARENT_END = 0,  /* right after the largest index used by any parent (fork alignment and
                                 the join rule, applied node by node)                                   */
  MV_POS_FRONTIER_ALIGNED = 1 /* one start for a whole frontier layer: the largest end of the previous
                                 layer (the sentence on fork alignment read literally)                  */
} mv_pos_mode;

typedef enum { MV_F32 = 0, MV_BF16 = 1 } mv_dtype;

/* A batch of request DAGs.  HOST memory, caller-owned, read only during mv_plan_dag.
 * A node is one reasoning step (one Petri-net transition); node 0 of a request is normally the shared
 * prefix (prompt + linear plan, Sec. 4.3 Phase I).  Node indices inside a request are local. */
typedef struct {
  int32_t n_req;
  const int32_t* node_off;   /* [n_req+1]   CSR over nodes                                             */
  const int32_t* node_len;   /* [n_nodes]   tokens of the node already in the KV pool                  */
  const int32_t* node_new;   /* [n_nodes]   tokens appended by this step (decode: 1 on frontier nodes,
                                            0 elsewhere; prefill: the node's length)                   */
  const int32_t* parent_off; /* [n_nodes+1] CSR over parent lists                                      */
  const int32_t* parent_idx; /* local parent indices, each < its child's local index                   */
  const int32_t* page_off;   /* [n_nodes+1] CSR over page lists                                        */
  const int32_t* page_idx;   /* physical page ids; a node's pages hold only that node's tokens; the
                                last page may be partial; ceil((len+new)/page_size) pages are required */
  int32_t page_size;         /* 16 */
  int32_t vis_mode;          /* mv_vis_mode */
  int32_t pos_mode;          /* mv_pos_mode */
} mv_dag_batch;

typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim, page_size;
  int64_t num_pages;   /* pages in each of the K and V pools (see "Layouts" above for the block layout) */
  int32_t dtype;       /* mv_dtype of q/k/v/out and of the pools */
  float sm_scale;      /* softmax scale; 0 means 1/sqrt(head_dim) */
  double rope_base;    /* theta_i = rope_base^(-2i/head_dim) */
} mv_attn_geom;

/* Optional tuning of the decode work lists (all zero = the defaults). */
typedef struct {
  int32_t chunk_tokens;      /* longest KV slice of one work unit in tokens (multiple of page_size);
                                0 = no limit (slices are cut only where a CTA's equal share of the step ends)  */
  int32_t sched_ctas;        /* shares the step's KV stream is cut into = half-CTAs the decode kernel runs with
                                (0 = 296, two per SM of a 148-SM part)                                         */
} mv_plan_tuning;

typedef struct mv_plan mv_plan;

/* Canonical integer tables of a plan (host memory, owned by the plan, valid until the plan is
 * re-planned or destroyed).  "q-node" = a node that receives new tokens in this step. */
typedef enum {
  MV_TAB_LAYER = 0,         /* int32 [n_nodes]      frontier layer: 0 for roots, else 1 + max over parents (Eq. 1) */
  MV_TAB_POS_START = 1,     /* int32 [n_nodes]      first position index of the node (Sec. 4.2)                 */
  MV_TAB_POS_ID = 2,        /* int32 [n_new_tokens] position index of every new token                           */
  MV_TAB_SLOT = 3,          /* int64 [n_new_tokens] pool slot = page_id * page_size + offset in page            */
  MV_TAB_QNODE = 4,         /* int32 [n_qnodes]     global node index of every q-node, ascending                 */
  MV_TAB_QNODE_TOK_OFF = 5, /* int32 [n_qnodes+1]   offsets of each q-node's new tokens                          */
  MV_TAB_SEG_OFF = 6,       /* int32 [n_qnodes+1]   CSR over the q-node's visible segments                       */
  MV_TAB_SEG_NODE = 7,      /* int32 [n_segs]       global node index of the segment (ascending in a q-node)     */
  MV_TAB_SEG_LEN = 8,       /* int32 [n_segs]       node_len + node_new of that node                             */
  MV_TAB_KV_LEN = 9,        /* int64 [n_qnodes]     tokens visible to the last new token of the q-node           */
  /* The decode kernels' work lists, as int32 words, for tests that replay them on the host (the layout is the
   * kernels' own and may change): */
  MV_TAB_WORK_STAGES = 10,        /* 16 words per stage: page[4], valid tokens (a byte per page slot), page slots
                                     in use, row mask low word [4], row mask high word [4], 2 unused              */
  MV_TAB_WORK_UNITS = 11,         /* 8 words per unit: first stage, stages, first item row, rows, KV head, 3 unused */
  MV_TAB_WORK_ITEM_ROWS = 12,     /* 2 words per (unit, row): row, first partial slot or -1                       */
  MV_TAB_WORK_CTA_UNIT_OFF = 13,  /* [n_ctas + 1] CSR over the units of every share                               */
  MV_TAB_WORK_ROWKV_PART_OFF = 14 /* [n_rows * n_kv_heads + 1] CSR over the partial slots of a (row, KV head)     */
} mv_plan_table_id;

typedef struct {
  int64_t n_nodes, n_new_tokens, n_qnodes, n_segs;
  int64_t decode_ready;        /* 1 if mv_dag_decode_attn applies: every node receives at most one token, or at
                                  most 256 each with no receiving node visible to another of its request        */
  int64_t prefill_ready;       /* 1 if no node holds older tokens (mv_dag_prefill_attn applies)            */
  int64_t n_items;             /* decode: work units = (KV slice of a node, KV head, row set)                */
  int64_t n_partials;          /* decode: split-KV partial results, each holding group_size head vectors    */
  int64_t chunk_tokens;        /* decode: the slice limit in effect, or a CTA's share in tokens if none    */
  int64_t unique_kv_tokens;    /* tokens of every node at least one row sees, each once                    */
  int64_t per_row_kv_tokens;   /* sum over rows of visible tokens                                          */
  int64_t n_q_tiles;           /* prefill: query tiles                                                      */
  int64_t visible_pairs;       /* prefill: allowed (query, key) pairs                                      */
  int64_t tile_pairs;          /* prefill: (query, key) pairs inside the KV ranges the kernel walks,
                                  rounded up to whole 128x64 tiles                                         */
  int64_t max_page_id;         /* largest page id referenced                                                */
  int64_t max_item_rows;       /* decode: largest row set of a work item                                    */
  int64_t sched_kv_heads, sched_group; /* head counts the decode work lists were cut for (0: no geometry yet) */
  int64_t n_ctas;              /* decode: CTAs the step was cut for                                         */
  int64_t max_cta_cost;        /* decode: largest share handed to one CTA, in tokens of one KV head (a unit
                                  counts as its tokens + 48)                                                */
  int64_t append_tiles;        /* node append: 128-row query tiles over the paged cache (0 when no node of a
                                  decode_ready batch receives several tokens)                               */
  int64_t max_node_new;        /* most new tokens any node receives                                         */
} mv_plan_stats;

enum { MV_OP_ROPE_WRITE_KV = 0, MV_OP_DECODE_ATTN = 1, MV_OP_PREFILL_ATTN = 2, MV_OP_PREFILL_ATTN_BWD = 3 };

/* DAG -> segment planner (Eq. 1 layering; Eq. 3 / Sec. 4.3 visibility; Sec. 4.2 positions; Sec. 3.2 KV index
 * lists).  Host only, integers only, deterministic.
 *   batch  host, read during the call only: the paper-level description of the step, nothing else.
 *   geom   host, optional.  The canonical tables, mv_rope_write_kv and the prefill calls need no geometry.  The decode
 *          kernels' work lists are cut for a head count (units are per KV head; a node's rows are grouped so that
 *          rows * group size <= 64), so only n_q_heads and n_kv_heads are read.  With geom == NULL the plan keeps a copy
 *          of the batch instead and mv_plan_bind_geometry cuts the lists later, for any supported geometry; until then
 *          mv_dag_decode_attn returns MV_ERR_UNSUPPORTED.
 *   tuning host, optional (NULL = defaults).
 *   plan   in/out: if *plan is NULL a new plan is created; otherwise the existing plan is re-planned in
 *          place and its host buffers are reused (no allocation once they are large enough).  The caller
 *          must not re-plan while an mv_plan_upload of the same plan is still in flight on a stream.
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_NOT_TOPOLOGICAL, MV_ERR_PAGE_CAPACITY, MV_ERR_UNSUPPORTED (head counts).  On
 * error *plan is unchanged if it was NULL and left in an unusable-but-destroyable state otherwise. */
mv_status mv_plan_dag(const mv_dag_batch* batch, const mv_attn_geom* geom, const mv_plan_tuning* tuning, mv_plan** plan);

/* Cuts (or re-cuts) the decode work lists of a plan that was made without a geometry, for `geom`'s head counts.  The
 * plan's canonical tables do not change; its device tables do: upload it again before the next kernel call.
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED (the plan was made with a geometry and kept no copy of its batch). */
mv_status mv_plan_bind_geometry(mv_plan* plan, const mv_attn_geom* geom, const mv_plan_tuning* tuning);

/* Canonical table access for parity checks.  *host_ptr points into the plan; *count is in elements. */
mv_status mv_plan_table(const mv_plan* plan, int which, const void** host_ptr, int64_t* count);

mv_status mv_plan_get_stats(const mv_plan* plan, mv_plan_stats* stats);

/* Bytes of device memory the plan's kernel tables need (positions, slots, page ids, work lists). */
size_t mv_plan_device_bytes(const mv_plan* plan);

/* Asynchronous host->device copy of the plan's kernel tables into `device_buf` (device, caller-owned,
 * 256-byte aligned, at least mv_plan_device_bytes(plan) bytes).  The plan remembers device_buf; the
 * kernel calls below read the tables from there, so device_buf must stay valid and unmodified while
 * calls that use this plan are in flight.  Errors: MV_ERR_WORKSPACE, MV_ERR_CUDA. */
mv_status mv_plan_upload(mv_plan* plan, void* device_buf, size_t device_buf_bytes, void* cuda_stream);

void mv_plan_destroy(mv_plan* plan);

/* Workspace bytes (device, caller-owned, 256-byte aligned) an op needs for this plan and geometry.
 * MV_OP_DECODE_ATTN: split-KV partial outputs and softmax statistics.  MV_OP_PREFILL_ATTN: the optional per-(token,
 * query head) log-sum-exp, n_new_tokens * n_q_heads floats (the call also runs without a workspace).
 * MV_OP_PREFILL_ATTN_BWD: as many floats again.  MV_OP_ROPE_WRITE_KV needs none (0). */
size_t mv_workspace_bytes(const mv_plan* plan, const mv_attn_geom* geom, int op);

/* RoPE with adaptive positions fused into the KV-cache write (P(i) of Eq. 2 at the indices of Sec. 4.2).
 * For new token t (n = n_new_tokens of the plan):
 *   q_rot[t] = RoPE(q[t], pos_id[t]);  k_pages[slot[t]] = k_rot[t] = RoPE(k[t], pos_id[t]);  v_pages[slot[t]] = v[t].
 * RoPE pairs element i with i + head_dim/2; the angle pos * rope_base^(-2i/head_dim) and its reduction modulo
 * pi/2 are evaluated in double precision, cos / sin of the reduced angle in float (within two float ulps of the
 * double-precision values at any position); the rotation is float; results are stored in `dtype`.
 *   q       device [n][n_q_heads][head_dim]   raw queries, or NULL (then q_rot is not written)
 *   k, v    device [n][n_kv_heads][head_dim]  raw keys / values
 *   q_rot   device [n][n_q_heads][head_dim]   out (may alias q); NULL exactly when q is NULL
 *   k_rot   device [n][n_kv_heads][head_dim]  out, optional (NULL to skip; may alias k): the rotated keys in
 *           token order, which is what mv_dag_prefill_attn reads
 *   k_pages, v_pages  device pools, updated in place at the new tokens' slots; both NULL skips the cache
 *           write (then k_rot must be given)
 * Requires mv_plan_upload first.  Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED, MV_ERR_WORKSPACE, MV_ERR_CUDA. */
mv_status mv_rope_write_kv(const mv_plan* plan, const mv_attn_geom* geom, const void* q, const void* k,
                           const void* v, void* q_rot, void* k_rot, void* k_pages, void* v_pages,
                           void* cuda_stream);

/* ---- Rotary forms ----------------------------------------------------------------------------------------------------
 * mv_rope_write_kv and its relatives rotate whole heads in two halves with angles pos * rope_base^(-2i/head_dim).  Backbones
 * differ in that: which elements are paired, how much of the head turns, and how the angles are stretched for contexts longer
 * than those trained on.  A form says so; the calls with _form take it in place of geom->rope_base (which they do not read).
 * With rotary_dim = R, pair i < R / 2 is (first + i, first + R/2 + i) as halves, (first + 2i, first + 2i + 1) as pairs, and
 *   a' = A (a cos x - b sin x),  b' = A (b cos x + a sin x),  x = pos * theta[i],  A = amplitude;
 * elements outside [first, first + R) are passed on as they are.  Angles and arithmetic as in mv_rope_write_kv (the products with
 * A are rounded once more, to float). */
typedef enum { MV_ROPE_HALVES = 0, MV_ROPE_PAIRS = 1 } mv_rope_layout;
typedef struct {
  int32_t layout;      /* mv_rope_layout                                                                     */
  int32_t first;       /* first rotated element of a head, a multiple of 16                                  */
  int32_t rotary_dim;  /* elements rotated, a multiple of 16, 16 .. head_dim - first                         */
  float amplitude;     /* A above, greater than 0 and at most 1024                                           */
  double theta[64];    /* angle per position of every pair, -1 .. 1; the first rotary_dim / 2 are read        */
} mv_rope_form;

/* How mv_rope_form_init stretches the angles theta_i = base^(-2i/R): */
typedef enum {
  MV_ROPE_PLAIN = 0,   /* not at all                                                                          */
  MV_ROPE_LINEAR = 1,  /* theta_i / factor                                                                    */
  MV_ROPE_BASE = 2,    /* with base * factor^(R / (R - 2)) for base: the slowest pair is stretched by factor, the fastest not */
  MV_ROPE_RAMP = 3     /* by the turns n = length * theta_i / (2 pi) a pair makes over the length it was trained on: with
                          w = (n - slow) / (fast - slow), held in [0, 1], w theta_i + (1 - w) theta_i / factor.  (Where a checkpoint's
                          ramp runs over the pair's index i between two rounded bounds instead, write its angles into theta.)  */
} mv_rope_scaling;

/* Fills a form (host only).  factor is read unless the scaling is MV_ROPE_PLAIN; length, slow and fast with MV_ROPE_RAMP only.
 * The angles before any stretching are computed as the calls without a form compute theirs: whole heads in halves with amplitude 1 and
 * rope_base for base give the bits of mv_rope_write_kv.  mv_rope_write_kv_fp8_blk fuses other products of k, so there k_rot, or a byte of K,
 * may come out one rounding apart.
 * The struct may as well be filled, or changed, by the caller's own code.
 * Errors: MV_ERR_INVALID_ARG (enums, base < 1 or, stretched, beyond a double, factor < 1, length <= 0, slow < 0, fast <= slow, amplitude),
 * MV_ERR_UNSUPPORTED (first or rotary_dim not a multiple of 16, rotary_dim outside 16 .. 128, first < 0 or > 112). */
mv_status mv_rope_form_init(mv_rope_form* form, int32_t layout, int32_t first, int32_t rotary_dim, double base, int32_t scaling,
                            double factor, double length, double slow, double fast, float amplitude);

/* The rotation by itself, and its backward pass: with backward = 0 q_out[t] = R(pos_id[t]) q[t] and k_out[t] = R(pos_id[t]) k[t],
 * with backward = 1 the transposed map (the sine changes its sign), which turns the gradients of q_rot and k_rot, as
 * mv_dag_prefill_attn_bwd gives them, into those of q and k.
 *   pos_id   device int32 [n_tokens], positions -2^30 .. 2^30: mv_step_tables.pos_id, mv_plan_positions, or the caller's own
 *   q, k     device, token t's heads at q + t * q_stride elements ([n_q_heads][head_dim], contiguous), k likewise: q and k may lie side by side
 *            in the rows of one projection.  Either may be NULL with its output
 *   q_out, k_out  device, with strides of their own; may be q and k with the same strides.  Otherwise no row of an output may overlap a row of
 *            an input or of the other output (refused)
 * geom: n_q_heads, n_kv_heads, head_dim and dtype are read.  Strides are multiples of 16 bytes and at least a token's heads;
 * all tensors are 16-byte aligned.
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED, MV_ERR_CUDA. */
mv_status mv_rope_rotate(const mv_rope_form* form, const mv_attn_geom* geom, const int32_t* pos_id, int64_t n_tokens, int32_t backward,
                         const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride,
                         void* k_out, int64_t k_out_stride, void* cuda_stream);

/* Positions of the plan's new tokens on the device (int32 [n_new_tokens], part of the uploaded tables; valid as long as they are).
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_WORKSPACE (not uploaded). */
mv_status mv_plan_positions(const mv_plan* plan, const int32_t** device_ptr);

/* mv_rope_write_kv with a form.  Errors: its own, and MV_ERR_INVALID_ARG for a form that does not fit head_dim. */
mv_status mv_rope_write_kv_form(const mv_plan* plan, const mv_attn_geom* geom, const mv_rope_form* form, const void* q, const void* k,
                                const void* v, void* q_rot, void* k_rot, void* k_pages, void* v_pages, void* cuda_stream);

/* Multi-branch decode attention (Eq. 2 with the DAG mask of Eq. 3 over a shared paged cache, Sec. 4.3
 * Fork / Join): for every row r (the single new token of a frontier node v) and query head h,
 *   out[r][h] = sum_j softmax_j(sm_scale * <q_rot[r][h], K_j>) V_j
 * over all tokens j of the nodes visible to v, the row's own just-written token included, so
 * mv_rope_write_kv must precede this call in stream order.  Pages shared by several rows of a request
 * (prefix, common ancestors) are read once per KV head and serve all those rows and the whole GQA group.
 * Node append (what follows a Join or the Phase I -> II hand-over of Sec. 4.3, where more than one token is
 * written to a node at once): a node may receive up to 256 new tokens, one row each in (node, token) order; new
 * token j of v then sees v's tokens 0 .. node_len(v) + j and every other visible node in full.  In a request
 * where some node receives several tokens, the nodes that receive tokens must not see one another, else the
 * plan is not decode_ready.  With head_dim 128, an even group size, 16-byte aligned q_rot and out, and some
 * node receiving at least 40 tokens, the step runs as 128-row query tiles over the paged cache (a node's
 * history is then read once per 128 new tokens); the workspace is still required but left untouched.
 *   q_rot   device [n_rows][n_q_heads][head_dim]  bf16
 *   k_pages, v_pages  device pools, bf16
 *   out     device [n_rows][n_q_heads][head_dim]  bf16
 *   workspace device, mv_workspace_bytes(plan, geom, MV_OP_DECODE_ATTN) bytes; contents are scratch
 * dtype must be MV_BF16 and the plan decode_ready, else MV_ERR_UNSUPPORTED. */
mv_status mv_dag_decode_attn(const mv_plan* plan, const mv_attn_geom* geom, const void* q_rot,
                             const void* k_pages, const void* v_pages, void* out, void* workspace,
                             size_t workspace_bytes, void* cuda_stream);

/* FP8 KV cache variant of the decode step (no counterpart in the paper: a storage format that halves the bytes a decode
 * step streams).  The pools hold 8-bit floats with 4 exponent and 3 mantissa bits (largest finite value 448, no
 * infinities), one scale per KV head: value = stored * scale[head].  kv_scale is a DEVICE array of 2 * n_kv_heads floats:
 * the K scales of all heads, then the V scales (positive; chosen by the caller, e.g. from calibration).
 * Pool layout: [num_pages][n_kv_heads][page_size][head_dim] bytes, K and V separate: the block of one (page, KV head) is
 * 2 KB, contiguous, one token per 128-byte row.
 *
 * mv_rope_write_kv_fp8 is mv_rope_write_kv writing such pools: k_pages8[slot[t]] = round(RoPE(k[t], pos_id[t]) / K scale),
 * v_pages8[slot[t]] = round(v[t] / V scale), rounding to nearest even and saturating at +-448; q_rot as before (bf16).
 * mv_dag_decode_attn_fp8 is mv_dag_decode_attn reading them: same plan, same work lists, same workspace, same result up
 * to the format's rounding.  Inside the kernel the queries and the softmax weights are 8-bit floats as well (one scale
 * per q-vector; each as a rounded value plus a rounded remainder, about seven bits of mantissa), so that both products
 * run on the tensor cores' 8-bit path straight on the pool bytes.
 * The write rotates as geom says; it has no counterpart that takes a rotary form.
 * MV_BF16 queries and outputs, head_dim 128, single-token steps only (max one new token per node); anything else is
 * MV_ERR_UNSUPPORTED.  Other errors as for mv_rope_write_kv and mv_dag_decode_attn. */
mv_status mv_rope_write_kv_fp8(const mv_plan* plan, const mv_attn_geom* geom, const void* q, const void* k, const void* v,
                               void* q_rot, void* k_pages8, void* v_pages8, const float* kv_scale, void* cuda_stream);
mv_status mv_dag_decode_attn_fp8(const mv_plan* plan, const mv_attn_geom* geom, const void* q_rot, const void* k_pages8,
                                 const void* v_pages8, const float* kv_scale, void* out, void* workspace,
                                 size_t workspace_bytes, void* cuda_stream);

/* ---- Decode steps planned on the device, over a block-scaled 8-bit cache -------------------------------------------
 * Three calls that make a decode step without a host step (no counterpart in the paper: a packaging of its decode step and a
 * storage format): the batch description lives in DEVICE memory, mv_step_tables_build turns it into positions, slots and
 * block tables, mv_rope_write_kv_fp8_blk fills a cache of 8-bit floats whose scales belong to (page, KV head) and follow
 * the data, and mv_dag_decode_attn_fp8_blk attends over it.  Lengths that advance on the device need no new launch
 * arguments, so a step can be captured into a CUDA graph once and replayed while the requests grow.
 *
 * The step's tables: device arrays of the caller.  A row is a new token of the step, rows ordered as everywhere (request,
 * node, token).  The rows of a request are cut into groups of at most rows_per_group consecutive rows (1 .. 64;
 * rows_per_group * group_size <= 64 for the attention call); a group never holds rows of two requests.  An ENTRY of a group
 * is four int32 words {page, tokens, mask low, mask high}: the rows of the group whose bits are set see the first `tokens`
 * (1 .. 16) tokens of the page, and nothing else of the page through this entry.  Entries of a group are ordered by (node, page of the node, tokens);
 * a page stands there once unless rows see different counts of it (several new tokens in one node).  A TILE is eight
 * consecutive entries of one group (the last of a group may have fewer).
 * What lies beyond the step's counts: slot = -1 and pos_id = 0 for unused rows, empty groups (every offset repeats the
 * total); entries beyond the total are left as they were.  The arrays may also be filled by the caller's own code. */
typedef struct {
  int32_t max_rows, max_groups, max_entries; /* capacities; max_groups = max_entries = 0: positions and slots only  */
  int32_t rows_per_group;
  int32_t* pos_id;         /* device [max_rows]       position index of every row (Sec. 4.2)                        */
  int64_t* slot;           /* device [max_rows]       pool slot = page * 16 + offset, -1 = unused row               */
  int32_t* group_row_off;  /* device [max_groups + 1] CSR over rows       (NULL when max_groups = 0, as the next three) */
  int32_t* group_ent_off;  /* device [max_groups + 1] CSR over entries                                              */
  int32_t* group_tile_off; /* device [max_groups + 1] running count of tiles                                        */
  int32_t* entries;        /* device [max_entries][4], 16-byte aligned                                              */
  int32_t* counts;         /* device [8]: rows, groups, entries, tiles, status (an mv_status), three zeros          */
} mv_step_tables;

/* What the launch has to know about the batch (everything else is read on the device). */
typedef struct {
  int32_t n_nodes;       /* length of node_len / node_new                                                       */
  int32_t n_parents;     /* length of parent_idx                                                                */
  int32_t n_pages;       /* length of page_idx                                                                  */
  int32_t max_req_nodes; /* most nodes of one request, 1 .. MV_STEP_MAX_REQ_NODES                               */
  int64_t num_pages;     /* pages of the pool: ids in [0, num_pages) are accepted                               */
} mv_step_shape;
#define MV_STEP_MAX_REQ_NODES 2048

/* Positions, slots and block tables of a step from its batch description, on the device (the canonical tables of
 * mv_plan_dag, and the block tables the attention call below reads).
 *   batch  the struct itself is read during the call; n_req, page_size, vis_mode and pos_mode are host values, every
 *          POINTER in it is a DEVICE pointer (4-byte aligned).  A request may have no nodes (node_off repeats), so a batch of fixed
 *          n_req serves a varying number of live requests.
 *   tables in: capacities and device pointers; out: the arrays' contents.
 *   workspace  device, 256-byte aligned, mv_step_tables_workspace_bytes(n_req) bytes, scratch.  Two calls that may
 *          overlap on the device must not share it, nor the tables.
 * Errors found on the host: MV_ERR_INVALID_ARG, MV_ERR_WORKSPACE, MV_ERR_UNSUPPORTED (max_req_nodes, rows_per_group), MV_ERR_CUDA.
 * Errors in the arrays' contents are found on the device: counts[4] then holds the status (the largest, if several
 * requests are wrong) and the tables describe an empty step, so that the calls below touch nothing:
 * MV_ERR_NOT_TOPOLOGICAL, MV_ERR_PAGE_CAPACITY, MV_ERR_INVALID_ARG (offsets, negative lengths, a page id outside the
 * pool), MV_ERR_WORKSPACE (more rows, groups or entries than the capacities), MV_ERR_UNSUPPORTED (a request with more
 * than max_req_nodes nodes; with block tables also a node with more than 256 new tokens).  mv_step_tables_read_status reads it.  Pages must
 * belong to one node each (as for mv_plan_dag; not checked). */
size_t mv_step_tables_workspace_bytes(int32_t n_req);
mv_status mv_step_tables_build(const mv_dag_batch* batch, const mv_step_shape* shape, const mv_step_tables* tables,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Status word of the tables (counts[4]): what the build found, or what the calls below recorded (MV_ERR_TIMEOUT,
 * MV_ERR_INVALID_ARG for a slot, page or row offset out of range, which they skip).  Synchronises the stream. */
mv_status mv_step_tables_read_status(const mv_step_tables* tables, void* cuda_stream, int32_t* status);

/* mv_rope_write_kv_fp8 with one scale per (page, KV head), K and V apart, kept by the call itself.
 * Pools as there: [num_pages][n_kv_heads][page_size][head_dim] bytes.  kv_scale: device float [num_pages][n_kv_heads][2],
 * the K scale then the V scale of every block; value = stored byte * scale; read and written in place.
 * A scale is a power of two, 2^-60 .. 2^40: the smallest s for which the block's new tokens have |k| <= 316 s before the
 * rotation (a rotated element is at most sqrt 2 times the largest raw one, and 316 sqrt 2 < 448), resp. |v| <= 448 s; where
 * the largest magnitude is exactly at that bound, s or 2 s (ceil(log2(max / 316)) as CUDA's double-precision log2 gives it).  A block
 * that already holds tokens of its node keeps the larger of its own scale and that one; if it grows, the stored tokens are
 * moved to it (dividing by a power of two: exact, but for what falls among the format's subnormals, which is rounded to
 * nearest even).  Values round to nearest even and saturate.  A block that receives an infinity or a NaN gets the
 * scale NaN and keeps it: rows that see the block get NaN, rows that do not see it are untouched.
 * A page whose first slot is written by this call starts afresh: its old scale and bytes count for nothing.
 * Rows with slot -1 are skipped and their outputs left as they were.  Rows of one page must be consecutive and ascending
 * (they are, in tables built above), and one page must not be written by two overlapping calls.
 * The kernel for prompts takes tables with max_rows >= 2048 (whatever their rows are): give decode steps tables of their own.
 *   q, k, v  device [max_rows][heads][head_dim] bf16, q may be NULL;  q_rot  out (may alias q), NULL exactly when q is;
 *   k_rot    out, optional (NULL to skip; may alias k): rotated keys in bf16, what mv_dag_prefill_attn reads
 * dtype MV_BF16, head_dim 64 or 128; all tensors 16-byte aligned.  Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED, MV_ERR_CUDA. */
mv_status mv_rope_write_kv_fp8_blk(const mv_step_tables* tables, const mv_attn_geom* geom, const void* q, const void* k, const void* v,
                                   void* q_rot, void* k_rot, void* k_pages8, void* v_pages8, float* kv_scale, void* cuda_stream);

/* mv_rope_write_kv_fp8_blk with a rotary form.  The rule of the K scale takes |k| times the form's amplitude (rounded to float) where that
 * is above 1, so that a rotated element still fits.  Errors: its own, and MV_ERR_INVALID_ARG for a form that does not fit head_dim. */
mv_status mv_rope_write_kv_fp8_blk_form(const mv_step_tables* tables, const mv_attn_geom* geom, const mv_rope_form* form, const void* q,
                                        const void* k, const void* v, void* q_rot, void* k_rot, void* k_pages8, void* v_pages8,
                                        float* kv_scale, void* cuda_stream);

/* Decode attention over that cache: for every row r of the tables and query head h
 *   out[r][h] = sum_j softmax_j(sm_scale * <q_rot[r][h], K_j>) V_j
 * over the tokens the entries of r's group give it (a row that no entry names gets zeros).  The step's new tokens must be
 * in the cache first (mv_rope_write_kv_fp8_blk before this call in stream order).  A group's pages are read once per KV head, for all
 * its rows and the whole GQA group.  Rows beyond the tables' count are left as they were.
 *   q_rot, out  device [max_rows][n_q_heads][head_dim] bf16;  pools, kv_scale as above
 *   workspace   device, 256-byte aligned, mv_decode_fp8_blk_workspace_bytes(geom) bytes (it does not depend on the step);
 *               scratch, not to be shared by calls that may overlap on the device
 * out must not overlap q_rot.  A scale counts as the power of two that its exponent gives (its sign and mantissa are not looked at);
 * V's has to be at most 2^40, and below 2^-80 (a scale of zero too) counts as 2^-80.
 * Arithmetic: q as two 8-bit floats at one power of two per row and query head (off by at most 2^-17 of its largest element),
 * weights as three 8-bit floats (off by at most 1.5 * 2^-10 of the weight or 2^-29 of the row's largest), sums and softmax statistics
 * in 32 bits.  The same inputs give the same bits on every call.
 * dtype MV_BF16, head_dim 64 or 128, group size at most 64 and rows_per_group * group size <= 64; all tensors 16-byte aligned.
 * Errors: MV_ERR_INVALID_ARG (also q_rot or out with tables of positions and slots only, max_groups = 0), MV_ERR_UNSUPPORTED (also a pool of 2^31 or more (page, KV head, token) rows, and capacities
 * of max_entries / 8 + max_groups tiles whose product with n_kv_heads passes 1.7e9), MV_ERR_WORKSPACE, MV_ERR_CUDA.  A wait inside the
 * kernel that runs out (seconds) ends the call with MV_ERR_TIMEOUT in counts[4]; `out` is then undefined. */
size_t mv_decode_fp8_blk_workspace_bytes(const mv_attn_geom* geom);
mv_status mv_dag_decode_attn_fp8_blk(const mv_step_tables* tables, const mv_attn_geom* geom, const void* q_rot, const void* k_pages8,
                                     const void* v_pages8, const float* kv_scale, void* out, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream);

/* ---- Chunks of new tokens over that cache ------------------------------------------------------------------------------
 * A node may receive any number of tokens in one step (a prompt or the next piece of it, text put in at a join, accepted drafts), in
 * batches described on the device as above.  Positions and slots come from mv_step_tables_build with max_groups = 0, K and V from
 * mv_rope_write_kv_fp8_blk (or _form); then these two calls.  New token j of a node sees its node's tokens 0 .. node_len + j and every
 * other visible node in full, what that node receives in the same step included.
 *
 * The tables: device arrays of the caller.  Rows are the step's new tokens, ordered (request, node, token).  A receiving node has
 * a list of ENTRIES of two int32 words {page, tokens}: the pages of the other nodes it sees, ordered by (node, page), then its own;
 * `tokens` (1 .. 16) of a page's slots are held.  Its rows are cut into TILES of rows_per_tile consecutive rows (the last may have fewer),
 * eight int32 words each: {first row, rows, first entry of the node's list, entries of other nodes in it, index of the first row's token in
 * its node, key tiles before this tile, key tiles, 0}; a key tile is eight entries, and a query tile walks those up to its last row's own page.
 * What lies beyond the step's counts is left as it was.  The arrays may also be filled by the caller's own code; a record that does not
 * fit the arrays is skipped. */
typedef struct {
  int32_t max_rows, max_tiles, max_entries;  /* capacities                                                                */
  int32_t rows_per_tile;                     /* 1 .. 256; for the attention call at most 2 * (128 / group_size): that many is best */
  int32_t* tiles;          /* device [max_tiles][8], 16-byte aligned                                                      */
  int32_t* entries;        /* device [max_entries][2], 16-byte aligned                                                    */
  int32_t* counts;         /* device [8]: rows, tiles, entries, key tiles, status (an mv_status), three zeros             */
} mv_chunk_tables;

/* Builds them (batch, shape and errors as for mv_step_tables_build; pos_mode is not read).
 *   workspace  device, 256-byte aligned, mv_chunk_tables_workspace_bytes(n_req) bytes, scratch.  Two calls that may overlap on the device
 *              must not share it, nor the tables.
 * Errors found on the host: MV_ERR_INVALID_ARG, MV_ERR_WORKSPACE, MV_ERR_UNSUPPORTED (max_req_nodes, rows_per_tile), MV_ERR_CUDA.
 * On the device counts[4] then holds the status and the tables describe an empty step: MV_ERR_NOT_TOPOLOGICAL, MV_ERR_PAGE_CAPACITY,
 * MV_ERR_INVALID_ARG, MV_ERR_WORKSPACE (more rows, tiles or entries than the capacities), MV_ERR_UNSUPPORTED (a request with more than
 * max_req_nodes nodes, a node of more than 2^30 tokens, 2^31 key tiles). */
size_t mv_chunk_tables_workspace_bytes(int32_t n_req);
mv_status mv_chunk_tables_build(const mv_dag_batch* batch, const mv_step_shape* shape, const mv_chunk_tables* tables, void* workspace,
                                size_t workspace_bytes, void* cuda_stream);
/* Status word of the tables (counts[4]), as mv_step_tables_read_status.  Synchronises the stream. */
mv_status mv_chunk_tables_read_status(const mv_chunk_tables* tables, void* cuda_stream, int32_t* status);

/* Attention of every row of the tables over what it sees: for row r and query head h
 *   out[r][h] = sum_j softmax_j(sm_scale * <q_rot[r][h], K_j>) V_j.
 * The step's new tokens must be in the cache first.  Rows that no tile names are left as they were.  Single tokens are served as well
 * (mv_dag_decode_attn_fp8_blk is the faster call where no node receives more than about ten, since there the rows of different nodes share what they
 * read, and the more accurate one: its weights keep more bits.  32 and 8 heads of 128, us, that call / this one, for 1, 4, 8, 16, 32 new tokens on each node:
 * 16 requests with four branches each behind 2304 tokens 36, 66, 92, 149, 266 / 151, 152, 153, 155, 158; 64 requests behind 1088 60, 61, 76, 109, 183 / 86, 88, 88, 89, 92;
 * one request with four branches 18, 26, 29, 31, 43 / 23, 23, 23, 24, 26).
 *   q_rot, out  device [max_rows][n_q_heads][head_dim] bf16, not overlapping;  pools, kv_scale as above
 *   workspace   device, 256-byte aligned, mv_chunk_attn_workspace_bytes(geom) bytes (it does not depend on the step); scratch, not to be
 *               shared by calls that may overlap on the device
 * A scale counts as the power of two that its exponent gives, at least 2^-80, and has to be at most 2^40; NaN in either scale of a block
 * gives NaN to the rows that see the block and leaves the others untouched.  (The format's two NaN bytes, which the cache write never
 * stores, count as +-480.)
 * Arithmetic: keys and values are bf16 exactly; scores, sums and softmax statistics in 32 bits; weights rounded to bf16.  The same
 * inputs give the same bits on every call.
 * dtype MV_BF16, head_dim 64 or 128, group size at most 128, sm_scale not negative (and finite times log2 e); all tensors 16-byte aligned.  Errors: MV_ERR_INVALID_ARG,
 * MV_ERR_UNSUPPORTED (also a pool of 2^31 or more (page, KV head, token) rows, max_tiles * n_kv_heads past 2^31), MV_ERR_WORKSPACE, MV_ERR_CUDA.
 * In counts[4]: MV_ERR_INVALID_ARG (records, lists of more than 2^26 pages, pages outside the pool, which are skipped); a wait inside
 * the kernel that runs out (seconds) ends the call with MV_ERR_TIMEOUT there, `out` is then undefined. */
size_t mv_chunk_attn_workspace_bytes(const mv_attn_geom* geom);
mv_status mv_dag_chunk_attn_fp8_blk(const mv_chunk_tables* tables, const mv_attn_geom* geom, const void* q_rot, const void* k_pages8,
                                    const void* v_pages8, const float* kv_scale, void* out, void* workspace, size_t workspace_bytes,
                                    void* cuda_stream);

/* Copies pages inside pools: page dst[i] of every pool becomes page src[i], for i < n (a fork that goes on writing gets a copy of
 * the partly filled last page; a compacted pool moves its upper pages down: mv_sched_clone_request and mv_sched_compact make
 * such lists).  One launch for all pools, K and V and scales of any number of layers.
 *   pools    host, read during the call: base address (device) and bytes of a page of each, both multiples of 4 (of 16: faster);
 *            a page of the 16-bit pools has n_kv_heads * head_dim * 32 bytes, of the 8-bit pools half as many, of kv_scale n_kv_heads * 8
 *   src, dst device int32 [n]; pages outside [0, num_pages) are skipped, and *status becomes MV_ERR_INVALID_ARG.
 *            No page may be a destination twice, nor a destination and the source of another pair (its content is then undefined)
 *   count    device int32 [1], or NULL: only the first min(n, *count) pairs are copied, so a captured call can do any number up to n
 *   status   device int32 [1], or NULL (counts + 4 of tables will do); not touched unless something is wrong
 * Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED (n_pools > MV_PAGES_MAX_POOLS, pages above 2 GB, more than 2^31 blocks of work), MV_ERR_CUDA. */
#define MV_PAGES_MAX_POOLS 256
typedef struct {
  void* base;
  int64_t page_bytes;
} mv_page_pool;
mv_status mv_pages_copy(const mv_page_pool* pools, int32_t n_pools, int64_t num_pages, const int32_t* src, const int32_t* dst, int32_t n,
                        const int32_t* count, int32_t* status, void* cuda_stream);

/* Decode attention for callers that cannot allocate device memory.  (The paper has no counterpart: this is
 * a packaging variant of mv_dag_decode_attn, same arithmetic, same kernels.)
 *
 * Some hosts of this library may not call cudaMalloc or an allocating library routine on the decode path:
 * a serving loop whose memory pool is fixed at start-up and fully handed out, a plug-in that runs inside
 * another runtime's allocator-free region, or code that must not synchronise the device (cudaMalloc and
 * cudaFree do).  For them the split-KV scratch that mv_dag_decode_attn takes as `workspace` is replaced by
 * a fixed array of MV_STATIC_WORKSPACE_BYTES bytes that is part of the library image: every GPU on which
 * the library is loaded holds that much memory until the process exits.  The caller still passes q_rot,
 * the pools and out, exactly as for mv_dag_decode_attn; nothing is allocated or freed by this call.
 *
 *   - Limit: plans with mv_workspace_bytes(plan, geom, MV_OP_DECODE_ATTN) > MV_STATIC_WORKSPACE_BYTES are
 *     refused with MV_ERR_WORKSPACE before anything is launched (query it with mv_static_workspace_bytes()).
 *   - Set-up: the first call on each device looks up the array's device address (one cudaGetSymbolAddress,
 *     with the calling thread's current device).  That first call is a set-up call: with lazy module loading it is
 *     also the moment the driver brings the array into being on that device (and may synchronise).  Make it at
 *     start-up, outside any stream capture and outside the region in which nothing may be allocated; every later
 *     call on that device allocates and frees nothing.
 *   - Sharing: every call on a device uses the same array and finds the previous call's contents in it.
 *     The kernels write each partial result before they read it, so nothing needs clearing; but two calls
 *     whose kernels overlap on the GPU (different streams, no ordering between them) race on it.  Order such
 *     calls, or give all but one of them their own workspace through mv_dag_decode_attn.
 * Other errors are those of mv_dag_decode_attn. */
#define MV_STATIC_WORKSPACE_BYTES (16u << 20)
size_t mv_static_workspace_bytes(void);
mv_status mv_dag_decode_attn_static(const mv_plan* plan, const mv_attn_geom* geom, const void* q_rot,
                                    const void* k_pages, const void* v_pages, void* out, void* cuda_stream);

/* Topology-masked prefill attention over a flattened DAG sequence (Eq. 3; the training-time layout of
 * Sec. 4.2 and the engine's re-prefill): all tokens of the batch are new and contiguous in
 * (request, node, token) order;
 *   out[i][h] = sum_j softmax_j(sm_scale * <q_rot[i][h], k_rot[j]> + M_ij) v[j],
 * M_ij = 0 iff token j belongs to a node visible to node(i) and, inside node(i) itself, j <= i.
 * Key/value ranges no query of a tile may see are never visited (tile skipping).
 *   q_rot  device [T][n_q_heads][head_dim]   position-embedded queries
 *   k_rot  device [T][n_kv_heads][head_dim]  position-embedded keys
 *   v      device [T][n_kv_heads][head_dim]
 *   out    device [T][n_q_heads][head_dim]
 * dtype MV_F32 runs a float32 SIMT kernel, MV_BF16 the tensor-core kernel (float32 accumulation).
 * The plan must be prefill_ready, else MV_ERR_UNSUPPORTED.
 *   workspace  NULL, or device, 16-byte aligned, mv_workspace_bytes(plan, geom, MV_OP_PREFILL_ATTN) bytes: receives
 *              lse[i][h] = log2 sum_j 2^(sm_scale * log2(e) * <q_i, k_j> + M_ij) as float [T][n_q_heads], which
 *              mv_dag_prefill_attn_bwd takes.  Only the tcgen05 kernel (MV_BF16, head_dim 128, even group size,
 *              16-byte aligned tensors) writes it; with any other shape a non-NULL workspace is MV_ERR_UNSUPPORTED. */
mv_status mv_dag_prefill_attn(const mv_plan* plan, const mv_attn_geom* geom, const void* q_rot,
                              const void* k_rot, const void* v, void* out, void* workspace,
                              size_t workspace_bytes, void* cuda_stream);

/* Backward of mv_dag_prefill_attn: the attention the model is fine-tuned through (Sec. 5.1) is Eq. 2 with the mask of
 * Eq. 3 over the flattened training sequence at the position indices of Sec. 4.2.  Given dout = d loss / d out, with
 * P_ij = softmax_j(sm_scale * <q_i, k_j> + M_ij) per query head and delta_i = <dout_i, out_i>:
 *   dv[j]     = sum_i P_ij dout[i]                                    (summed over the query heads of j's KV head)
 *   dS_ij     = P_ij * (<dout[i], v[j]> - delta_i)
 *   dq_rot[i] = sm_scale * sum_j dS_ij k_rot[j],   dk_rot[j] = sm_scale * sum_i dS_ij q_rot[i]   (summed over the group)
 * The gradients are with respect to the position-embedded q_rot and k_rot (the rotation of mv_rope_write_kv is a fixed
 * orthogonal map per token).  Masked pairs contribute nothing; key tiles walk the transposed visibility (which query
 * runs see this key's node), so ranges no query can see are never visited.
 *   q_rot, k_rot, v, out   device, as given to / written by mv_dag_prefill_attn (bf16)
 *   dout      device [T][n_q_heads][head_dim] bf16
 *   lse       device [T][n_q_heads] float, as written by mv_dag_prefill_attn into its workspace
 *   dq_rot    device [T][n_q_heads][head_dim] bf16, out;  dk_rot, dv  device [T][n_kv_heads][head_dim] bf16, out
 *   workspace device, 256-byte aligned, mv_workspace_bytes(plan, geom, MV_OP_PREFILL_ATTN_BWD) bytes (scratch)
 * All tensors 16-byte aligned.  MV_BF16, head_dim 128 and an even group size only (MV_ERR_UNSUPPORTED otherwise); the plan
 * must be prefill_ready.  Deterministic (no atomics).  Errors: MV_ERR_INVALID_ARG, MV_ERR_UNSUPPORTED, MV_ERR_WORKSPACE,
 * MV_ERR_CUDA. */
mv_status mv_dag_prefill_attn_bwd(const mv_plan* plan, const mv_attn_geom* geom, const void* q_rot, const void* k_rot,
                                  const void* v, const void* out, const void* dout, const void* lse, void* dq_rot,
                                  void* dk_rot, void* dv, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* One decode step with HOST inputs and outputs (the end-to-end form of the path: Sec. 4.3 Phase II, one
 * frontier step).  Copies q, k, v (host, preferably page-locked, [n_rows][heads][head_dim]) to the device
 * staging buffer, uploads the plan, runs mv_rope_write_kv and mv_dag_decode_attn on `cuda_stream`, copies
 * `out` back to host memory and returns after enqueueing everything (asynchronous; synchronise the stream
 * before reading out_host).
 *   staging  device, caller-owned, mv_decode_step_staging_bytes(plan, geom) bytes, 256-byte aligned; holds
 *            the plan tables, q/k/v/out device copies and the decode workspace
 *   k_pages, v_pages  device pools (the resident KV cache) */
size_t mv_decode_step_staging_bytes(const mv_plan* plan, const mv_attn_geom* geom);
mv_status mv_decode_step_host(mv_plan* plan, const mv_attn_geom* geom, const void* q_host, const void* k_host,
                              const void* v_host, void* out_host, void* k_pages, void* v_pages, void* staging,
                              size_t staging_bytes, void* cuda_stream);

/* The same step starting from the batch description instead of a finished plan: the copies of q, k, v are
 * enqueued first and travel while the host plans the step (mv_plan_dag into *plan, which is created when NULL
 * and reused otherwise), then the step runs as in mv_decode_step_host.  The staging layout depends on the plan
 * only behind the q / k / v / out copies; size the buffer with mv_decode_step_staging_bytes on a plan of a batch
 * of the same shape (a too small buffer is refused with MV_ERR_WORKSPACE, possibly after the input copies were
 * enqueued).  *plan must not have an upload in flight (synchronise the stream between steps that share a plan).
 * Errors: those of mv_plan_dag and of mv_decode_step_host. */
mv_status mv_decode_step_host_batch(const mv_dag_batch* batch, mv_plan** plan, const mv_attn_geom* geom,
                                    const void* q_host, const void* k_host, const void* v_host, void* out_host,
                                    void* k_pages, void* v_pages, void* staging, size_t staging_bytes,
                                    void* cuda_stream);

/* The same step cut into slices that overlap (Sec. 4.3: the requests of a batch advance independently of one
 * another, so a batch may be cut between requests).  The batch is split into n_slices runs of consecutive requests with
 * about equal numbers of new tokens; every slice is planned on its own (plans[i], created when NULL, reused
 * otherwise) and runs as mv_decode_step_host_batch does, on one of two streams that the library keeps per device
 * (created by the first call on that device, with two event pairs, and kept until the process exits): slice i + 1's
 * inputs travel while slice i computes, and slice i's output travels while slice i + 1 computes.  The work starts
 * behind everything already enqueued on `cuda_stream`, and `cuda_stream` continues behind all of it: synchronise
 * `cuda_stream` before reading out_host, as with the other forms.  Rows of q, k, v, out are those of the whole batch
 * (a slice's rows are consecutive).  Results are those of the unsliced call up to the rounding order of the split-KV
 * merge (a slice's key ranges are cut for its own share of the step).
 *   plans    host array of n_slices plan pointers (in/out); none may have an upload in flight
 *   n_slices 1 .. min(8, batch->n_req)
 *   staging  device, 256-byte aligned; mv_decode_step_pipelined_staging_bytes(plans, n_slices, geom) bytes after
 *            mv_decode_step_pipelined_plan on a batch of the same shape (0 if a plan is missing or invalid)
 * The library's two streams and their events are shared by every call on a device: host threads must not run this
 * call on the same device at the same time.
 * mv_decode_step_pipelined_plan plans the slices only (host work; for sizing the staging buffer).
 * Errors: MV_ERR_INVALID_ARG (n_slices out of range, a slice without a request, null pointers), MV_ERR_WORKSPACE,
 * MV_ERR_CUDA, and those of mv_plan_dag; after an error, work of earlier slices may already be enqueued. */
mv_status mv_decode_step_pipelined_plan(const mv_dag_batch* batch, mv_plan** plans, int32_t n_slices,
                                        const mv_attn_geom* geom);
size_t mv_decode_step_pipelined_staging_bytes(mv_plan* const* plans, int32_t n_slices, const mv_attn_geom* geom);
mv_status mv_decode_step_host_pipelined(const mv_dag_batch* batch, mv_plan** plans, int32_t n_slices,
                                        const mv_attn_geom* geom, const void* q_host, const void* k_host,
                                        const void* v_host, void* out_host, void* k_pages, void* v_pages,
                                        void* staging, size_t staging_bytes, void* cuda_stream);

/* Reads the device-side status word of the kernels that last ran with this plan's uploaded tables: MV_OK, or
 * MV_ERR_TIMEOUT if a bounded wait inside a kernel ran out (the kernel then still terminated, with an
 * undefined result).  Copies 4 bytes device->host on `cuda_stream` and synchronises that stream.
 *   status  host, out */
mv_status mv_plan_read_status(const mv_plan* plan, void* cuda_stream, int32_t* status);

const char* mv_status_string(mv_status s);

/* Number of kernel launches the library has issued in this process since load (diagnostic counter). */
int64_t mv_launch_count(void);

/* Self-tests (diagnostics; no counterpart in the paper, nothing of the attention path runs).
 *
 * mv_selftest_bounded_wait: every wait inside the kernels is bounded and reports through the plan's status word
 * (mv_plan_read_status).  This call exercises that mechanism alone: one thread of a one-CTA kernel waits, with the
 * same bounded wait and a limit of `limit_ns` nanoseconds (1 .. 100 000 000), on a barrier that nothing ever
 * completes; when the limit has passed it records MV_ERR_TIMEOUT in the status word of `plan` (which must have been
 * uploaded) and returns.  No copy or product is in flight, the context stays usable; upload the plan again to clear
 * the word.  Asynchronous on `cuda_stream`.  Errors: MV_ERR_INVALID_ARG, MV_ERR_WORKSPACE, MV_ERR_CUDA.
 *
 * mv_selftest_tmap_cache: the launchers keep the tensor maps of recent calls in a small cache keyed by (device index,
 * up to three base pointers, row count, one more word).  This call runs the same lookup on a private instance with
 * four entries: returns 1 if the key is cached, else 0 after caching it (the oldest entry is replaced); reset != 0
 * empties the instance first.  Host only. */
mv_status mv_selftest_bounded_wait(const mv_plan* plan, uint64_t limit_ns, void* cuda_stream);
int32_t mv_selftest_tmap_cache(int32_t device, const void* a, const void* b, const void* c, int64_t rows, int64_t aux,
                               int32_t reset);

#ifdef __cplusplus
}
#endif
#endif /* MEDVERSE_ATTN_H_ */
