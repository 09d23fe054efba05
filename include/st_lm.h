/*
 * st_lm.h - C ABI of the fused multi-tenant operators of language models for MI355X (gfx950): matrix products with their
 * epilogue.
 *
 * They follow st_conv.h (Section 4 of the paper: the kernels of several tenants merged into one launch): an array of
 * per-tenant descriptors with device pointers makes a plan, the plan's run calls issue its work for all tenants together.
 * The conventions of st_conv.h hold:
 *   - Tensor pointers are DEVICE pointers, owned by the caller and borrowed by the plan until it is destroyed or rebound.
 *   - Streams are hipStream_t passed as void*; NULL is the default stream.  Run calls are asynchronous, never synchronise and
 *     never allocate device memory, and can be captured into graphs.  A plan belongs to the device that was current when it
 *     was made, and runs there whichever device is current.
 *   - Every function returns st_status; on failure no output argument is written and st_last_error_message() tells why.
 *   - Same plan + same inputs => bitwise identical outputs on every run.
 *   - A plan may own a workspace: two runs of one plan must not overlap in time, replays of captured ones included.
 *   - What one tenant writes must not overlap what another reads or writes.
 */
#ifndef ST_LM_H
#define ST_LM_H

#include "st_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Matrix products --------------------------------------------------------------------------------------------
 * One tenant's product y = act(x w^T + bias + residual), or act(x w^T + bias) + residual with ST_EPI_RESIDUAL_LAST:
 *   y[m,n] = act(sum_k x[m,k] w[n,k] + bias[n] + residual[m,n])
 * The sum, the bias, the residual and the activation are computed in fp32 (products of 16-bit operands are exact in it), and
 * rounded to out_dtype once, to nearest, ties to even.  At most one activation:
 *   ST_EPI_RELU       v > 0 ? v : 0 (also for a value that is not a number, as in st_conv.h)
 *   ST_EPI_GELU       v/2 erfc(-v/sqrt(2))
 *   ST_EPI_GELU_TANH  v/2 (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3)))
 *   ST_EPI_SILU       v / (1 + exp(-v)) */
enum { ST_EPI_BIAS = 4u, ST_EPI_GELU = 8u, ST_EPI_GELU_TANH = 16u, ST_EPI_SILU = 32u, ST_EPI_RESIDUAL_LAST = 64u };

typedef struct st_matmul_desc {
  int32_t M, N, K;       /* rows, outputs, inputs; M = 0 is a tenant with nothing to do this time             */
  int32_t in_dtype;      /* st_dtype of x, w and bias                                                         */
  int32_t out_dtype;     /* ST_DT_F32 or equal to in_dtype: of y and residual                                 */
  uint32_t epilogue;     /* ST_EPI_RELU, ST_EPI_RESIDUAL and the bits above; one ST_EPI_RESIDUAL* at most     */
  int64_t ldx, ldw, ldy, ldr; /* elements from a row of x, w, y, residual to the next; 0 = K, K, N, N         */
  const void* x;         /* device, M rows of K elements                                                      */
  const void* w;         /* device, N rows of K elements                                                      */
  const void* bias;      /* device, N elements; required iff ST_EPI_BIAS                                      */
  void* y;               /* device, M rows of N elements, written; elements between rows stay as they are     */
  const void* residual;  /* device, M rows of N elements; required iff ST_EPI_RESIDUAL*.  May be y itself, row */
                         /* for row, but not overlap it otherwise                                             */
} st_matmul_desc;

typedef struct st_matmul_plan_info {
  int32_t n_tenants, host_only;
  int32_t launches;        /* kernels per run: tenants whose operand types or kinds of tile differ go in one each */
  int32_t reserved;
  int64_t n_items;         /* workgroups of all launches                                                      */
  int64_t flops, bytes;    /* 2 M N K, and every operand once, over all tenants                               */
  int64_t workspace_bytes; /* partial sums and counters of divided reductions                                 */
} st_matmul_plan_info;

typedef struct st_matmul_tenant_info {
  int32_t tile_cfg;        /* index into st_matmul_tile_shape()                                               */
  int32_t MT, NT;          /* rows and outputs per tile                                                       */
  int32_t tiles_m, tiles_n, split_k;
  int64_t item_count;
} st_matmul_tenant_info;

typedef struct st_matmul st_matmul; /* opaque */

/* Validates the descriptors, picks a tile shape and a division of the reduction per tenant, lists the work items and uploads
 * them.  Of opts (NULL: defaults) tile_cfg, split_k and host_only are read, as in st_conv_plan.
 * n_tenants = 0, or M = 0 everywhere, gives a plan whose runs do nothing.
 * ST_ERR_UNSUPPORTED: a row longer than 2^20 elements or rows further apart than 2^21; more than 2^31 tiles. */
st_status st_matmul_plan(const st_matmul_desc* descs, int32_t n_tenants, const st_plan_opts* opts, st_matmul** out_plan);
st_status st_matmul_run(const st_matmul* plan, void* hip_stream);
/* All tenants' pointers at once, in stream order (as st_conv_plan_rebind_all): x, w, bias, y and residual are taken from descs,
 * everything else in them is ignored. */
st_status st_matmul_rebind_all(st_matmul* plan, const st_matmul_desc* descs, int32_t n_tenants, void* hip_stream);
st_status st_matmul_get_info(const st_matmul* plan, st_matmul_plan_info* out);
st_status st_matmul_get_tenant_info(const st_matmul* plan, int32_t tenant, st_matmul_tenant_info* out);
void st_matmul_destroy(st_matmul* plan);
/* Tile family: rows and outputs of config `index`; ST_ERR_INVALID_ARG past the end. */
st_status st_matmul_tile_shape(int32_t index, int32_t* MT, int32_t* NT);
int32_t st_matmul_tile_count(void);

#ifdef __cplusplus
}
#endif
#endif /* ST_LM_H */
