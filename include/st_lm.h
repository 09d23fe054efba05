/*
 * st_lm.h - C ABI of the fused multi-tenant operators of language models for MI355X (gfx950): matrix products with their
 * epilogue, and attention over a paged key-value cache held in 4 bits.
 *
 * They follow st_conv.h (Section 4 of the paper: the kernels of several tenants merged into one launch): an array of
 * per-tenant descriptors with device pointers makes a plan, the plan's run calls issue its work for all tenants together.
 * A decoding step of several tenants is a product (queries, keys and values), st_attn_append, st_attn_run, and the products
 * that follow, each a call for all of them.  The conventions of st_conv.h hold:
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
 * them.  Of opts (NULL: defaults) tile_cfg, split_k and host_only are read, as in st_conv_plan; split_k as far as there are steps for it and a
 * tile's partial sums take 2^30 bytes.
 * n_tenants = 0, or M = 0 everywhere, gives a plan whose runs do nothing.
 * ST_ERR_UNSUPPORTED: a row longer than 2^20 elements or rows further apart than 2^21; 2^23 workgroups or more. */
st_status st_matmul_plan(const st_matmul_desc* descs, int32_t n_tenants, const st_plan_opts* opts, st_matmul** out_plan);
st_status st_matmul_run(const st_matmul* plan, void* hip_stream);
/* All tenants' pointers at once, in stream order (as st_conv_plan_rebind_all): x, w, bias, y and residual are taken from descs,
 * everything else in them is ignored.  Captured into a graph it happens at each replay, after which the plan has these pointers until the next call. */
st_status st_matmul_rebind_all(st_matmul* plan, const st_matmul_desc* descs, int32_t n_tenants, void* hip_stream);
st_status st_matmul_get_info(const st_matmul* plan, st_matmul_plan_info* out);
st_status st_matmul_get_tenant_info(const st_matmul* plan, int32_t tenant, st_matmul_tenant_info* out);
void st_matmul_destroy(st_matmul* plan);
/* Tile family: rows and outputs of config `index`; ST_ERR_INVALID_ARG past the end. */
st_status st_matmul_tile_shape(int32_t index, int32_t* MT, int32_t* NT);
int32_t st_matmul_tile_count(void);

/* ---- Attention over a paged cache in 4 bits -----------------------------------------------------------------------
 * The cache.  A token's key and value of one head are head_dim elements E2M1 (sign, 2 bits of exponent, 1 of mantissa: 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6) in groups of 32, each with one scale byte s that stands for 2^(s - 127).  Written from values x: with a = max|x| of the
 * group = m 2^k (1 <= m < 2), the exponent is k - 2 if m <= 1.5 and k - 1 if not, at least -126 and at most 125 (-126 for a = 0), so
 * that the largest value is never cut off below 2^127; each x is divided by the scale and rounded to the nearest element, ties to the one with the
 * even code, at most 6.  A value that is not finite makes its token's head unreadable: all its scales become 255 (keys) and 1 (values),
 * all its codes 0; attention reads its key as not a number and its value as 0.
 * Attention takes keys and values in the descriptor's dtype: bfloat16 any element under a scale of 2^-126 to 2^125; fp16 any under a scale of up to 2^14, the
 * largest that is written from that type (one above it counts as it), elements below 2^-22 as multiples of 2^-23.  fp16 outputs that would be above 65504 are 65504.
 * st_attn_read gives every element as the nearest number of dtype, in fp16 65504 at most, and not a number for keys of an unreadable head.
 * A pool is n_pages pages of st_attn_page_bytes() bytes.  A page holds page_tokens tokens: for each key head in turn its
 * page_tokens / 16 blocks, each of 16 tokens t and head_dim + head_dim / 16 bytes a token:
 *   keys' codes     [t][head_dim / 2]          byte j holds elements 2j (lower half) and 2j + 1
 *   values' codes   [16][t][head_dim / 32]     group i of head_dim / 16 elements, two to a byte as above
 *   keys' scales    [t][head_dim / 32]
 *   values' scales  [head_dim / 32][t]
 * A page is one run of bytes that means the same at any index of any pool of the same head layout: copying, forking and moving pages
 * is copying bytes and writing tables.
 *
 * A tenant's sequences.  Sequence i holds length[i] tokens, its new ones included; token p is in page table[i * table_pages +
 * p / page_tokens].  Its new tokens, the last ones, are rows first[i] .. first[i+1]-1 of q, k, v and out: row first[i] + j is token
 * p = length[i] - (first[i+1] - first[i]) + j.  table, first and length are read on the device at every run, so that a captured
 * step can be replayed on other lengths.  Every row that belongs to no sequence is left as it is, in all outputs.
 *
 * What a run finds there is checked: a page index outside the pool is not followed (its tokens are not written, and hide from
 * every query); first is held to [0, max_tokens], what a sequence has more of than max_new new tokens are left out (the rows behind
 * them are left as they are), and a length is held to [0, table_pages * page_tokens].  st_attn_status reports that it happened, and that a
 * sequence has more new tokens than tokens: those before its start see nothing (zeros), are not written and read as 0.  Attention does not
 * report pages that no new token of the sequence sees (all of it before their windows): they may be gone, and their entries hold anything. */
enum { ST_ATTN_CAUSAL = 1u };
enum { ST_ATTN_BAD_PAGE = 1, ST_ATTN_BAD_LENGTH = 2 };

typedef struct st_attn_desc {
  int32_t heads, kv_heads;   /* query heads and key heads; heads a multiple of kv_heads: query head h reads key head        */
                             /* h / (heads / kv_heads)                                                                      */
  int32_t head_dim;          /* 64, 128 or 256                                                                              */
  int32_t dtype;             /* ST_DT_BF16 or ST_DT_F16, of q, k, v and the outputs                                          */
  int32_t n_seqs;            /* sequences, >= 0                                                                             */
  int32_t max_tokens;        /* rows of q, k, v and the outputs, >= 0                                                       */
  int32_t max_new;           /* most new tokens of one sequence, >= 1                                                       */
  int32_t n_pages, page_tokens, table_pages;   /* page_tokens 16, 32, 64, ..., 1024                                         */
  int32_t window;            /* > 0 (causal only): a token sees itself and the window - 1 tokens before it; 0: all           */
  uint32_t flags;            /* ST_ATTN_CAUSAL: token p sees tokens 0 .. p of its sequence; else all length[i] of them       */
  float scale;               /* of the scores, before the softmax; finite; its size counts as 6e-31 at least, 2e38 at most (fp16 1e38) */
  int32_t reserved;          /* must be 0                                                                                   */
  int64_t ldq, ldk, ldv, ldo; /* elements from a row to the next of q, k (and k_out), v (and v_out), out; 0 = dense          */
  const void* q;             /* [max_tokens][heads][head_dim], for st_attn_run                                              */
  const void *k, *v;         /* [max_tokens][kv_heads][head_dim], for st_attn_append                                        */
  void* out;                 /* as q, for st_attn_run                                                                       */
  void *k_out, *v_out;       /* as k and v, for st_attn_read                                                                */
  void* pages;               /* n_pages * st_attn_page_bytes() bytes, a multiple of 16 as an address                        */
  const int32_t* table;      /* [n_seqs][table_pages]; entries behind a sequence's last page are not read                   */
  const int32_t* first;      /* [n_seqs + 1], ascending                                                                     */
  const int32_t* length;     /* [n_seqs]                                                                                    */
} st_attn_desc;

typedef struct st_attn_info {
  int32_t n_tenants, host_only;
  int32_t launches;          /* kernels of an st_attn_run: tenants of one head_dim, type and kind of division go in one      */
  int32_t reserved;
  int64_t n_items;           /* workgroups of these                                                                         */
  int64_t workspace_bytes;   /* partial results of divided lengths                                                          */
} st_attn_info;

typedef struct st_attn st_attn; /* opaque */

/* Bytes of a page for these kv_heads, head_dim and page_tokens (nothing else of desc is read); negative if they are not valid. */
int64_t st_attn_page_bytes(const st_attn_desc* desc);
/* Validates the descriptors, divides the work by what they allow at most (max_new, max_tokens, table_pages) and, within that, on the device by
 * the lengths that there are, uploads the tables and allocates the workspace.  A pointer may be NULL that none of the calls made with the
 * plan needs.  opts: host_only is read, and split_k (> 0: into how many parts the tokens that a row sees are divided; at most 64 are, 16 where
 * there are many rows).
 * max_new decides how a tenant's work is divided: where max_new * heads / kv_heads is up to 128 (64 with heads of 256) a workgroup's wavefronts go over a
 * sequence's tokens for the same rows, else each has rows of its own.  Sequences of one new token among prompts belong in a descriptor of their own: two tenants of a plan may read one pool, and
 * append to different pages of it.
 * ST_ERR_UNSUPPORTED: more than 2^16 heads, rows more than 2^32 elements apart; a page of 2^31 bytes, 2^30 tokens (of a table or a sequence's
 * rows), 2^24 sequences, 2^23 workgroups or more of them. */
st_status st_attn_plan(const st_attn_desc* descs, int32_t n_tenants, const st_plan_opts* opts, st_attn** out_plan);
/* New tokens' keys and values (k, v) into the cache.  Two sequences that share a page must not both write to it. */
st_status st_attn_append(const st_attn* plan, void* hip_stream);
/* What the cache holds of the new tokens, as values of dtype (k_out, v_out).  To read a sequence back from its start, call all of its
 * tokens new ones.  A token on a page outside the pool reads as 0. */
st_status st_attn_read(const st_attn* plan, void* hip_stream);
/* out = softmax(scale q k^T) v over the tokens that each new token sees, which have to be in the cache by now (its own included).
 * Scores, the softmax's maximum and sum, and the mixed values are held in fp32, weights are rounded to dtype before they
 * multiply values.  A query that sees no token gets zeros. */
st_status st_attn_run(const st_attn* plan, void* hip_stream);
/* All tenants' pointers at once, as st_matmul_rebind_all: the ten tensors and tables are taken from descs, everything else in them is ignored. */
st_status st_attn_rebind_all(st_attn* plan, const st_attn_desc* descs, int32_t n_tenants, void* hip_stream);
/* Waits for the device, then *bits = the ST_ATTN_BAD_* that any run since the last call met; they are cleared. */
st_status st_attn_status(st_attn* plan, int32_t* bits);
st_status st_attn_get_info(const st_attn* plan, st_attn_info* out);
void st_attn_destroy(st_attn* plan);

#ifdef __cplusplus
}
#endif
#endif /* ST_LM_H */
