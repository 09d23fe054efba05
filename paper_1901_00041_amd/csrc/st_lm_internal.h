// Internals shared by the host and device sources of the operators of language models (not part of the C ABI).
#pragma once
#include <stdint.h>

#include "st_lm.h"

namespace st {

// ---- matrix products ----------------------------------------------------------------------------------------------
// MT rows x NT outputs per workgroup.  `skinny`: few rows, operands from memory to registers, the four wavefronts divide the
// reduction; else tiles through LDS (see st_matmul.hip).
struct MatmulShape {
  int MT, NT, threads;
  bool skinny;
};
constexpr MatmulShape kMatmulShapes[] = {
    {256, 256, 512, false},   // 0
    {128, 128, 256, false},   // 1
    {64, 64, 256, false},     // 2
    {64, 32, 256, true},      // 3
    {32, 32, 256, true},      // 4
    {16, 32, 256, true},      // 5
    {16, 16, 256, true},      // 6
};
constexpr int kNumMatmulShapes = (int)(sizeof(kMatmulShapes) / sizeof(kMatmulShapes[0]));
constexpr int kMatmulStepBytes = 128;    // of a row, per step of a tile through LDS
constexpr int kMatmulUnitBytes = 64;     // of a row, per MFMA step of a skinny tile
constexpr int kMatmulMaxK = 1 << 20, kMatmulMaxLd = 1 << 21;     // a tile's rows stay below 2^31 bytes

struct MatmulDev {
  const void* x;
  const void* w;
  const void* bias;
  const void* res;
  void* y;
  float* ws;             // partial tiles of a divided reduction
  uint32_t* counters;    // one arrival counter per output tile, zero between runs
  int32_t M, N, K;
  int32_t ldx, ldw, ldy, ldr;
  uint32_t epilogue;
  int32_t out_f32;
  int32_t tiles_n, split, per_split;   // per_split: steps (units of a skinny tile) per slice
  int32_t pad[6];
};
static_assert(sizeof(MatmulDev) == 128, "two lines of the scalar cache, a multiple of 16 bytes for launch_poke");

struct MatmulItem { uint32_t tenant, tile_m, tile_n, slice; };

int launch_matmul(int dtype, int shape, const MatmulDev* table_dev, const MatmulItem* items_dev, int64_t n_items, void* stream);

// ---- attention over a paged cache in 4 bits ---------------------------------------------------------------------------
// How an st_attn_run divides the work (see st_attn.hip).  kAttnTokens1, 2: a workgroup's wavefronts take the tokens of a stretch in turn, all for
// the same rows, of which there are 16 R; kAttnRows: each wavefront takes 16 R rows of its own and all the tokens they see, or (kAttnRowsSplit) a stretch of them.
constexpr int kAttnBlock = 16;           // tokens per cache block
constexpr int kAttnStep = 32;            // tokens per step of a wavefront
constexpr int kAttnTokenWaves = 8;
constexpr int attn_row_waves(int dim) { return dim == 256 ? 8 : 4; }
constexpr int kAttnRowTokens = 64;       // of a tile that they widen together
constexpr int kAttnMaxSplit = 64;
constexpr int attn_level_steps(int dim) { return dim == 256 ? 24 : 48; }      // a stretch of rows that levels out unlike lengths is as long as that: its joining is then a twentieth of it
constexpr int kAttnTokens1 = 0, kAttnTokens2 = 1, kAttnRows = 2, kAttnRowsSplit = 3, kNumAttnKinds = 4;
// R of a kind: rows are as many as the registers hold beside their queries, scores and outputs
constexpr int attn_blocks(int kind, int dim) { return kind == kAttnTokens1 ? 1 : kind == kAttnTokens2 ? (dim == 256 ? 1 : 2) : dim == 64 ? 4 : dim == 128 ? 3 : 1; }

// Floats of a stretch's partial result with kAttnRowsSplit: each thread's outputs, maxima and sums.
constexpr int attn_row_slot(int kind, int dim) { return attn_row_waves(dim) * 64 * attn_blocks(kind, dim) * (dim / 4 + 2); }

// Bytes of a block of 16 tokens of one head, and where its parts begin.
constexpr int attn_block_bytes(int dim) { return kAttnBlock * (dim + dim / 16); }

struct AttnDev {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  void* k_out;
  void* v_out;
  void* pages;
  const int32_t* table;
  const int32_t* first;
  const int32_t* length;
  float* ws;             // partial results: [tile][split][rows][dim], then their maxima and sums, [tile][split][2][rows]; with kAttnRowsSplit slots
  uint32_t* counters;    // one arrival counter per tile, zero between runs
  uint32_t* status;      // ST_ATTN_BAD_* that runs have met
  int64_t ldq, ldk, ldv, ldo;
  int64_t page_bytes;
  int32_t heads, kv_heads, group, n_seqs;
  int32_t max_tokens, max_new, n_pages, page_shift;
  int32_t table_pages, window, causal;
  float scale;           // its size times log2(e), above zero; fp16: twice that
  int32_t row_tiles;     // per sequence and key head
  int32_t split;         // at most so many stretches.  How many, of wavefronts that take turns:
  int32_t whole;         // one for no more steps than these, else
  int32_t want;          // these, or, if it is one, so many that
  int32_t most;          // none has more steps than these, but
  int32_t least;         // so few that none but the last has fewer than these, and
  int32_t chunk;         // none has more than these.
  float root;            // With kAttnRowsSplit (a step: a tile of the workgroup): one up to `whole` steps, else the square root of root times the
                         // steps, if that is `most` or more just these, else not more than `want`; but one per attn_level_steps() up to `least`
  uint32_t flip;         // sign bits of two query elements, where scale is negative
  int32_t pad[3];
};
static_assert(sizeof(AttnDev) == 240, "a multiple of 16 bytes for launch_poke");

struct AttnItem { uint32_t tenant, seq, head, part; };   // part: row tile * split + stretch, or the stretch of new tokens
// In place of a sequence: the part-th of all sequences' parts together, or a look at all their numbers (see find_sequence in st_attn.hip).
constexpr uint32_t kAttnCheck = 0xffffffffu, kAttnFind = 0xfffffffeu;

int launch_attn(int dtype, int dim, int kind, const AttnDev* table_dev, const AttnItem* items_dev, int64_t n_items, void* stream);
// New tokens into the cache, or (read) out of it; part: the stretch of attn_move_count() of a sequence's new tokens x key heads, or (many: for
// tenants that may have 16 new tokens or more) of kAttnMoveTurns times as many.
int launch_attn_move(bool read, bool many, int dtype, int dim, const AttnDev* table_dev, const AttnItem* items_dev, int64_t n_items, void* stream);
constexpr int kAttnMoveTurns = 2;
constexpr int attn_move_count(int dim) { return 256 / (dim / 8); }

}  // namespace st
