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

// How a tenant's outputs, residual and bias are reached: 16 bytes at a time where address and row length allow it.
constexpr uint32_t kMatmulVecY = 1u, kMatmulVecRes = 2u, kMatmulVecBias = 4u;

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
  uint32_t epilogue, vec;
  int32_t out_f32;
  int32_t tiles_n, split, per_split;   // per_split: steps (units of a skinny tile) per slice
  int32_t pad[5];
};
static_assert(sizeof(MatmulDev) == 128, "two lines of the scalar cache, a multiple of 16 bytes for launch_poke");

struct MatmulItem { uint32_t tenant, tile_m, tile_n, slice; };

int launch_matmul(int dtype, int shape, const MatmulDev* table_dev, const MatmulItem* items_dev, int64_t n_items, void* stream);

}  // namespace st
