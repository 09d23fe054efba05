// Matrix products of several tenants for gfx950 (MI355X): y = act(x w^T + bias + residual), one workgroup per output tile or slice
// of its reduction.
//
// Both operands have the reduction index contiguous, so a 16-byte chunk of a row is an MFMA operand as it stands.  w is operand A
// and x operand B: a lane then ends with 4 consecutive outputs of one row.  The reduction runs over whole 16-byte chunks; what is
// left of a row (K off the vector) is one more MFMA step whose operands are put together element by element.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "st_launch.h"
#include "st_lm_internal.h"
#include "st_tiles.hpp"

namespace st {

typedef __attribute__((address_space(4))) const MatmulDev ConstMatmul;
typedef __attribute__((address_space(4))) const MatmulItem ConstMatmulItem;

// ---- epilogue -------------------------------------------------------------------------------------------------------
// v/2 erfc(-v/sqrt 2) = max(v, 0) - |v| q(|v|) with q(z) = erfc(z/sqrt 2)/2 = e^(-z^2/2) r(z); r is smooth and falls from 1/2 like 0.4/z, and
// is taken as a polynomial in t = 1/(1 + 0.35 z), fitted to the least relative error on [0, 13.5] (3.6e-7), behind which e^(-z^2/2) is below the
// smallest normal number.  Neither tail cancels, as 1 + erf would, at a third of the instructions of the library's function (two products
// 4096x8192x4096 with it 466 us, without an activation 446).  Measured against 64 bits, relative: 5.4e-7 for positive v; for negative ones 6.0e-7 down to -1 and 1.0e-6
// to -4, then the rounding of the exponent z^2/2 shows: 2.2e-6 at -6, 7.8e-6 at -13.
__device__ __forceinline__ float gelu_f32(float v) {
  const float z = __builtin_fabsf(v), t = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.35f, 1.f));
  float r = 0.04885588213801384f;
  r = __builtin_fmaf(r, t, -0.20177894830703735f);
  r = __builtin_fmaf(r, t, 0.24009785056114197f);
  r = __builtin_fmaf(r, t, -0.016571706160902977f);
  r = __builtin_fmaf(r, t, 0.155751571059227f);
  r = __builtin_fmaf(r, t, 0.1334092766046524f);
  r = __builtin_fmaf(r, t, 0.1402631551027298f);
  r = __builtin_fmaf(r, t, -2.69360352831427e-05f);
  const float q = r * __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  return relu_f32(v) - __builtin_amdgcn_fmed3f(z, 0.f, 16.f) * q;      // q is 0 long before z = 16, and so is their product for an infinite z
}
__device__ __forceinline__ float exp_neg(float v) { return __builtin_amdgcn_exp2f(v * -1.4426950408889634f); }      // e^-v
__device__ __forceinline__ float silu_f32(float v) { return v * __builtin_amdgcn_rcpf(1.f + exp_neg(v)); }
// v/2 (1 + tanh u) = v / (1 + e^(-2u))
__device__ __forceinline__ float gelu_tanh_f32(float v) {
  const float u = 1.5957691216057308f * (v + 0.044715f * v * v * v);
  return v * __builtin_amdgcn_rcpf(1.f + exp_neg(u));
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool f32, int dt) {
  if (f32) return ((const float*)p)[i];
  const uint16_t h = ((const uint16_t*)p)[i];
  return dt == ST_DT_BF16 ? bf16_bits_to_f32(h) : f16_bits_to_f32(h);
}

template <int W>
__device__ __forceinline__ void activate(uint32_t epi, float (&v)[W]) {
  if (epi & ST_EPI_RELU) {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = relu_f32(v[e]);
  } else if (epi & ST_EPI_GELU) {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = gelu_f32(v[e]);
  } else if (epi & ST_EPI_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = gelu_tanh_f32(v[e]);
  } else if (epi & ST_EPI_SILU) {
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = silu_f32(v[e]);
  }
}

// Vectors at any address that is a multiple of the element's size: the hardware takes them, and one such access costs less than one per element.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// W (4 or 8) consecutive values of one row
template <int DT, int W>
__device__ __forceinline__ void load_row(const void* p, int64_t i, bool f32, float (&v)[W]) {
  if (DT == ST_DT_F32 || f32) {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
      const f32x4 a = *(const f32x4_any*)((const float*)p + i + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = a[e];
    }
  } else {
    uint32_t a[W / 2];
    if constexpr (W == 8) {
      const u32x4 b = *(const u32x4_any*)((const uint16_t*)p + i);
      a[0] = b[0], a[1] = b[1], a[2] = b[2], a[3] = b[3];
    } else {
      const u32x2_any b = *(const u32x2_any*)((const uint16_t*)p + i);
      a[0] = b[0], a[1] = b[1];
    }
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = unpack16<DT>(a[e / 2], e & 1);
  }
}

// What a lane needs to finish W consecutive outputs [n, n + W) of any row from their sums.
template <int DT, int W>
struct RowEnd {
  const void* res;
  void* y;
  int64_t ldr, ldy;
  uint32_t epi;
  int n, left;            // outputs that there are from n on
  bool f32, whole;
  float bias[W];

  __device__ __forceinline__ RowEnd(ConstMatmul& T, int first) {
    n = first;
    left = T.N - n;
    whole = left >= W;
    epi = T.epilogue;
    f32 = DT == ST_DT_F32 || T.out_f32 != 0;
    res = T.res, y = T.y, ldr = T.ldr, ldy = T.ldy;
#pragma unroll
    for (int e = 0; e < W; ++e) bias[e] = 0.f;
    if (left > 0 && (epi & ST_EPI_BIAS)) {
      if (whole) {
        load_row<DT, W>(T.bias, n, false, bias);
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e) bias[e] = e < left ? load_elem(T.bias, n + e, DT == ST_DT_F32, DT) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void operator()(int64_t m, float (&v)[W]) const {
    if (left <= 0) return;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] += bias[e];
    float r[W];
    if (epi & (ST_EPI_RESIDUAL | ST_EPI_RESIDUAL_LAST)) {
      const int64_t at = m * ldr + n;
      if (whole) {
        load_row<DT, W>(res, at, f32, r);
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e) r[e] = e < left ? load_elem(res, at + e, f32, DT) : 0.f;
      }
    }
    if (epi & ST_EPI_RESIDUAL) {
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] += r[e];
    }
    activate(epi, v);
    if (epi & ST_EPI_RESIDUAL_LAST) {
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] += r[e];
    }
    const int64_t at = m * ldy + n;
    if (f32) {
      float* to = (float*)y + at;
      if (whole) {
#pragma unroll
        for (int q = 0; q < W / 4; ++q) *(f32x4_any*)(to + 4 * q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (e < left) to[e] = v[e];
      }
    } else if constexpr (DT != ST_DT_F32) {
      uint16_t* to = (uint16_t*)y + at;
      uint32_t o[W / 2];
#pragma unroll
      for (int e = 0; e < W / 2; ++e) o[e] = pack16<DT>(v[2 * e], v[2 * e + 1]);
      if (whole) {
        if constexpr (W == 8) *(u32x4_any*)to = u32x4{o[0], o[1], o[2], o[3]};
        else *(u32x2_any*)to = u32x2_any{o[0], o[1]};
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (e < left) to[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
      }
    }
  }
};

// The elements of a row behind its whole 16-byte chunks, as one chunk; zeros for a row that there is not.  Where the row is as long as a
// chunk, it is the row's last one with what the whole chunks have cleared: the same places in both operands.
template <int DT>
__device__ __forceinline__ u32x4 row_end(const void* p, int64_t row, int64_t rows, int ld, int K, bool mine) {
  constexpr int ES = ElemOf<DT>::ES, VEC = 16 / ES;
  u32x4 out = {0u, 0u, 0u, 0u};
  if (!mine || row >= rows) return out;
  const int left = K % VEC;
  if (K >= VEC) {
    const u32x4 v = *(const u32x4_any*)((const char*)p + (row * ld + K - VEC) * ES);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t keep = ES == 4 ? (d >= VEC - left ? 0xffffffffu : 0u) : (2 * d >= VEC - left ? 0x0000ffffu : 0u) | (2 * d + 1 >= VEC - left ? 0xffff0000u : 0u);
      out[d] = v[d] & keep;
    }
    return out;
  }
#pragma unroll
  for (int e = 0; e < VEC - 1; ++e) {
    if (e < K) {
      const int64_t i = row * ld + e;
      if constexpr (ES == 4) out[e] = ((const uint32_t*)p)[i];
      else out[e >> 1] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (e & 1));
    }
  }
  return out;
}

// Publishes this workgroup's partial sums and returns whether it is the last of its tile, which then has the slices' sum, in slice
// order.  get(q) / set(q, v): the thread's q-th group of four sums, at 16 (q THREADS + thread) bytes of its slice; a slice is as long as the
// tile's fp32 sums, SLICE bytes, and a group past its end is not one of the tile's.  As in st_tiles.hpp: device-scope stores and loads, no L2-wide
// fence, nobody waits.
template <int NQ, int THREADS, uint32_t SLICE, class Get, class Set>
__device__ __forceinline__ bool join_slices(ConstMatmul& T, const MatmulItem it, Get&& get, Set&& set, uint32_t* flag) {
  const int tid = (int)threadIdx.x, split = T.split;
  const int64_t tile = (int64_t)it.tile_m * T.tiles_n + it.tile_n;
  static_assert(SLICE == NQ * THREADS * 16u || (NQ == 1 && SLICE < THREADS * 16u), "groups fill a slice, or one is enough");
  float* base = T.ws + tile * split * (SLICE / 4);
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, (uint32_t)split * SLICE);
  // A group's place is the thread's plus a scalar.  Nothing but scalar instructions may come between these stores and the wait: a vector
  // instruction right behind a store with a scalar offset has been seen to overwrite registers that the store had still to read
  // (two values of eight lanes, in one run out of three of a 256x256 fp32 tile), and the compiler puts no distance between such two.
  const uint32_t mine = (uint32_t)(tid * 16) < SLICE ? (uint32_t)(tid * 16) : kInvalidOffset;
  __builtin_amdgcn_sched_barrier(0);
  static_for<NQ>([&](auto Q) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, get(Q)), rs, (int)mine, (int)(it.slice * SLICE) + decltype(Q)::value * THREADS * 16, kAuxDeviceCoherent);
  });
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_sched_barrier(0);
  __syncthreads();
  if (tid == 0) {
    const uint32_t old = __hip_atomic_fetch_add(&T.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t last = old == (uint32_t)(split - 1);
    if (last) __hip_atomic_store(&T.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  if (*flag == 0u) return false;
  constexpr int QB = NQ < 4 ? NQ : 4, SB = 4;
  static_assert(NQ % QB == 0, "batches");
  static_for<NQ / QB>([&](auto Q0) {
    constexpr int q0 = decltype(Q0)::value * QB;
    f32x4 sum[QB];
#pragma unroll
    for (int q = 0; q < QB; ++q) sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < split; s0 += SB) {
      f32x4 part[SB][QB];
#pragma unroll
      for (int s = 0; s < SB; ++s)
#pragma unroll
        for (int q = 0; q < QB; ++q) {
          const uint32_t off = s0 + s < split ? mine : kInvalidOffset;
          part[s][q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, (s0 + s) * (int)SLICE + (q0 + q) * THREADS * 16, kAuxDeviceCoherent));
        }
#pragma unroll
      for (int s = 0; s < SB; ++s)
#pragma unroll
        for (int q = 0; q < QB; ++q) sum[q] += part[s][q];
    }
    static_for<QB>([&](auto Q) { set(std::integral_constant<int, q0 + decltype(Q)::value>{}, sum[decltype(Q)::value]); });
  });
  return true;
}

// ---- few rows: the weights stream from memory to registers -----------------------------------------------------------
// 16 R rows x 16 F outputs per workgroup.  The four wavefronts divide the slice's reduction; a lane (i = lane mod 16, g = lane / 16)
// loads 16 bytes of output row i and of row i of x, chunk g of a 64-byte unit, which is a 16x16 MFMA operand; the four partial
// sums meet in LDS.  Bound by reading w once; x is small and comes from the L2 for every workgroup.
template <int DT, int R, int F>
__global__ __launch_bounds__(256) void st_matmul_skinny_kernel(const MatmulDev* table, const MatmulItem* items) {
  constexpr int ES = ElemOf<DT>::ES, VEC = 16 / ES;
  constexpr int UN = R + F <= 2 ? 8 : R + F <= 4 ? 4 : 2;      // units in flight, twice over
  __shared__ f32x4 part[4][R * F][64];
  __shared__ uint32_t flag;
  const ConstMatmulItem& ci = ((ConstMatmulItem*)items)[blockIdx.x];
  const MatmulItem it = {ci.tenant, ci.tile_m, ci.tile_n, ci.slice};
  ConstMatmul& T = ((ConstMatmul*)table)[it.tenant];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, g = lane >> 4;
  const int m0 = (int)it.tile_m * 16 * R, n0 = (int)it.tile_n * 16 * F;
  const int rows_x = T.M - m0 < 16 * R ? T.M - m0 : 16 * R, rows_w = T.N - n0 < 16 * F ? T.N - n0 : 16 * F;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc((const char*)T.x + (int64_t)m0 * T.ldx * ES, (uint32_t)(((int64_t)(rows_x - 1) * T.ldx + T.K) * ES));
  const __amdgpu_buffer_rsrc_t rw = make_rsrc((const char*)T.w + (int64_t)n0 * T.ldw * ES, (uint32_t)(((int64_t)(rows_w - 1) * T.ldw + T.K) * ES));
  const int chunks = T.K / VEC, units = (chunks + 3) / 4;
  const int s_begin = (int)it.slice * T.per_split, s_end = s_begin + T.per_split < units ? s_begin + T.per_split : units;
  const int each = (s_end - s_begin + 3) / 4;
  int u = s_begin + wave * each;
  const int u_end = u + each < s_end ? u + each : s_end;

  uint32_t ox[R], ow[F];
#pragma unroll
  for (int r = 0; r < R; ++r) ox[r] = r * 16 + i < rows_x ? (uint32_t)((r * 16 + i) * T.ldx * ES + g * 16) : kInvalidOffset;
#pragma unroll
  for (int f = 0; f < F; ++f) ow[f] = f * 16 + i < rows_w ? (uint32_t)((f * 16 + i) * T.ldw * ES + g * 16) : kInvalidOffset;
  typedef Mma<DT, 16> Op;
  f32x4 acc[F][R];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int r = 0; r < R; ++r) acc[f][r] = f32x4{0.f, 0.f, 0.f, 0.f};

  struct Batch { u32x4 x[UN][R], w[UN][F]; };
  auto fetch = [&](Batch& b, int at) {
#pragma unroll
    for (int s = 0; s < UN; ++s) {
      // a unit past the range, or a chunk past the row, is out of every buffer's range
      const uint32_t kill = (at + s < u_end && (at + s) * 4 + g < chunks) ? 0u : kInvalidOffset;
#pragma unroll
      for (int f = 0; f < F; ++f) b.w[s][f] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)((ow[f] + (uint32_t)((at + s) * 64)) | kill), 0, 0);
#pragma unroll
      for (int r = 0; r < R; ++r) b.x[s][r] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)((ox[r] + (uint32_t)((at + s) * 64)) | kill), 0, 0);
    }
  };
  auto multiply = [&](const Batch& b) {
#pragma unroll
    for (int s = 0; s < UN; ++s)
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[f][r] = Op::run(b.w[s][f], b.x[s][r], acc[f][r]);
  };
  if (u < u_end) {
    Batch b0, b1;
    fetch(b0, u);
    for (; u < u_end; u += 2 * UN) {
      fetch(b1, u + UN);
      multiply(b0);
      fetch(b0, u + 2 * UN);
      multiply(b1);
    }
  }
  if (T.K % VEC != 0 && s_end == units && wave == 3) {
    u32x4 ex[R];
#pragma unroll
    for (int r = 0; r < R; ++r) ex[r] = row_end<DT>(T.x, (int64_t)m0 + r * 16 + i, T.M, T.ldx, T.K, g == 0);
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const u32x4 ew = row_end<DT>(T.w, (int64_t)n0 + f * 16 + i, T.N, T.ldw, T.K, g == 0);
#pragma unroll
      for (int r = 0; r < R; ++r) acc[f][r] = Op::run(ew, ex[r], acc[f][r]);
    }
  }
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int r = 0; r < R; ++r) part[wave][f * R + r][lane] = acc[f][r];
  __syncthreads();
  // a thread takes four outputs of a row: block q, lane l of the MFMA layout
  constexpr int NQ = (R * F + 3) / 4;
  f32x4 v[NQ];
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const int q = k * 4 + wave;
    v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (q < R * F) v[k] = (part[0][q][lane] + part[1][q][lane]) + (part[2][q][lane] + part[3][q][lane]);
  }
  if (T.split > 1 && !join_slices<NQ, 256, R * F * 1024>(T, it, [&](auto Q) { return v[decltype(Q)::value]; }, [&](auto Q, f32x4 s) { v[decltype(Q)::value] = s; }, &flag)) return;
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const int q = k * 4 + wave;
    if (q < R * F) {
      const int f = q / R, r = q % R, m = m0 + r * 16 + i;
      float o[4] = {v[k][0], v[k][1], v[k][2], v[k][3]};
      const RowEnd<DT, 4> finish(T, n0 + f * 16 + 4 * g);
      if (m < T.M) finish(m, o);
    }
  }
}

// ---- tiles through LDS -------------------------------------------------------------------------------------------------
// MT rows x NT outputs, WM x WN wavefronts, 32x32 MFMA blocks, 128 bytes of the reduction per row and step, ST steps resident.
// Operands go from memory to LDS directly, 16-byte chunk c of row r to position c ^ (r mod 8), so that the eight rows that an
// operand read takes at a time lie in different banks.  One barrier per step, placed before the last quarter of its MFMAs: by then
// all its operands are in registers, so its stage can be refilled and the next step's operands read while that quarter runs.
template <int DT, int MT, int NT, int WM, int WN, int ST>
__global__ __launch_bounds__(WM * WN * 64) void st_matmul_tile_kernel(const MatmulDev* table, const MatmulItem* items) {
  constexpr int ES = ElemOf<DT>::ES, VEC = 16 / ES, KB = kMatmulStepBytes, WAVES = WM * WN, THREADS = WAVES * 64;
  constexpr int BM = MT / WM / 32, BN = NT / WN / 32;
  constexpr int kStage = (MT + NT) * KB, LX = MT * KB / 1024 / WAVES, LW = NT * KB / 1024 / WAVES, NL = LX + LW;
  constexpr int NW = BN * 32, kPitch = NW + 4;                  // epilogue: floats per row in LDS
  constexpr int kOut = WAVES * 32 * kPitch * 4;
  constexpr int kSmem = ST * kStage > kOut ? ST * kStage : kOut;
  static_assert(LX * WAVES * 1024 == MT * KB && LW * WAVES * 1024 == NT * KB, "whole load instructions");
  __shared__ __align__(128) char smem[kSmem];
  __shared__ uint32_t flag;
  const ConstMatmulItem& ci = ((ConstMatmulItem*)items)[blockIdx.x];
  const MatmulItem it = {ci.tenant, ci.tile_m, ci.tile_n, ci.slice};
  ConstMatmul& T = ((ConstMatmul*)table)[it.tenant];
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave % WM) * BM * 32, wn0 = (wave / WM) * BN * 32;
  const int m0 = (int)it.tile_m * MT, n0 = (int)it.tile_n * NT;
  const int rows_x = T.M - m0 < MT ? T.M - m0 : MT, rows_w = T.N - n0 < NT ? T.N - n0 : NT;
  const u32x4 rx = rsrc_words((const char*)T.x + (int64_t)m0 * T.ldx * ES, (uint32_t)(((int64_t)(rows_x - 1) * T.ldx + T.K) * ES));
  const u32x4 rw = rsrc_words((const char*)T.w + (int64_t)n0 * T.ldw * ES, (uint32_t)(((int64_t)(rows_w - 1) * T.ldw + T.K) * ES));
  const int chunks = T.K / VEC, steps = (chunks + 7) / 8;
  const int s_begin = (int)it.slice * T.per_split, s_end = s_begin + T.per_split < steps ? s_begin + T.per_split : steps;

  const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;
  uint32_t vx[LX], vw[LW];
#pragma unroll
  for (int l = 0; l < LX; ++l) {
    const int row = (l * WAVES + wave) * 8 + lrow;
    vx[l] = row < rows_x ? (uint32_t)(row * T.ldx * ES + chunk * 16) : kInvalidOffset;
  }
#pragma unroll
  for (int l = 0; l < LW; ++l) {
    const int row = (l * WAVES + wave) * 8 + lrow;
    vw[l] = row < rows_w ? (uint32_t)(row * T.ldw * ES + chunk * 16) : kInvalidOffset;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + (uint32_t)wave * 1024u;
  // load instruction L of step s, into the stage at LDS offset `stage`; past the range and past the row's end every lane is out of range
  auto issue = [&](auto L, int s, uint32_t stage, uint32_t kill) {
    constexpr int l = decltype(L)::value;
    const uint32_t soff = (uint32_t)s * KB;
    if constexpr (l < LX) load_to_lds<0, l * WAVES * 1024>(rx, vx[l] | kill, soff, lds0 + stage);
    else load_to_lds<0, MT * KB + (l - LX) * WAVES * 1024>(rw, vw[l - LX] | kill, soff, lds0 + stage);
  };
  auto killed = [&](int s) { return s < s_end && s * 8 + chunk < chunks ? 0u : kInvalidOffset; };

  typedef Mma<DT, 32> Op;
  typename Op::Acc acc[BN][BM];
#pragma unroll
  for (int j = 0; j < BN; ++j)
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;

  struct Frags { u32x4 x[BM], w[BN]; };
  const int r32 = lane & 31, half = lane >> 5;
  uint32_t sub_off[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) sub_off[s] = (uint32_t)(r32 * KB + (((s * 2 + half) ^ (r32 & 7)) << 4));
  auto read = [&](Frags& f, uint32_t stage, int sub) {
#pragma unroll
    for (int j = 0; j < BN; ++j) f.w[j] = *(const u32x4*)(smem + stage + sub_off[sub] + MT * KB + (wn0 + j * 32) * KB);
#pragma unroll
    for (int i = 0; i < BM; ++i) f.x[i] = *(const u32x4*)(smem + stage + sub_off[sub] + (wm0 + i * 32) * KB);
  };
  // A sub-step's MFMAs, with load instructions [FROM, TO) of step s spread among them: the vector-memory unit takes 16 clocks for each,
  // and a burst of them would hold up the MFMAs behind it.
  auto multiply = [&](const Frags& f, auto FROM, auto TO, int s, uint32_t stage, uint32_t kill) __attribute__((always_inline)) {
    constexpr int from = decltype(FROM)::value, n = decltype(TO)::value - from, N = BN * BM;
    __builtin_amdgcn_s_setprio(1);      // 8192^3 in bf16 838 us -> 826
    static_for<N>([&](auto M) __attribute__((always_inline)) {
      constexpr int m = decltype(M)::value, j = m / BM, i = m % BM, l0 = from + m * n / N, l1 = from + (m + 1) * n / N;
      acc[j][i] = Op::run(f.w[j], f.x[i], acc[j][i]);
      static_for<l1 - l0>([&](auto L) __attribute__((always_inline)) { issue(std::integral_constant<int, l0 + decltype(L)::value>{}, s, stage, kill); });
      if constexpr (l1 > l0) __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_s_setprio(0);
  };
  constexpr std::integral_constant<int, 0> none;
  constexpr std::integral_constant<int, NL / 2> half_of;
  constexpr std::integral_constant<int, NL> all_of;

  // Half of a step's loads go out behind the barrier that frees its stage, half with the sub-step after.
  if (s_begin < s_end) {
    static_for<ST>([&](auto S) {
      constexpr int s = decltype(S)::value;
      const uint32_t kill = killed(s_begin + s);
      static_for<s < ST - 1 ? NL : NL / 2>([&](auto L) { issue(L, s_begin + s, s * kStage, kill); });
    });
    wait_loads_barrier<(ST - 2) * NL + NL / 2>();
    Frags f0, f1;
    read(f0, 0, 0);
    uint32_t cur = 0, last = (ST - 1) * kStage, kill = killed(s_begin + ST - 1);
    for (int s = s_begin; s < s_end; ++s) {
      const uint32_t next = cur + kStage < ST * kStage ? cur + kStage : 0;
      read(f1, cur, 1);
      multiply(f0, half_of, all_of, s + ST - 1, last, kill);
      read(f0, cur, 2);
      multiply(f1, none, none, 0, 0, 0);
      read(f1, cur, 3);
      multiply(f0, none, none, 0, 0, 0);
      kill = killed(s + ST);
      wait_loads_barrier<(ST - 2) * NL>();
      read(f0, next, 0);
      multiply(f1, none, half_of, s + ST, cur, kill);
      last = cur;
      cur = next;
    }
  }
  if (T.K % VEC != 0 && s_end == steps) {
    Frags f;
#pragma unroll
    for (int j = 0; j < BN; ++j) f.w[j] = row_end<DT>(T.w, (int64_t)n0 + wn0 + j * 32 + r32, T.N, T.ldw, T.K, half == 0);
#pragma unroll
    for (int i = 0; i < BM; ++i) f.x[i] = row_end<DT>(T.x, (int64_t)m0 + wm0 + i * 32 + r32, T.M, T.ldx, T.K, half == 0);
    multiply(f, none, none, 0, 0, 0);
  }
  wait_loads_barrier<0>();          // nothing is on its way into LDS any more, and nobody reads operands

  if (T.split > 1) {
    auto get = [&](auto Q) {
      constexpr int q = decltype(Q)::value, j = q / 4 / BM, i = q / 4 % BM, g = q % 4;
      return f32x4{acc[j][i][4 * g], acc[j][i][4 * g + 1], acc[j][i][4 * g + 2], acc[j][i][4 * g + 3]};
    };
    auto set = [&](auto Q, f32x4 v) {
      constexpr int q = decltype(Q)::value, j = q / 4 / BM, i = q / 4 % BM, g = q % 4;
      acc[j][i][4 * g] = v[0], acc[j][i][4 * g + 1] = v[1], acc[j][i][4 * g + 2] = v[2], acc[j][i][4 * g + 3] = v[3];
    };
    if (!join_slices<BN * BM * 4, THREADS, MT * NT * 4>(T, it, get, set, &flag)) return;
  }
  // A wavefront turns its rows round in LDS of its own, 32 of them at a time, so that a row's outputs leave together.
  float* mine = (float*)smem + wave * 32 * kPitch;
  constexpr int LPR = NW / 8, RPP = 64 / LPR;
  const int c8 = lane % LPR * 8, rr = lane / LPR;
  const RowEnd<DT, 8> finish(T, n0 + wn0 + c8);
  const int64_t rows_end = T.M;
  static_for<BM>([&](auto I) {
    constexpr int i = decltype(I)::value;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < BN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(mine + r32 * kPitch + j * 32 + 8 * g + 4 * half) = f32x4{acc[j][i][4 * g], acc[j][i][4 * g + 1], acc[j][i][4 * g + 2], acc[j][i][4 * g + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < 32 / RPP; ++p) {
      const int r = p * RPP + rr;
      const int64_t m = (int64_t)m0 + wm0 + i * 32 + r;
      float o[8];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f32x4 a = *(const f32x4*)(mine + r * kPitch + c8 + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[4 * q + e] = a[e];
      }
      if (m < rows_end) finish(m, o);
    }
  });
}

// ---- launches ------------------------------------------------------------------------------------------------------------
template <int DT>
static hipError_t launch_shape(int shape, unsigned blocks, void* stream, const MatmulDev* table, const MatmulItem* items) {
  switch (shape) {
    case 0: return launch(st_matmul_tile_kernel<DT, 256, 256, 4, 2, 2>, blocks, 512, stream, table, items);
    case 1: return launch(st_matmul_tile_kernel<DT, 128, 128, 2, 2, 2>, blocks, 256, stream, table, items);
    case 2: return launch(st_matmul_tile_kernel<DT, 64, 64, 2, 2, 4>, blocks, 256, stream, table, items);
    case 3: return launch(st_matmul_skinny_kernel<DT, 4, 2>, blocks, 256, stream, table, items);
    case 4: return launch(st_matmul_skinny_kernel<DT, 2, 2>, blocks, 256, stream, table, items);
    case 5: return launch(st_matmul_skinny_kernel<DT, 1, 2>, blocks, 256, stream, table, items);
    case 6: return launch(st_matmul_skinny_kernel<DT, 1, 1>, blocks, 256, stream, table, items);
  }
  return hipErrorInvalidValue;
}

int launch_matmul(int dtype, int shape, const MatmulDev* table_dev, const MatmulItem* items_dev, int64_t n_items, void* stream) {
  if (n_items <= 0) return 0;
  const auto run = dtype == ST_DT_F32 ? launch_shape<ST_DT_F32> : dtype == ST_DT_BF16 ? launch_shape<ST_DT_BF16> : launch_shape<ST_DT_F16>;
  return (int)run(shape, (unsigned)n_items, stream, table_dev, items_dev);
}

}  // namespace st
