// Attention of several tenants' sequences over paged caches in 4 bits, and the way into and out of these caches, for gfx950 (MI355X).
//
// A cache block holds 16 tokens of one head so that MFMA operands come from it without a trip through LDS:
//   scores   S^T = K Q^T, 16x16 blocks of tokens x query rows.  A lane (i = lane mod 16, g = lane / 16) holds a quarter of token i's
//            key, dim / 4 elements with one or two scales; which elements meet in one MFMA does not matter as long as the query's lanes
//            hold the same ones.  The result leaves a lane with the scores of query row i for tokens 4g .. 4g+3.
//   values   O^T = V^T P^T, dims x query rows, over 32 tokens: the weights of two blocks as they stand are operand B (tokens 4g .. 4g+3 of
//            both), and the values' codes are stored so that a lane reads, as one vector, the same four tokens of dim / 16 elements.
//   sums     of the weights, as they were rounded, lane by lane.
// Elements E2M1 become 16-bit ones, scaled, in v_cvt_scalef32_pk_*_fp4 (exact).  The softmax runs in one pass; its reference is raised, and
// what has been summed scaled down, only when a score exceeds it by 2^kLag, so that most steps need nothing from another lane.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "st_launch.h"
#include "st_lm_internal.h"
#include "st_tiles.hpp"

namespace st {

typedef __attribute__((address_space(4))) const AttnDev ConstAttn;
typedef __attribute__((address_space(4))) const AttnItem ConstAttnItem;
typedef __attribute__((address_space(4))) const int32_t ConstInt;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));      // tensors ask no more of an address than their element's size
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// A sequence's numbers, held to what the descriptor allows.
struct Seq {
  int first;      // row of its first new token
  int n;          // new tokens, at most max_new
  int length;     // tokens in the cache
  int before;     // position of the first new token (negative: there are more new tokens than tokens)
};
__device__ __forceinline__ Seq sequence(ConstAttn& T, int seq, bool reports) {      // reports: this thread, what was held
  const int a = ((ConstInt*)T.first)[seq], b = ((ConstInt*)T.first)[seq + 1], len = ((ConstInt*)T.length)[seq];
  const int64_t cap = (int64_t)T.table_pages << T.page_shift;
  const int f0 = a < 0 ? 0 : a > T.max_tokens ? T.max_tokens : a, f1 = b < f0 ? f0 : b > T.max_tokens ? T.max_tokens : b;
  const int length = len < 0 ? 0 : len > cap ? (int)cap : len;
  const int all = f1 - f0, n = all < T.max_new ? all : T.max_new;
  if (reports && (f0 != a || f1 != b || length != len || n != all || all > length)) atomicOr(T.status, (uint32_t)ST_ATTN_BAD_LENGTH);
  return {f0, n, length, length - all};
}
// The last token that its j-th new token sees; below 0 for none, which are those before the sequence's start.
__device__ __forceinline__ int last_seen(ConstAttn& T, const Seq& S, int j) { return T.causal || S.before + j < 0 ? S.before + j : S.length - 1; }
// Where max_new allows far more work than max_tokens, items are not listed for each sequence, which leaves most of them without any, but
// as many as there can be at most in all (kAttnFind): the part-th of all parts belongs to the sequence that is found here, 64 sequences at a
// time, and is that sequence's part-th then.  parts(n): of a sequence with n new tokens.  One more item (kAttnCheck) looks at every sequence's numbers.
template <class Parts>
__device__ __forceinline__ bool find_sequence(ConstAttn& T, uint32_t item_seq, int& seq, int& part, Parts&& parts) {
  seq = (int)item_seq;
  if (__builtin_expect(item_seq < kAttnFind, 1)) return true;
  const int lane = (int)threadIdx.x & 63;
  if (item_seq == kAttnCheck) {
    for (int s = (int)threadIdx.x; s < T.n_seqs; s += (int)blockDim.x) (void)sequence(T, s, true);
    return false;
  }
  for (int s0 = 0, before = 0; s0 < T.n_seqs; s0 += 64) {      // before <= part: no sum passes 2^31
    int up_to = s0 + lane < T.n_seqs ? parts(sequence(T, s0 + lane, false).n) : 0;
    up_to = up_to < 1 << 24 ? up_to : 1 << 24;
    const int mine = up_to;
    for (int k = 1; k < 64; k *= 2) {
      const int below = __shfl_up(up_to, k);
      up_to += lane >= k ? below : 0;
    }
    const uint64_t behind = __ballot(before + up_to > part);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind);
      seq = s0 + at;
      part -= before + __builtin_amdgcn_readlane(up_to - mine, at);
      return true;
    }
    before += __builtin_amdgcn_readlane(up_to, 63);
  }
  return false;
}
// A stretch of a sequence's table, an entry a lane, so that looking a page up costs no trip to memory (nor a scalar load, which would
// make every wait for LDS a wait for all of it).
struct Table {
  int entry, base;
  const int32_t* row;
  int last;               // column of the last token that is looked up
  __device__ __forceinline__ void load(int column, int lane) {
    base = column;
    entry = row[column + lane < last ? column + lane : last];
    __builtin_amdgcn_s_waitcnt(0x0f70);      // here: else every look-up waits for all loads in flight, in case this one is among them
  }
  __device__ __forceinline__ Table(ConstAttn& T, int seq, int first_token, int last_token, int lane) {
    row = T.table + (int64_t)seq * T.table_pages;
    last = last_token >> T.page_shift;
    load(first_token >> T.page_shift, lane);
  }
  // the page of token t (not before those already looked up, except by a few), or -1; t may lie behind the last one
  __device__ __forceinline__ int page(ConstAttn& T, int t, int lane) {
    const int column = t >> T.page_shift;
    if (column > last) return -1;
    if ((unsigned)(column - base) >= 64u) load(column, lane);
    const int p = __builtin_amdgcn_readlane(entry, column - base);
    return (uint32_t)p < (uint32_t)T.n_pages ? p : -1;
  }
};
__device__ __forceinline__ const char* block_of(ConstAttn& T, int page, int head, int t, int block_bytes) {
  const uint32_t in_page = (uint32_t)t & ((1u << T.page_shift) - 1u), blocks = 1u << (T.page_shift - 4);
  return (const char*)T.pages + (uint64_t)(uint32_t)page * (uint32_t)T.page_bytes + ((uint32_t)head * blocks + (in_page >> 4)) * (uint32_t)block_bytes;
}

// ---- elements and scales ----------------------------------------------------------------------------------------------
template <int DT, int BYTE>
__device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {      // byte BYTE's two elements, the lower one first
  if constexpr (DT == ST_DT_BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, BYTE));
}
// fp16 ends at 65504, but a group whose largest value is above 49152 has the scale 2^14, under which the elements 4 and 6 are 65536 and 98304.
// Attention therefore widens under half the scale, kHalved of it in all: scores are made up for by twice the factor behind them, outputs by the division
// by the sum, both without a rounding.  What it costs: elements below 2^-22 become multiples of 2^-23.
template <int DT> constexpr bool kHalved = DT == ST_DT_F16;
// Scales above these (of another type, or memory that was never written) count as these, so that no value is infinite (and weight 0 times it not a number).
template <int DT> constexpr uint32_t kMostScale = kHalved<DT> ? 141u : 252u;
template <int DT>
__device__ __forceinline__ float value_scale(uint32_t code) {
  const uint32_t held = code < kMostScale<DT> ? code : kMostScale<DT>;
  return __builtin_bit_cast(float, kHalved<DT> ? ((held > 1u ? held : 1u) << 23) - (1u << 23) : held << 23);
}
template <int DT>
__device__ __forceinline__ float key_scale(uint32_t code) {      // 255: not a number
  const float f = value_scale<DT>(code);
  return code == 255u ? __builtin_bit_cast(float, 0x7fc00000u) : f;
}

template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  if constexpr (DT == ST_DT_BF16) return pack16<DT>(a, b);
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}
// The larger of two values in one instruction: as a median with an infinity that the compiler does not know (fmaxf of what an MFMA left
// costs another one per operand, which quiets NaNs).
__device__ __forceinline__ float max_raw(float a, float b, float inf) { return __builtin_amdgcn_fmed3f(a, b, inf); }
// sum + both of a pair
template <int DT>
__device__ __forceinline__ float add_pair(uint32_t pair, float sum) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  if constexpr (DT == ST_DT_BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
  else return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), __builtin_bit_cast(f16x2, 0x3c003c00u), sum, false);
}
__device__ __forceinline__ float sum_of_row(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float max_of_row(float v) {      // over the four lanes that hold a query row
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// ---- one wavefront's rows over a stretch of tokens -----------------------------------------------------------------------
// MFMA_SUMS: the weights' sums by an MFMA with ones, which costs the fewest instructions where the vector unit is short (six prompts 454 us ->
// 444); else by dot products, which costs the fewest registers (64 single tokens 70.6 us -> 67.2).
template <int DT, int D, int R, bool MFMA_SUMS>
struct Attend {
  static constexpr int KW = D / 32;        // dwords of a key quarter; MFMAs per score block
  static constexpr int VW = D / 32;        // dwords of four tokens' group of values
  static constexpr int NE = D / 16;        // output blocks (elements of a group)
  static constexpr int kBlock = attn_block_bytes(D);
  // Weights are 2^(score - m) with m lagging behind the true maximum by at most kLag; in fp16 they are moved up to the end of the type's
  // range, so that a weight has all its bits down to 2^-25 of the largest.
  static constexpr float kLag = DT == ST_DT_BF16 ? 8.f : 5.f, kUp = DT == ST_DT_BF16 ? 0.f : 10.f;
  static constexpr uint32_t kOnes = DT == ST_DT_BF16 ? 0x3f803f80u : 0x3c003c00u;
  static constexpr float kNothing = -3.0e38f;
  typedef Mma<DT, 16> Op;

  u32x4 q[R][KW];
  f32x4 acc[NE][R];
  f32x4 sum[R];            // MFMA_SUMS: each of them the row's; else [0] is that of the lane's own weights
  float m[R];              // reference, less kUp; kNothing: the row has seen no token yet
  int pos[R];              // the lane's rows' tokens; a row that there is not has queries of 0 and is not stored

  struct Raw {
    uint32_t k[2][KW], v[2][VW], ks[2], vs[2];
    int bad;               // bit b: block b is on no page
  };
  struct Pages { int p[2]; };

  __device__ __forceinline__ float row_sum(int r) const { return MFMA_SUMS ? sum[r][0] : sum_of_row(sum[r][0]); }
  __device__ __forceinline__ void clear() {
    static_for<R>([&](auto J) {
      constexpr int r = decltype(J)::value;
      static_for<NE>([&](auto E) { acc[decltype(E)::value][r] = f32x4{0.f, 0.f, 0.f, 0.f}; });
      sum[r] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[r] = kNothing;
    });
  }
  // rows [row0, row0 + 16 R) of the sequence's new tokens x heads of a group: row = token * group + head
  __device__ __forceinline__ void load_rows(ConstAttn& T, const Seq& S, int head, int row0, int lane) {
    const int i = lane & 15, g = lane >> 4, rows = S.n * T.group;
    static_for<R>([&](auto J) {
      constexpr int r = decltype(J)::value;
      const int row = row0 + r * 16 + i, j = row / T.group, h = row - j * T.group;
      const bool real = row < rows;
      const uint16_t* p = (const uint16_t*)T.q + (int64_t)(S.first + (real ? j : 0)) * T.ldq + (int64_t)(head * T.group + (real ? h : 0)) * D + g * (D / 4);
      static_for<KW>([&](auto B) {
        constexpr int b = decltype(B)::value;
        q[r][b] = real ? *(const u32x4_any*)(p + 8 * b) ^ T.flip : u32x4{0u, 0u, 0u, 0u};
      });
      pos[r] = last_seen(T, S, j);
    });
  }
  // the page of both blocks of step s; a block behind `last` takes the first one's
  static __device__ __forceinline__ Pages look_up(ConstAttn& T, Table& table, int s, int last, int lane) {
    const int t = s * kAttnStep;
    const int a = table.page(T, t, lane);
    return {{a, t + 16 <= last ? table.page(T, t + 16, lane) : a}};
  }
  static __device__ __forceinline__ void fetch(ConstAttn& T, Raw& raw, int head, int s, int last, const Pages& pages, int lane) {
    const int i = lane & 15, g = lane >> 4;
    raw.bad = 0;
    static_for<2>([&](auto B) {
      constexpr int b = decltype(B)::value;
      const int t = s * kAttnStep + (b && s * kAttnStep + 16 <= last ? 16 : 0), page = pages.p[b];
      if (page < 0) raw.bad |= 1 << b;
      const char* at = block_of(T, page < 0 ? 0 : page, head, t, kBlock);
      const char *kp = at + (uint32_t)(i * (D / 2) + g * (D / 8)), *vp = at + (uint32_t)(8 * D + (i * 16 + 4 * g) * (D / 32));
      if constexpr (D == 64) {
        const u32x2 a = *(const u32x2*)kp, c = *(const u32x2*)vp;
        raw.k[b][0] = a[0], raw.k[b][1] = a[1], raw.v[b][0] = c[0], raw.v[b][1] = c[1];
      } else {
        static_for<D / 128>([&](auto W) {
          constexpr int w = decltype(W)::value;
          const u32x4 a = *(const u32x4*)(kp + 16 * w), c = *(const u32x4*)(vp + 16 * w);
          static_for<4>([&](auto X) { raw.k[b][4 * w + decltype(X)::value] = a[decltype(X)::value], raw.v[b][4 * w + decltype(X)::value] = c[decltype(X)::value]; });
        });
      }
      const char* ks = at + (uint32_t)(16 * D + i * (D / 32) + (D == 64 ? g / 2 : D == 128 ? g : 2 * g));
      if constexpr (D == 256) raw.ks[b] = *(const uint16_t*)ks;
      else raw.ks[b] = *(const uint8_t*)ks;
      raw.vs[b] = *(const uint32_t*)(at + (uint32_t)(16 * D + D / 2 + (D == 64 ? i / 8 : D == 128 ? i / 4 : i / 2) * 16 + 4 * g));
    });
  }

  // The weights of 32 tokens from t0 on, as operand B of the values' MFMAs, and their sums.  mask: some row does not see some of them; bit b
  // of bad: nobody sees block b.
  // Weights are rounded to the operands' type, 8 bits or 11, since that is what the MFMAs take (fp32 ones run at a sixteenth of the rate); their sum is
  // of the rounded ones, so that a row's weights add up to 1.  Against 64 bits outputs are off by 2.1e-3 to 2.3e-3 in bf16 and 2.8e-4 in fp16 (2-norms), where weights in fp32
  // and one rounding at the end give 1.7e-3 and 2.1e-4.
  __device__ __forceinline__ void weigh(f32x4 (&score)[2][R], u32x4 (&p)[R], int t0, bool mask, int bad, int window, float scale, int lane) {
    if (mask) {
      const int g = lane >> 4;
      static_for<R>([&](auto J) {
        constexpr int r = decltype(J)::value;
        static_for<8>([&](auto X) {
          constexpr int x = decltype(X)::value;
          const int t = t0 + (x / 4) * 16 + 4 * g + x % 4;
          // without a window (0, taken as 2^32 - 1) only t <= pos counts
          const bool seen = ((uint32_t)(pos[r] - t) <= (uint32_t)window - 1u) & (t <= pos[r]) & !((bad >> (x / 4)) & 1);
          score[x / 4][r][x % 4] = seen ? score[x / 4][r][x % 4] : -__builtin_inff();
        });
      });
    }
    // the scale is above zero: a row's largest score is its largest exponent
    float top[R], inf;
    asm("s_mov_b32 %0, 0x7f800000" : "=s"(inf));
    bool above = false;
    static_for<R>([&](auto J) {
      constexpr int r = decltype(J)::value;
      const f32x4 a = score[0][r], b = score[1][r];
      top[r] = max_raw(max_raw(max_raw(a[0], a[1], inf), max_raw(a[2], a[3], inf), inf), max_raw(max_raw(b[0], b[1], inf), max_raw(b[2], b[3], inf), inf), inf);
      above |= __builtin_fmaf(top[r], scale, -m[r]) > kLag + kUp;
    });
    if (__builtin_expect(__any(above) != 0, 0)) {
      static_for<R>([&](auto J) {
        constexpr int r = decltype(J)::value;
        const float next = fmaxf(m[r], max_of_row(top[r]) * scale - kUp), down = __builtin_amdgcn_exp2f(m[r] - next);
        m[r] = next;
        static_for<NE>([&](auto E) { acc[decltype(E)::value][r] *= down; });
        sum[r] *= down;
      });
    }
    static_for<R>([&](auto J) {
      constexpr int r = decltype(J)::value;
      static_for<4>([&](auto X) {
        constexpr int x = decltype(X)::value;
        auto weight = [&](int e) { return __builtin_amdgcn_exp2f(__builtin_fmaf(score[x / 2][r][e], scale, -m[r])); };
        p[r][x] = pack_pair<DT>(weight(x % 2 * 2), weight(x % 2 * 2 + 1));
      });
      if constexpr (MFMA_SUMS) sum[r] = Op::run(u32x4{kOnes, kOnes, kOnes, kOnes}, p[r], sum[r]);
      else static_for<4>([&](auto X) { sum[r][0] = add_pair<DT>(p[r][decltype(X)::value], sum[r][0]); });
    });
  }

  // Tokens [32 s, 32 s + 32).  mask: some row does not see some of them.
  __device__ __forceinline__ void step(const Raw& raw, int s, int length, int window, float scale, int lane, bool mask) {
    const int g = lane >> 4;
    f32x4 score[2][R];
    static_for<2>([&](auto B) {
      constexpr int b = decltype(B)::value;
      static_for<R>([&](auto J) { score[b][decltype(J)::value] = f32x4{0.f, 0.f, 0.f, 0.f}; });
      static_for<KW>([&](auto W) {
        constexpr int w = decltype(W)::value;
        const float sc = key_scale<DT>(D == 256 ? (w < KW / 2 ? raw.ks[b] & 255u : raw.ks[b] >> 8) : raw.ks[b]);
        const uint32_t c = raw.k[b][w];
        const u32x4 a = {widen<DT, 0>(c, sc), widen<DT, 1>(c, sc), widen<DT, 2>(c, sc), widen<DT, 3>(c, sc)};
        static_for<R>([&](auto J) { score[b][decltype(J)::value] = Op::run(a, q[decltype(J)::value][w], score[b][decltype(J)::value]); });
      });
    });
    u32x4 p[R];
    weigh(score, p, s * kAttnStep, mask, raw.bad, window, scale, lane);
    float vsc[8];
    static_for<8>([&](auto X) {
      constexpr int x = decltype(X)::value;
      vsc[x] = value_scale<DT>((raw.vs[x / 4] >> (8 * (x % 4))) & 255u);
    });
    if (mask) {                // what lies behind the sequence's end, or on no page, may be anything
      static_for<8>([&](auto X) {
        constexpr int x = decltype(X)::value;
        const int t = s * kAttnStep + (x / 4) * 16 + 4 * g + x % 4;
        vsc[x] = (t < length) & !((raw.bad >> (x / 4)) & 1) ? vsc[x] : 1.f;
      });
    }
    // two elements of the group at a time: byte e2 of a token's part of the group
    static_for<NE / 2>([&](auto E2) {
      constexpr int e2 = decltype(E2)::value;
      u32x4 a0, a1;
      static_for<4>([&](auto X) {          // token pairs
        constexpr int x = decltype(X)::value, b = x / 2, t0 = 2 * (x % 2);
        constexpr int at0 = t0 * (D / 32) + e2, at1 = (t0 + 1) * (D / 32) + e2;
        const uint32_t c0 = widen<DT, at0 % 4>(raw.v[b][at0 / 4], vsc[4 * b + t0]), c1 = widen<DT, at1 % 4>(raw.v[b][at1 / 4], vsc[4 * b + t0 + 1]);
        a0[x] = __builtin_amdgcn_perm(c1, c0, 0x05040100u);
        a1[x] = __builtin_amdgcn_perm(c1, c0, 0x07060302u);
      });
      static_for<R>([&](auto J) {
        constexpr int r = decltype(J)::value;
        acc[2 * e2][r] = Op::run(a0, p[r], acc[2 * e2][r]);
        acc[2 * e2 + 1][r] = Op::run(a1, p[r], acc[2 * e2 + 1][r]);
      });
    });
  }

  // Steps begin, begin + STRIDE, ... before end; `first`, `last`: the first and last tokens that any row sees; tokens [all_lo, all_hi] are seen by all rows.
  template <int STRIDE>
  __device__ __forceinline__ void run(ConstAttn& T, int seq, int head, int length, int begin, int end, int first, int last, int all_lo, int all_hi, int lane) {
    if (begin >= end) return;
    const float scale = T.scale;
    const int final_step = end - 1;
    auto held = [&](int s) { return s < final_step ? s : final_step; };      // what is fetched ahead stays inside
    int bad = 0;
    auto compute = [&](const Raw& raw, int s) __attribute__((always_inline)) {
      const int t = s * kAttnStep;
      bad |= t + 16 <= first ? raw.bad & 2 : raw.bad;      // a page before all windows may be gone
      step(raw, s, length, T.window, scale, lane, !(t >= all_lo && t + kAttnStep - 1 <= all_hi && raw.bad == 0));
    };
    Table table(T, seq, begin * kAttnStep, last, lane);
    Raw r0, r1;
    fetch(T, r0, head, begin, last, look_up(T, table, begin, last, lane), lane);
    Pages next = look_up(T, table, held(begin + STRIDE), last, lane);
    for (int s = begin; s < end; s += 2 * STRIDE) {
      fetch(T, r1, head, held(s + STRIDE), last, next, lane);
      next = look_up(T, table, held(s + 2 * STRIDE), last, lane);
      compute(r0, s);
      if (s + STRIDE >= end) break;
      fetch(T, r0, head, held(s + 2 * STRIDE), last, next, lane);
      next = look_up(T, table, held(s + 3 * STRIDE), last, lane);
      compute(r1, s + STRIDE);
    }
    if (bad && lane == 0) atomicOr(T.status, (uint32_t)ST_ATTN_BAD_PAGE);
  }
};

// A stretch's steps, of so many.  The division goes by what there is, not by what the table has room for.
__device__ __forceinline__ int tokens_chunk(int steps, ConstAttn& T) {
  if (steps <= T.whole) return steps > 0 ? steps : 1;
  // where the sequences alone fill the chip, stretches of one length, not halves: the short ones left over fill the gaps (64 of up to 8192: 67.6 us, 68.3)
  const int one = T.most < T.chunk ? T.most : T.chunk, want = T.want > 1 ? T.want : T.split, even = (steps + want - 1) / want;
  if (T.want == 1) return even > one ? even : one;
  const int chunk = even > T.least ? even : T.least;
  return chunk < T.chunk ? chunk : T.chunk;
}
template <int D>
__device__ __forceinline__ int rows_chunk(int steps, ConstAttn& T) {
  if (steps <= T.whole) return steps;
  const int best = (int)(__builtin_amdgcn_sqrtf((float)steps * T.root) + 0.5f), few = best < T.want ? best : T.want, room = best >= T.most ? T.most : few;
  const int level = steps / attn_level_steps(D) < T.least ? steps / attn_level_steps(D) : T.least, many = room > level ? room : level;
  const int parts = many < T.split ? many : T.split;
  return parts > 1 ? (steps + parts - 1) / parts : steps;
}

// The tokens that rows [row0, row1) of a sequence see: any of them, and all of them.
struct Seen { int lo, hi, all_lo, all_hi; };
__device__ __forceinline__ Seen seen_by(ConstAttn& T, const Seq& S, int row0, int row1) {
  const int j0 = row0 / T.group, j1 = (row1 - 1) / T.group, p0 = S.before + j0, p1 = S.before + j1;
  Seen s;
  s.hi = last_seen(T, S, j1);
  s.all_hi = last_seen(T, S, j0);
  s.lo = T.window && p0 - T.window + 1 > 0 ? p0 - T.window + 1 : 0;
  s.all_lo = T.window && p1 - T.window + 1 > 0 ? p1 - T.window + 1 : 0;
  if (T.n_pages == 0) {
    if (s.hi >= 0 && threadIdx.x == 0) atomicOr(T.status, (uint32_t)ST_ATTN_BAD_PAGE);
    s.hi = -1;
  }
  return s;
}

// One over a row's sum, and what the values' scales lack.
template <int DT>
__device__ __forceinline__ float inverse_of(float total) { return total == 0.f ? 0.f : (kHalved<DT> ? 2.f : 1.f) / total; }
// W of a row's outputs: sums of its values, `inverse` for all of them.
template <int DT, int W>
__device__ __forceinline__ void store_out(ConstAttn& T, const Seq& S, int head, int row, int dim, int D, const float* sums, float inverse) {
  const int j = row / T.group, h = row - j * T.group;
  uint16_t* p = (uint16_t*)T.out + (int64_t)(S.first + j) * T.ldo + (int64_t)(head * T.group + h) * D + dim;
  float v[W];
#pragma unroll
  for (int e = 0; e < W; ++e) v[e] = sums[e] * inverse;
  if constexpr (DT == ST_DT_F16) {      // of values that are 65536 in the cache; a row's outputs are all NaN or none is, by its sum, and a median with NaN alone is NaN
    const float most = inverse == inverse ? 65504.f : inverse;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = __builtin_amdgcn_fmed3f(v[e], -most, most);
  }
  if constexpr (W == 8) *(u32x4_any*)p = u32x4{pack_pair<DT>(v[0], v[1]), pack_pair<DT>(v[2], v[3]), pack_pair<DT>(v[4], v[5]), pack_pair<DT>(v[6], v[7])};
  else *(u32x2_any*)p = u32x2{pack_pair<DT>(v[0], v[1]), pack_pair<DT>(v[2], v[3])};
}

// ---- each wavefront its own rows ----------------------------------------------------------------------------------------
// The wavefronts of a workgroup go through the same tokens, TT at a time.  Each of them widens a block of the next tile (or half of one)
// into LDS, in operand order (fragment f, lane l at 16 bytes (64 f + l)), while all compute on the present one: two buffers, one barrier a
// tile.  A wavefront issues a vector instruction every five to six clocks at best and its MFMAs take sixteen each, so the widening is cut
// into pieces that are issued between MFMAs.  Fewer tokens to a tile cost more: the look-ups and addresses are a tile's (heads of 256, chunks of
// 333 in windows, with 32 97.5 us, with 64 82.0).
//
// SPLIT: few rows over many tokens, which are divided into stretches.  A stretch's sums lie in memory as they lie in the lanes, and whoever
// arrives last adds them up in order.
template <int DT, int D, int R, bool SPLIT>
__global__ __launch_bounds__(attn_row_waves(D) * 64, 2) void st_attn_rows_kernel(const AttnDev* table, const AttnItem* items) {
  typedef Attend<DT, D, R, true> A;
  constexpr int W = attn_row_waves(D), TT = kAttnRowTokens, BLOCKS = TT / 16, KW = A::KW, NE = A::NE;
  constexpr int SHARE = W / BLOCKS;                                     // wavefronts to a block
  constexpr int KWAVE = KW / SHARE, VWAVE = NE / SHARE;                 // fragments that a wavefront makes of its block's keys and values
  constexpr int KF = BLOCKS * KW, VF = TT / 32 * NE;                    // fragments of a tile
  static_assert(W % BLOCKS == 0 && (D == 256 ? SHARE == 2 : SHARE == 1) && (KWAVE == 2 || KWAVE == 4), "a part is whole fragments, and lies in one word of a token's codes");
  __shared__ __align__(16) u32x4 frags[2][KF + VF][64];
  __shared__ __align__(16) int hidden[2][BLOCKS];
  const ConstAttnItem& ci = ((ConstAttnItem*)items)[blockIdx.x];
  ConstAttn& T = ((ConstAttn*)table)[ci.tenant];
  constexpr int ROWS = W * 16 * R;
  const int group = T.group, split = SPLIT ? T.split : 1, item = SPLIT ? (int)ci.part / split : (int)ci.part, stretch = SPLIT ? (int)ci.part - item * split : 0;
  int seq, part_of = item;
  if (!find_sequence(T, ci.seq, seq, part_of, [group](int n) { return (n * group + ROWS - 1) / ROWS; })) return;
  const int head = (int)ci.head;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  const Seq S = sequence(T, seq, threadIdx.x == 0);
  const int rows = S.n * group, block0 = (ci.seq == kAttnFind ? (rows - 1) / ROWS - part_of : part_of) * ROWS, row0 = block0 + wave * 16 * R;
  if (block0 >= rows || block0 < 0) return;
  const int block1 = block0 + ROWS < rows ? block0 + ROWS : rows;
  const int row1 = row0 + 16 * R < rows ? row0 + 16 * R : rows;
  const Seen all = seen_by(T, S, block0, block1);
  Seen see = seen_by(T, S, row0 < rows ? row0 : block0, row0 < rows ? row1 : block1);
  if (row0 >= rows) see.hi = -1;                                         // helps widening, has nothing to compute
  int n0 = all.lo / TT, n1 = all.hi >= all.lo ? all.hi / TT + 1 : n0, active = 1;
  if constexpr (SPLIT) {      // stretches as long as those of the sequence's last rows, so that all take about as long
    const int most = T.window && T.window + ROWS < S.length ? T.window + ROWS : S.length;
    const int chunk = rows_chunk<D>((most + TT - 1) / TT + 1, T);
    active = n1 - n0 > chunk ? (n1 - n0 + chunk - 1) / chunk : 1;
    if (stretch >= active) return;
    if (active > 1) {
      n0 += stretch * chunk;
      n1 = stretch + 1 < active ? n0 + chunk : n1;
    }
  }
  A a;
  a.clear();
  a.load_rows(T, S, head, row0, lane);
  const int kb = wave / SHARE, part = wave % SHARE;                     // the wavefront's block of a tile, and its part of it

  struct Raw { uint32_t k[KWAVE], v[4], ks, vs; int page; };            // the part as it lies in the cache; v: a word per token (D = 64: per two)
  Raw raw;
  Table pages_of(T, seq, n0 < n1 ? n0 * TT : 0, n0 < n1 ? all.hi : 0, lane);
  const uint32_t k_at = (uint32_t)(i * (D / 2) + g * (D / 8) + part * KWAVE * 4), v_at = (uint32_t)(8 * D + (i * 16 + 4 * g) * (D / 32) + part * 4);
  const uint32_t ks_at = (uint32_t)(16 * D + i * (D / 32) + (D == 64 ? g / 2 : D == 128 ? g : 2 * g + part));
  const uint32_t vs_at = (uint32_t)(16 * D + D / 2 + (D == 64 ? i / 8 : D == 128 ? i / 4 : i / 2) * 16 + 4 * g);
  auto look_up = [&](int n) __attribute__((always_inline)) {
    const int t = n * TT + kb * 16;
    return t <= all.hi ? pages_of.page(T, t, lane) : -1;
  };
  auto fetch = [&](int n, int page) __attribute__((always_inline)) {
    const int t = n * TT + kb * 16;
    raw.page = page;
    const char* at = block_of(T, raw.page < 0 ? 0 : raw.page, head, t, A::kBlock);
    if constexpr (KWAVE == 2) {
      const u32x2 w = *(const u32x2*)(at + k_at);
      raw.k[0] = w[0], raw.k[1] = w[1];
    } else {
      const u32x4 w = *(const u32x4*)(at + k_at);
      static_for<4>([&](auto X) { raw.k[decltype(X)::value] = w[decltype(X)::value]; });
    }
    if constexpr (D == 64) {
      const u32x2 c = *(const u32x2*)(at + v_at);
      raw.v[0] = c[0], raw.v[1] = c[1];
    } else if constexpr (D == 128) {
      const u32x4 c = *(const u32x4*)(at + v_at);
      static_for<4>([&](auto X) { raw.v[decltype(X)::value] = c[decltype(X)::value]; });
    } else {
      static_for<4>([&](auto X) { raw.v[decltype(X)::value] = *(const uint32_t*)(at + v_at + 8 * decltype(X)::value); });
    }
    raw.ks = *(const uint8_t*)(at + ks_at);
    raw.vs = *(const uint32_t*)(at + vs_at);
  };
  // the pieces of making tile n in buffer buf from what was fetched, and of fetching tile n + 1 (held inside the range) after it
  constexpr int PIECES = 2 + KWAVE + VWAVE / 2;
  float ksc, vsc[4];
  int next_page = -1;
  auto piece = [&](auto P, int n, int buf) __attribute__((always_inline)) {
    constexpr int p = decltype(P)::value;
    if constexpr (p == 0) {
      ksc = key_scale<DT>(raw.ks);
      static_for<4>([&](auto X) { vsc[decltype(X)::value] = value_scale<DT>((raw.vs >> (8 * decltype(X)::value)) & 255u); });
      // what lies behind the sequence's end, or on no page, may be anything: it takes a scale of 1
      const int real = raw.page < 0 ? 0 : S.length - (n * TT + kb * 16 + 4 * g);
      static_for<4>([&](auto X) { vsc[decltype(X)::value] = decltype(X)::value < real ? vsc[decltype(X)::value] : 1.f; });
      hidden[buf][kb] = raw.page < 0;
    } else if constexpr (p <= KWAVE) {
      constexpr int f = p - 1;
      const uint32_t c = raw.k[f];
      frags[buf][kb * KW + part * KWAVE + f][lane] = u32x4{widen<DT, 0>(c, ksc), widen<DT, 1>(c, ksc), widen<DT, 2>(c, ksc), widen<DT, 3>(c, ksc)};
    } else if constexpr (p <= KWAVE + VWAVE / 2) {
      constexpr int e2 = p - 1 - KWAVE;             // elements 2 e2, 2 e2 + 1 of the part's groups, for the lane's four tokens
      uint32_t c[4];
      static_for<4>([&](auto X) {
        constexpr int t = decltype(X)::value;
        if constexpr (D == 64) c[t] = widen<DT, t % 2 * 2 + e2>(raw.v[t / 2], vsc[t]);
        else c[t] = widen<DT, e2>(raw.v[t], vsc[t]);
      });
      u32x2* to = (u32x2*)&frags[buf][KF + kb / 2 * NE + part * VWAVE + 2 * e2][lane] + kb % 2;
      to[0] = u32x2{__builtin_amdgcn_perm(c[1], c[0], 0x05040100u), __builtin_amdgcn_perm(c[3], c[2], 0x05040100u)};
      to[128] = u32x2{__builtin_amdgcn_perm(c[1], c[0], 0x07060302u), __builtin_amdgcn_perm(c[3], c[2], 0x07060302u)};
    } else {
      fetch(n + 1 < n1 ? n + 1 : n1 - 1, next_page);
    }
  };
  const float scale = T.scale;
  // A tile's sub-steps read their fragments in order, keys then values, AHEAD of them before they are multiplied.
  constexpr int AHEAD = D == 256 ? 8 : 4, SF = 2 * KW + NE, EVERY = 2;
  auto compute = [&](int n, int buf, int bad) __attribute__((always_inline)) {
    auto slot = [&](auto N) __attribute__((always_inline)) {
      constexpr int k = decltype(N)::value;
      if constexpr (k % EVERY == EVERY - 1 && k / EVERY < PIECES) piece(std::integral_constant<int, k / EVERY>{}, n + 1, buf ^ 1);
      __builtin_amdgcn_sched_barrier(0);
    };
    static_for<TT / 32>([&](auto U) __attribute__((always_inline)) {
      constexpr int u = decltype(U)::value;
      const int t0 = n * TT + 32 * u, hid = bad >> (2 * u) & 3;
      const bool mask = !(t0 >= see.all_lo && t0 + 31 <= see.all_hi && hid == 0);
      u32x4 f[AHEAD];
      auto read = [&](auto F) __attribute__((always_inline)) {
        constexpr int k = decltype(F)::value;
        if constexpr (k < SF) f[k % AHEAD] = frags[buf][k < 2 * KW ? 2 * u * KW + (R > 1 ? k : k % 2 * KW + k / 2) : KF + u * NE + k - 2 * KW][lane];
      };
      static_for<AHEAD>([&](auto F) { read(F); });
      f32x4 score[2][R];
      static_for<2 * R>([&](auto J) { score[decltype(J)::value / R][decltype(J)::value % R] = f32x4{0.f, 0.f, 0.f, 0.f}; });
      static_for<2 * KW>([&](auto Q) __attribute__((always_inline)) {
        // block after block, or, where a block's MFMAs would wait for one another, both in turn
        constexpr int k = decltype(Q)::value, b = R > 1 ? k / KW : k % 2, w = R > 1 ? k % KW : k / 2;
        static_for<R>([&](auto J) { score[b][decltype(J)::value] = A::Op::run(f[k % AHEAD], a.q[decltype(J)::value][w], score[b][decltype(J)::value]); });
        read(std::integral_constant<int, k + AHEAD>{});
        slot(std::integral_constant<int, u * SF + k>{});
      });
      u32x4 p[R];
      a.weigh(score, p, t0, mask, hid, T.window, scale, lane);
      static_for<NE>([&](auto E) __attribute__((always_inline)) {
        constexpr int e = decltype(E)::value, k = 2 * KW + e;
        static_for<R>([&](auto J) { a.acc[e][decltype(J)::value] = A::Op::run(f[k % AHEAD], p[decltype(J)::value], a.acc[e][decltype(J)::value]); });
        read(std::integral_constant<int, k + AHEAD>{});
        slot(std::integral_constant<int, u * SF + k>{});
      });
    });
  };
  int bad_pages = 0;
  if (n0 < n1) {
    fetch(n0, look_up(n0));
    next_page = look_up(n0 + 1 < n1 ? n0 + 1 : n1 - 1);
    static_for<PIECES>([&](auto P) { piece(P, n0, 0); });
    __syncthreads();
    for (int n = n0; n < n1; ++n) {
      const int buf = (n - n0) & 1;
      next_page = look_up(n + 2 < n1 ? n + 2 : n1 - 1);
      int bad = 0;
      static_for<BLOCKS>([&](auto B) { bad |= hidden[buf][decltype(B)::value] << decltype(B)::value; });
      bad = __builtin_amdgcn_readfirstlane(bad);
      // of blocks from the first token to the last that somebody sees: pages before all windows may be gone
      const int from = all.lo - n * TT > 0 ? (all.lo - n * TT) / 16 : 0, to = (all.hi - n * TT) / 16 < BLOCKS ? (all.hi - n * TT) / 16 : BLOCKS - 1;
      bad_pages |= bad & ((2 << to) - (1 << from));
      compute(n, buf, bad);      // also where the wavefront's rows see none of it, a few tiles at a sequence's ends: one path keeps the sums in place
      __syncthreads();
    }
  }
  if (bad_pages && lane == 0) atomicOr(T.status, (uint32_t)ST_ATTN_BAD_PAGE);
  if constexpr (SPLIT) {
    if (active > 1) {
      __shared__ uint32_t flag;
      constexpr int THREADS = W * 64, kVectors = NE * R, kSlot = attn_row_slot(kAttnRows, D) * 4;
      const int tid = (int)threadIdx.x;
      const int64_t tile = ci.seq == kAttnFind ? (int64_t)item * T.kv_heads + head : ((int64_t)seq * T.kv_heads + head) * T.row_tiles + item;
      float* slots = T.ws + tile * split * (kSlot / 4);
      const __amdgpu_buffer_rsrc_t rs = make_rsrc(slots + (int64_t)stretch * (kSlot / 4), kSlot);
      static_for<kVectors>([&](auto Q) {
        constexpr int q = decltype(Q)::value;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, a.acc[q / R][q % R]), rs, tid * 16 + q * THREADS * 16, 0, kAuxDeviceCoherent);
      });
      static_for<R>([&](auto J) {
        constexpr int r = decltype(J)::value;
        const u32x2 stat = {__builtin_bit_cast(uint32_t, a.m[r]), __builtin_bit_cast(uint32_t, a.sum[r][0])};
        __builtin_amdgcn_raw_buffer_store_b64(stat, rs, tid * 8 + kVectors * THREADS * 16 + r * THREADS * 8, 0, kAuxDeviceCoherent);
      });
      __builtin_amdgcn_s_waitcnt(0);      // this thread's stores have been written through
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();
      if (tid == 0) {
        const uint32_t old = __hip_atomic_fetch_add(&T.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t is_last = old == (uint32_t)(active - 1);
        if (is_last) __hip_atomic_store(&T.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        flag = is_last;
      }
      __syncthreads();
      if (flag == 0u) return;
      auto stat_of = [&](int s, int r) __attribute__((always_inline)) {
        return __builtin_amdgcn_raw_buffer_load_b64(make_rsrc(slots + (int64_t)s * (kSlot / 4), kSlot), tid * 8 + kVectors * THREADS * 16 + r * THREADS * 8, 0, kAuxDeviceCoherent);
      };
      a.clear();
      for (int s = 0; s < active; ++s)
        static_for<R>([&](auto J) { a.m[decltype(J)::value] = fmaxf(a.m[decltype(J)::value], __builtin_bit_cast(float, stat_of(s, decltype(J)::value)[0])); });
      for (int s = 0; s < active; ++s) {
        const __amdgpu_buffer_rsrc_t from = make_rsrc(slots + (int64_t)s * (kSlot / 4), kSlot);
        float w[R];
        static_for<R>([&](auto J) {
          constexpr int r = decltype(J)::value;
          const u32x2 stat = stat_of(s, r);
          w[r] = __builtin_amdgcn_exp2f(__builtin_bit_cast(float, (uint32_t)stat[0]) - a.m[r]);
          a.sum[r][0] += w[r] * __builtin_bit_cast(float, (uint32_t)stat[1]);
        });
        static_for<kVectors>([&](auto Q) {
          constexpr int q = decltype(Q)::value;
          a.acc[q / R][q % R] += w[q % R] * __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, tid * 16 + q * THREADS * 16, 0, kAuxDeviceCoherent));
        });
      }
    }
  }
  static_for<R>([&](auto J) {
    constexpr int r = decltype(J)::value;
    const int row = row0 + r * 16 + i;
    const float inv = inverse_of<DT>(a.row_sum(r));
    if (row < rows) {
      static_for<4>([&](auto X) {
        constexpr int x = decltype(X)::value;
        float v[D / 16];
        static_for<D / 16>([&](auto E) { v[decltype(E)::value] = a.acc[decltype(E)::value][r][x]; });
        const int dim = (4 * g + x) * (D / 16);
        if constexpr (D == 64) store_out<DT, 4>(T, S, head, row, dim, D, v, inv);
        else static_for<D / 128>([&](auto C) { store_out<DT, 8>(T, S, head, row, dim + 8 * decltype(C)::value, D, v + 8 * decltype(C)::value, inv); });
      });
    }
  });
}

// ---- a workgroup's wavefronts take turns over a stretch of tokens -------------------------------------------------------
// The wavefronts' results meet in LDS; where a sequence has several stretches their results meet in memory, and the last workgroup to
// arrive joins them in order.
template <int DT, int D, int R>
__global__ __launch_bounds__(kAttnTokenWaves * 64, D <= 128 && R == 1 ? 4 : 2) void st_attn_tokens_kernel(const AttnDev* table, const AttnItem* items) {
  constexpr int W = kAttnTokenWaves, THREADS = W * 64, ROWS = 16 * R;
  constexpr int DP = D < 128 ? D : 128, PASS = D / DP, EP = DP / 16, kPitch = DP + 4;       // dims per pass
  __shared__ __align__(16) float part[W][16][kPitch];
  __shared__ float wave_m[W][ROWS], wave_l[W][ROWS], weight[kAttnMaxSplit][ROWS], inverse[ROWS];
  __shared__ uint32_t flag;
  const ConstAttnItem& ci = ((ConstAttnItem*)items)[blockIdx.x];
  ConstAttn& T = ((ConstAttn*)table)[ci.tenant];
  const int seq = (int)ci.seq, head = (int)ci.head, row_tile = (int)ci.part / T.split, stretch = (int)ci.part - row_tile * T.split;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const Seq S = sequence(T, seq, tid == 0);
  const int rows = S.n * T.group, row0 = row_tile * ROWS;
  if (row0 >= rows) return;
  const int row1 = row0 + ROWS < rows ? row0 + ROWS : rows;
  const Seen see = seen_by(T, S, row0, row1);
  const int s_lo = see.lo / kAttnStep, steps = see.hi >= see.lo ? see.hi / kAttnStep + 1 - s_lo : 0;
  const int chunk = tokens_chunk(steps, T), active = steps > chunk ? (steps + chunk - 1) / chunk : 1;      // stretches that there are
  if (stretch >= active) return;
  const int begin = s_lo + stretch * chunk, end = stretch + 1 < active ? begin + chunk : s_lo + steps;

  Attend<DT, D, R, false> a;
  a.clear();
  a.load_rows(T, S, head, row0, lane);
  a.template run<W>(T, seq, head, S.length, begin + wave, end, see.lo, see.hi, see.all_lo, see.all_hi, lane);

  // all wavefronts' sums to one reference
  static_for<R>([&](auto J) {
    constexpr int r = decltype(J)::value;
    if (g == 0) wave_m[wave][r * 16 + i] = a.m[r];
  });
  __syncthreads();
  float ref[R];
  static_for<R>([&](auto J) {
    constexpr int r = decltype(J)::value;
    float top = a.m[r];
    for (int w = 0; w < W; ++w) top = fmaxf(top, wave_m[w][r * 16 + i]);
    ref[r] = top;
    const float down = __builtin_amdgcn_exp2f(a.m[r] - top);
    static_for<D / 16>([&](auto E) { a.acc[decltype(E)::value][r] *= down; });
    const float mine = a.row_sum(r) * down;
    if (g == 0) wave_l[wave][r * 16 + i] = mine;
  });
  __syncthreads();
  if (tid < ROWS) {
    float total = 0.f;
    for (int w = 0; w < W; ++w) total += wave_l[w][tid];
    wave_l[0][tid] = total;
    inverse[tid] = inverse_of<DT>(total);
  }
  const int64_t tile = ((int64_t)seq * T.kv_heads + head) * T.row_tiles + row_tile;
  const int64_t slots = (int64_t)T.n_seqs * T.kv_heads * T.row_tiles * T.split;
  float* parts = T.ws + tile * T.split * (ROWS * D);
  float* stats = T.ws + slots * (ROWS * D) + tile * T.split * (2 * ROWS);
  __syncthreads();
  static_for<R * PASS>([&](auto RP) {
    constexpr int r = decltype(RP)::value / PASS, pass = decltype(RP)::value % PASS;
    static_for<4>([&](auto X) {
      constexpr int x = decltype(X)::value;
      static_for<EP / 4>([&](auto C) {
        constexpr int c = decltype(C)::value, e = pass * EP + 4 * c;
        *(f32x4*)&part[wave][i][(4 * g + x) * EP + 4 * c] = f32x4{a.acc[e][r][x], a.acc[e + 1][r][x], a.acc[e + 2][r][x], a.acc[e + 3][r][x]};
      });
    });
    __syncthreads();
    for (int at = tid; at < 16 * DP / 4; at += THREADS) {
      const int row16 = at / (DP / 4), c = at % (DP / 4) * 4, row = r * 16 + row16;
      f32x4 v = *(const f32x4*)&part[0][row16][c];
#pragma unroll
      for (int w = 1; w < W; ++w) v += *(const f32x4*)&part[w][row16][c];
      const int dim = c / EP * (D / 16) + pass * EP + c % EP;
      if (row0 + row < row1) {
        if (active == 1) {
          const float o[4] = {v[0], v[1], v[2], v[3]};
          store_out<DT, 4>(T, S, head, row0 + row, dim, D, o, inverse[row]);
        } else {
          const __amdgpu_buffer_rsrc_t rs = make_rsrc(parts + (int64_t)stretch * (ROWS * D), ROWS * D * 4);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, (row * D + dim) * 4, 0, kAuxDeviceCoherent);
        }
      }
    }
    __syncthreads();
  });
  if (active == 1) return;
  const __amdgpu_buffer_rsrc_t rstat = make_rsrc(stats, (uint32_t)T.split * 2 * ROWS * 4);
  if (wave == 0) {
    static_for<R>([&](auto J) {
      constexpr int r = decltype(J)::value;
      if (g == 0) {
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, ref[r]), rstat, (stretch * 2 * ROWS + r * 16 + i) * 4, 0, kAuxDeviceCoherent);
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, wave_l[0][r * 16 + i]), rstat, (stretch * 2 * ROWS + ROWS + r * 16 + i) * 4, 0, kAuxDeviceCoherent);
      }
    });
  }
  __builtin_amdgcn_s_waitcnt(0);      // this thread's stores have been written through
  __syncthreads();
  if (tid == 0) {
    const uint32_t old = __hip_atomic_fetch_add(&T.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t is_last = old == (uint32_t)(active - 1);
    if (is_last) __hip_atomic_store(&T.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    flag = is_last;
  }
  __syncthreads();
  if (flag == 0u) return;
  // every stretch's maximum and sum of every row, all on their way at once
  static_assert(sizeof(part) >= kAttnMaxSplit * ROWS * 4 && sizeof(part) >= THREADS * 16, "room for the sums, then for the groups' results");
  float* sums = &part[0][0][0];
  for (int at = tid; at < active * ROWS; at += THREADS) {
    const int s = at / ROWS, row = at % ROWS;
    weight[s][row] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rstat, (s * 2 * ROWS + row) * 4, 0, kAuxDeviceCoherent));
    sums[at] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rstat, (s * 2 * ROWS + ROWS + row) * 4, 0, kAuxDeviceCoherent));
  }
  __syncthreads();
  if (tid < ROWS) {
    float top = Attend<DT, D, R, false>::kNothing, total = 0.f;
    for (int s = 0; s < active; ++s) top = fmaxf(top, weight[s][tid]);
    for (int s = 0; s < active; ++s) {
      const float w = __builtin_amdgcn_exp2f(weight[s][tid] - top);
      weight[s][tid] = w;
      total += w * sums[s * ROWS + tid];
    }
    inverse[tid] = inverse_of<DT>(total);
  }
  __syncthreads();
  // Four outputs to a thread.  Where that leaves threads over, they share the stretches: group k takes stretches k, k + groups, ...
  const __amdgpu_buffer_rsrc_t rp = make_rsrc(parts, (uint32_t)T.split * ROWS * D * 4);
  const int vectors = (row1 - row0) * (D / 4), groups = vectors < THREADS ? THREADS / vectors : 1, group = groups > 1 ? tid / vectors : 0;
  for (int first = 0; first < vectors; first += THREADS) {
    const int at = first + (groups > 1 ? tid - group * vectors : tid), row = at / (D / 4), dim = at % (D / 4) * 4;
    const bool mine = at < vectors && group < groups;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
      for (int s0 = group; s0 < active; s0 += 8 * groups) {
        f32x4 one[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int s = s0 + k * groups;
          one[k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rp, (int)(s < active ? (uint32_t)((s * ROWS + row) * D + dim) * 4u : kInvalidOffset), 0, kAuxDeviceCoherent));
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (s0 + k * groups < active) v += one[k] * weight[s0 + k * groups][row];
      }
    }
    if (groups > 1) {
      f32x4* shared = (f32x4*)&part[0][0][0];
      if (mine) shared[tid] = v;
      __syncthreads();
      if (tid < vectors)
        for (int k = 1; k < groups; ++k) v += shared[k * vectors + tid];
    }
    if (mine && group == 0) {
      const float o[4] = {v[0], v[1], v[2], v[3]};
      store_out<DT, 4>(T, S, head, row0 + row, dim, D, o, inverse[row]);
    }
  }
}

// ---- into the cache and out of it ---------------------------------------------------------------------------------------
// dim / 8 lanes to a token's head: each has eight elements of the key and of the value.  A wavefront's instructions are what a prompt costs
// (13 000 tokens of eight heads of 128, 68 MB, in 23 us with 430 of them for each 2 KB; 18.3 now), so a workgroup takes kAttnMoveTurns
// stretches of them, 16 tokens of a head side by side, and looks at values as integers: of a type's absolute values the larger one has the larger bits.
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t in_quad(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true); }
// Eight elements' codes and their group's scale; finite: all of the group's are.
template <int DT>
__device__ __forceinline__ void encode8(const u32x4 in, uint32_t& codes, uint32_t& scale, bool& finite) {
  const uint32_t all = 0x7fff7fffu;
  uint32_t m = max16(max16(in[0] & all, in[1] & all), max16(in[2] & all, in[3] & all));
  m = max16(m, m >> 16) & 0xffffu;
  m = max16(m, in_quad<0xB1>(m));      // four lanes to a group of 32
  m = max16(m, in_quad<0x4E>(m));
  finite = m < (DT == ST_DT_BF16 ? 0x7f80u : 0x7c00u);
  const uint32_t bits = __builtin_bit_cast(uint32_t, unpack16<DT>(m, 0));
  int e = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x400000u ? 1 : 0);
  e = e < 1 ? 1 : e > 252 ? 252 : e;
  scale = (uint32_t)e;
  const float f = __builtin_bit_cast(float, scale << 23);
  uint32_t c = 0;
  static_for<4>([&](auto X) {
    constexpr int x = decltype(X)::value;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, unpack16<DT>(in[x], 0), unpack16<DT>(in[x], 1), f, x);
  });
  codes = c;
}

// Of a pair of fp16 values, the infinite ones as the largest number of their sign.
__device__ __forceinline__ uint32_t finite_pair(uint32_t p) { return p - ((p & 0x7fffu) == 0x7c00u ? 1u : 0u) - ((p & 0x7fff0000u) == 0x7c000000u ? 0x10000u : 0u); }

template <int DT, int D, bool READ, int TURNS>
__global__ __launch_bounds__(256) void st_attn_move_kernel(const AttnDev* table, const AttnItem* items) {
  constexpr int LPT = D / 8, TH = attn_move_count(D), kBlock = attn_block_bytes(D);
  const ConstAttnItem& ci = ((ConstAttnItem*)items)[blockIdx.x];
  ConstAttn& T = ((ConstAttn*)table)[ci.tenant];
  const int tid = (int)threadIdx.x, lane = tid & 63, c = tid % LPT, slot = tid / LPT, kv = T.kv_heads, shift = T.page_shift;
  int seq = (int)ci.seq, part = (int)ci.part;
  if constexpr (TURNS > 1) {
    if (!find_sequence(T, ci.seq, seq, part, [kv](int n) { return (int)(((int64_t)(n + 15) / 16 * 16 * kv + TURNS * TH - 1) / (TURNS * TH)); })) return;
  }
  const Seq S = sequence(T, seq, tid == 0);
  const int32_t* row_of_table = T.table + (int64_t)seq * T.table_pages;
  int j[TURNS], head[TURNS], page[TURNS];
  u32x4 k[TURNS], v[TURNS];
  static_for<TURNS>([&](auto N) {
    constexpr int n = decltype(N)::value;
    const int th = (part * TURNS + n) * TH + slot;
    if constexpr (TURNS > 1) {            // 16 tokens of a head, then those of the next: a wavefront has tokens of one head
      const int group = __builtin_amdgcn_readfirstlane(th / 16);
      head[n] = group % kv;
      j[n] = group / kv * 16 + th % 16;
    } else {
      j[n] = th / kv;
      head[n] = th - j[n] * kv;
    }
    const bool real = j[n] < S.n;
    const int pos = S.before + j[n];
    page[n] = real && pos >= 0 ? row_of_table[pos >> shift] : -1;
    k[n] = v[n] = u32x4{0u, 0u, 0u, 0u};
    if (!READ && real) {
      const int64_t row = S.first + j[n];
      k[n] = *(const u32x4_any*)((const uint16_t*)T.k + row * T.ldk + head[n] * D + c * 8);
      v[n] = *(const u32x4_any*)((const uint16_t*)T.v + row * T.ldv + head[n] * D + c * 8);
    }
  });
  static_for<TURNS>([&](auto N) {
    constexpr int n = decltype(N)::value;
    const bool real = j[n] < S.n;
    const int pos = S.before + j[n], t = pos & 15;
    if (real && pos >= 0 && (uint32_t)page[n] >= (uint32_t)T.n_pages) {
      page[n] = -1;
      if (c == 0) atomicOr(T.status, (uint32_t)ST_ATTN_BAD_PAGE);
    }
    char* at = const_cast<char*>(block_of(T, page[n] < 0 ? 0 : page[n], head[n], pos, kBlock));
    char *kp = at + t * (D / 2) + c * 4, *ks = at + 16 * D + t * (D / 32) + c / 4, *vs = at + 16 * D + D / 2 + (c / 4) * 16 + t;
    char* vp = at + 8 * D + (D == 64 ? (2 * c * 16 + t) * 2 : D == 128 ? (c * 16 + t) * 4 : (c / 2 * 16 + t) * 8 + c % 2 * 4);
    if constexpr (!READ) {
      uint32_t kc, kscale, vc, vscale;
      bool kfin, vfin;
      encode8<DT>(k[n], kc, kscale, kfin);
      encode8<DT>(v[n], vc, vscale, vfin);
      const uint64_t odd = __ballot(!(kfin && vfin));
      if (odd != 0 && ((odd >> (lane & ~(LPT - 1))) & (((uint64_t)1 << LPT) - 1)) != 0) kc = vc = 0u, kscale = 255u, vscale = 1u;
      if (page[n] >= 0) {
        *(uint32_t*)kp = kc;
        if constexpr (D == 64) {
          *(uint16_t*)vp = (uint16_t)vc;
          *(uint16_t*)(vp + 32) = (uint16_t)(vc >> 16);
        } else {
          *(uint32_t*)vp = vc;
        }
        if (c % 4 == 0) {
          *ks = (char)kscale;
          *vs = (char)vscale;
        }
      }
    } else if (real) {
      if (page[n] >= 0) {
        const uint32_t kc = *(const uint32_t*)kp;
        uint32_t vc;
        if constexpr (D == 64) vc = *(const uint16_t*)vp | (uint32_t)*(const uint16_t*)(vp + 32) << 16;
        else vc = *(const uint32_t*)vp;
        // whole scales here, the largest one that is written at most; fp16: what is infinite under them is the largest number
        const uint32_t kb = *(const uint8_t*)ks, vb = *(const uint8_t*)vs, most = 252u;
        const float kf = __builtin_bit_cast(float, kb == 255u ? 0x7fc00000u : (kb < most ? kb : most) << 23), vf = __builtin_bit_cast(float, (vb < most ? vb : most) << 23);
        k[n] = u32x4{widen<DT, 0>(kc, kf), widen<DT, 1>(kc, kf), widen<DT, 2>(kc, kf), widen<DT, 3>(kc, kf)};
        v[n] = u32x4{widen<DT, 0>(vc, vf), widen<DT, 1>(vc, vf), widen<DT, 2>(vc, vf), widen<DT, 3>(vc, vf)};
        if (DT == ST_DT_F16 && __builtin_expect(__any((kb > vb ? kb : vb) > 140u) != 0, 0)) {
          static_for<4>([&](auto X) {
            constexpr int x = decltype(X)::value;
            k[n][x] = finite_pair(k[n][x]);
            v[n][x] = finite_pair(v[n][x]);
          });
        }
      }
      const int64_t row = S.first + j[n];
      *(u32x4_any*)((uint16_t*)T.k_out + row * T.ldk + head[n] * D + c * 8) = k[n];
      *(u32x4_any*)((uint16_t*)T.v_out + row * T.ldv + head[n] * D + c * 8) = v[n];
    }
  });
}

// ---- launches -------------------------------------------------------------------------------------------------------------
template <int DT, int D>
static hipError_t launch_kind(int kind, unsigned blocks, void* stream, const AttnDev* table, const AttnItem* items) {
  switch (kind) {
    case kAttnTokens1: return launch(st_attn_tokens_kernel<DT, D, attn_blocks(kAttnTokens1, D)>, blocks, kAttnTokenWaves * 64, stream, table, items);
    case kAttnTokens2: return launch(st_attn_tokens_kernel<DT, D, attn_blocks(kAttnTokens2, D)>, blocks, kAttnTokenWaves * 64, stream, table, items);
    case kAttnRows: return launch(st_attn_rows_kernel<DT, D, attn_blocks(kAttnRows, D), false>, blocks, attn_row_waves(D) * 64, stream, table, items);
    case kAttnRowsSplit: return launch(st_attn_rows_kernel<DT, D, attn_blocks(kAttnRows, D), true>, blocks, attn_row_waves(D) * 64, stream, table, items);
  }
  return hipErrorInvalidValue;
}
template <int DT>
static hipError_t launch_dim(int dim, int kind, unsigned blocks, void* stream, const AttnDev* table, const AttnItem* items) {
  return dim == 64 ? launch_kind<DT, 64>(kind, blocks, stream, table, items) : dim == 128 ? launch_kind<DT, 128>(kind, blocks, stream, table, items)
                                                                                          : launch_kind<DT, 256>(kind, blocks, stream, table, items);
}
int launch_attn(int dtype, int dim, int kind, const AttnDev* table_dev, const AttnItem* items_dev, int64_t n_items, void* stream) {
  if (n_items <= 0) return 0;
  return (int)(dtype == ST_DT_BF16 ? launch_dim<ST_DT_BF16>(dim, kind, (unsigned)n_items, stream, table_dev, items_dev)
                                   : launch_dim<ST_DT_F16>(dim, kind, (unsigned)n_items, stream, table_dev, items_dev));
}

template <int DT, bool READ, int TURNS>
static hipError_t launch_move(int dim, unsigned blocks, void* stream, const AttnDev* table, const AttnItem* items) {
  auto kernel = dim == 64 ? st_attn_move_kernel<DT, 64, READ, TURNS> : dim == 128 ? st_attn_move_kernel<DT, 128, READ, TURNS> : st_attn_move_kernel<DT, 256, READ, TURNS>;
  return launch(kernel, blocks, 256, stream, table, items);
}
template <int DT>
static hipError_t launch_move_any(bool read, bool many, int dim, unsigned blocks, void* stream, const AttnDev* table, const AttnItem* items) {
  const auto run = read ? (many ? launch_move<DT, true, kAttnMoveTurns> : launch_move<DT, true, 1>) : (many ? launch_move<DT, false, kAttnMoveTurns> : launch_move<DT, false, 1>);
  return run(dim, blocks, stream, table, items);
}
int launch_attn_move(bool read, bool many, int dtype, int dim, const AttnDev* table_dev, const AttnItem* items_dev, int64_t n_items, void* stream) {
  if (n_items <= 0) return 0;
  return (int)(dtype == ST_DT_BF16 ? launch_move_any<ST_DT_BF16>(read, many, dim, (unsigned)n_items, stream, table_dev, items_dev)
                                   : launch_move_any<ST_DT_F16>(read, many, dim, (unsigned)n_items, stream, table_dev, items_dev));
}

}  // namespace st
