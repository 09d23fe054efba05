// Attention over paged caches in 4 bits: validation, division of the work and the C ABI (include/st_lm.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "st_host.h"
#include "st_lm_host.h"
#include "st_lm_internal.h"

using namespace st;

struct st_attn {
  std::vector<st_attn_desc> descs;
  std::vector<AttnDev> tenants;        // host mirror of the device table
  struct Launch { int dtype, dim, kind; int64_t begin, count; };      // kind of a move: many new tokens
  std::vector<Launch> runs, moves;
  std::vector<AttnItem> items;         // of all launches, one after another
  bool can_append = true, can_read = true, can_run = true;      // every pointer is there that the call needs
  st_attn_info totals = {};
  int device = 0;
  bool graphs_rebind = false;          // a graph may put other pointers into the device's table than the host's has
  char* d_arena = nullptr;             // the one device allocation: table, items, status, counters, partial results
  AttnDev* d_tenants = nullptr;
  AttnItem* d_items = nullptr;
  uint32_t* d_status = nullptr;
};

namespace {

int64_t or_dense(int64_t ld, int64_t dense) { return ld ? ld : dense; }

bool layout_ok(const st_attn_desc& d) {
  const bool pages = d.page_tokens >= 16 && d.page_tokens <= 1024 && (d.page_tokens & (d.page_tokens - 1)) == 0;
  return d.kv_heads > 0 && (d.head_dim == 64 || d.head_dim == 128 || d.head_dim == 256) && pages;
}
int64_t page_bytes(const st_attn_desc& d) { return (int64_t)d.kv_heads * (d.page_tokens / kAttnBlock) * attn_block_bytes(d.head_dim); }

st_status validate_sizes(const st_attn_desc& d, int t) {
  if (d.heads <= 0 || d.kv_heads <= 0 || d.heads % d.kv_heads != 0)
    return fail(ST_ERR_INVALID_ARG, "tenant %d: heads must be a positive multiple of kv_heads", t);
  if (d.head_dim != 64 && d.head_dim != 128 && d.head_dim != 256) return fail(ST_ERR_UNSUPPORTED, "tenant %d: head_dim must be 64, 128 or 256", t);
  if (d.dtype != ST_DT_BF16 && d.dtype != ST_DT_F16) return fail(ST_ERR_UNSUPPORTED, "tenant %d: dtype must be bf16 or f16", t);
  if (!layout_ok(d)) return fail(ST_ERR_UNSUPPORTED, "tenant %d: page_tokens must be a power of two from 16 to 1024", t);
  if (d.n_seqs < 0 || d.max_tokens < 0 || d.max_new <= 0 || d.n_pages < 0 || d.table_pages < 0 || (d.n_seqs > 0 && d.table_pages == 0) || d.window < 0)
    return fail(ST_ERR_INVALID_ARG, "tenant %d: a negative size, or none where one is needed", t);
  if (d.flags & ~(uint32_t)ST_ATTN_CAUSAL) return fail(ST_ERR_UNSUPPORTED, "tenant %d: unknown flags 0x%x", t, d.flags);
  if (d.window > 0 && !(d.flags & ST_ATTN_CAUSAL)) return fail(ST_ERR_INVALID_ARG, "tenant %d: a window needs ST_ATTN_CAUSAL", t);
  if (!std::isfinite(d.scale)) return fail(ST_ERR_INVALID_ARG, "tenant %d: scale must be finite", t);
  if (d.reserved != 0) return fail(ST_ERR_INVALID_ARG, "tenant %d: reserved field must be 0", t);
  const int64_t wide = (int64_t)d.heads * d.head_dim, narrow = (int64_t)d.kv_heads * d.head_dim, far = (int64_t)1 << 32;
  if (d.ldq < 0 || d.ldk < 0 || d.ldv < 0 || d.ldo < 0 || (d.ldq && d.ldq < wide) || (d.ldo && d.ldo < wide) || (d.ldk && d.ldk < narrow) || (d.ldv && d.ldv < narrow))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: rows must not overlap the rows behind them", t);
  if (d.heads > (1 << 16) || page_bytes(d) >= ((int64_t)1 << 31) || std::max(std::max(d.ldq, d.ldk), std::max(d.ldv, d.ldo)) > far || (int64_t)d.table_pages * d.page_tokens >= ((int64_t)1 << 30) ||
      (int64_t)d.max_new * (d.heads / d.kv_heads) >= ((int64_t)1 << 30) || d.max_tokens >= (1 << 30) || d.n_seqs >= (1 << 24))
    return fail(ST_ERR_UNSUPPORTED, "tenant %d: more than 2^16 heads, a page of 2^31 bytes, rows more than 2^32 elements apart, or 2^30 tokens or more", t);
  return ST_OK;
}

// d: sizes, p: pointers.  *append, *read, *run are cleared where a pointer is missing that these calls need.
st_status validate_pointers(const st_attn_desc& d, const st_attn_desc& p, int t, bool* append, bool* read, bool* run) {
  const bool idle = d.n_seqs == 0 || d.max_tokens == 0;
  for (const void* e : {p.q, p.k, p.v, (const void*)p.out, (const void*)p.k_out, (const void*)p.v_out})
    if ((uintptr_t)e % 2) return fail(ST_ERR_INVALID_ARG, "tenant %d: a pointer is not a multiple of its element's size", t);
  for (const void* e : {(const void*)p.table, (const void*)p.first, (const void*)p.length})
    if ((uintptr_t)e % 4) return fail(ST_ERR_INVALID_ARG, "tenant %d: a pointer is not a multiple of its element's size", t);
  if ((uintptr_t)p.pages % 16) return fail(ST_ERR_INVALID_ARG, "tenant %d: pages must be a multiple of 16", t);
  auto rows = [&](const void* q, int64_t heads, int64_t ld) { return Span{(uintptr_t)q, q ? d.max_tokens : 0, heads * d.head_dim * 2, or_dense(ld, heads * d.head_dim) * 2}; };
  const Span q = rows(p.q, d.heads, d.ldq), out = rows(p.out, d.heads, d.ldo), k_out = rows(p.k_out, d.kv_heads, d.ldk), v_out = rows(p.v_out, d.kv_heads, d.ldv);
  const int64_t pool_bytes = d.n_pages * page_bytes(d);
  const Span pool = {(uintptr_t)p.pages, p.pages && pool_bytes ? 1 : 0, pool_bytes, pool_bytes};
  const Span k = rows(p.k, d.kv_heads, d.ldk), v = rows(p.v, d.kv_heads, d.ldv);
  if (overlap(out, q) || overlap(out, pool) || overlap(k_out, pool) || overlap(v_out, pool) || overlap(k_out, v_out) || overlap(k, pool) || overlap(v, pool))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: outputs must not overlap q, the pages or each other, nor k and v the pages", t);
  if (idle) return ST_OK;
  const bool tables = p.table && p.first && p.length && (p.pages || d.n_pages == 0);
  *append &= tables && p.k && p.v;
  *read &= tables && p.k_out && p.v_out;
  *run &= tables && p.q && p.out;
  return ST_OK;
}

void set_pointers(AttnDev& T, const st_attn_desc& p) {
  T.q = p.q; T.k = p.k; T.v = p.v; T.out = p.out; T.k_out = p.k_out; T.v_out = p.v_out;
  T.pages = p.pages; T.table = p.table; T.first = p.first; T.length = p.length;
}

// ---- division of the work ---------------------------------------------------------------------------------------------
// A window that the table has no room for hides nothing; left out, sums with it stay far below 2^31 on the device.
int window_of(const st_attn_desc& d) { return d.window < (int64_t)d.table_pages * d.page_tokens ? d.window : 0; }
int most_rows(const st_attn_desc& d) { return (int)((int64_t)d.max_new * (d.heads / d.kv_heads)); }
int most_steps(const st_attn_desc& d) {      // that a row tile of single tokens can have to go through
  int64_t tokens = (int64_t)d.table_pages * d.page_tokens;
  if (const int window = window_of(d)) tokens = std::min(tokens, (int64_t)window + d.max_new + kAttnStep);
  return cdiv(tokens, kAttnStep) + 1;
}
// Few rows: the tokens are divided among wavefronts and workgroups, for 32 rows at a time (16 with heads of 256); else the rows are.  Four times over
// the widening costs less than wavefronts without rows (one sequence of 8192, 8 and 47 of 4096; us by tokens and by rows): 64 rows of heads
// of 128 19.6 and 44, 24.6 and 46, 92 and 201; 128 rows 18.4 and 44, 30 and 46, 171 and 204; 192 33 and 45, but 57 and 47, 254
// and 210.  Heads of 256: 64 rows 21.6 and 64, 30.5 and 53, 132 and 185; 128 rows 22 and 65, 43 and 54, but 260 and 189.
int kind_of(const st_attn_desc& d) {
  const int rows = most_rows(d);
  return rows <= 16 ? kAttnTokens1 : rows <= (d.head_dim == 256 ? 64 : 128) ? kAttnTokens2 : kAttnRows;
}

// Workgroups that move a sequence's new tokens.
bool moves_many(const st_attn_desc& d) { return d.max_new >= kAttnBlock; }
int move_unit(const st_attn_desc& d) { return attn_move_count(d.head_dim) * (moves_many(d) ? kAttnMoveTurns : 1); }      // tokens x key heads of one
int64_t move_parts(const st_attn_desc& d) {
  const int64_t tokens = moves_many(d) ? ((int64_t)d.max_new + kAttnBlock - 1) / kAttnBlock * kAttnBlock : d.max_new;
  return (tokens * d.kv_heads + move_unit(d) - 1) / move_unit(d);
}
// How many parts all sequences' max_tokens rows can make together.  Where listing what each sequence can have alone takes more than kAttnLoose
// times as many, the parts' sequences are looked up instead: a workgroup without work holds its place for some two microseconds, a look-up
// costs every one that has some as much.  Append and attention in us, listed and looked up: 256 sequences of 32 new tokens and some 500 in
// all, max_new and max_tokens 8192 (107 times as many) 634 and 423, 12.7 and 148; 16 of 128, 2048 (12 times) 12.8 and 40.5, 5.1 and
// 36.9; 4 of 1024, 4096 (4 times) 8.7 and 66.5, 6.2 and 71.3.
constexpr int kAttnLoose = 4;
int64_t all_moves(const st_attn_desc& d) { return (int64_t)d.max_tokens * d.kv_heads / move_unit(d) + (int64_t)d.n_seqs * ((kAttnBlock - 1) * (int64_t)d.kv_heads / move_unit(d) + 2); }
bool find_moves(const st_attn_desc& d) { return moves_many(d) && d.n_seqs * move_parts(d) > kAttnLoose * all_moves(d); }
int64_t all_row_tiles(const st_attn_desc& d) {
  return (int64_t)d.max_tokens * (d.heads / d.kv_heads) / (attn_row_waves(d.head_dim) * 16 * attn_blocks(kAttnRows, d.head_dim)) + d.n_seqs;
}
bool find_rows(const st_attn_desc& d, int64_t row_tiles) { return kind_of(d) == kAttnRows && d.n_seqs * row_tiles > kAttnLoose * all_row_tiles(d); }

// Rows whose tokens are divided.  A stretch's tile of tokens takes some 1.7 us, and 2.9 where two workgroups share a compute unit (one does
// with heads of 256: 2.2); the last workgroup reads each stretch's sums in 2.8 us (5.5): sqrt(root tiles) stretches take least time, as
// far as there is room for them.  Either one workgroup to a compute unit, or two, if that makes nearly twice as many stretches.  Between one and
// two the chip is filled unevenly, and many short stretches even that out; so they do where lengths differ, if they are long (heads 16 and 2 of
// 256, 3000 of 8192 420 and 391 us; 1500 280 and 240), but not where one round of equal ones is just full.  In us, whole and divided (heads 32 and 8 of 128): 512 new tokens of
// 16384 430 and 159 (in 5), of 4096 112 and 58 (5), 128 of 8192 215 and 50 (9), 64 of 32768 843 and 89 (16), 2048 of 8192 304 and 254 (5).
constexpr int kMostRowSplit = 16;
void row_stretches(AttnDev& T, const st_attn_desc& d, double tiles, int most_steps) {
  const int one = std::max(1, (int)(kNumCUs / tiles)), two = d.head_dim == 256 ? one : std::max(1, (int)(2 * kNumCUs / tiles));
  T.root = d.head_dim == 256 ? 0.4f : 0.62f;
  T.whole = d.head_dim == 256 ? 10 : 8;
  T.want = std::min(one, kMostRowSplit);
  T.most = std::min(two > 1.8 * one ? two : one, kMostRowSplit);
  if (tiles > kNumCUs && tiles < 1.6 * kNumCUs && d.head_dim != 256) T.want = 3, T.most = 5;
  const double places = kNumCUs * (d.head_dim == 256 ? 1 : 2);
  T.least = tiles < 0.8 * places || (tiles > places && tiles < 1.6 * places) ? 3 : 1;
  const int room = std::min(std::max(T.most, T.want), (int)(std::sqrt((double)most_steps * T.root) + 1.0));
  T.split = most_steps <= T.whole ? 1 : std::max({1, room, std::min(T.least, most_steps / attn_level_steps(d.head_dim))});
}

st_status upload(st_attn* p) {
  const size_t n = p->tenants.size();
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  std::vector<size_t> tiles(n), floats(n);
  size_t all_tiles = 0, all_floats = 0;
  for (size_t t = 0; t < n; ++t) {
    const AttnDev& T = p->tenants[t];
    const st_attn_desc& d = p->descs[t];
    const int kind = kind_of(d);
    if (T.split <= 1) continue;
    tiles[t] = (size_t)T.kv_heads * (size_t)(find_rows(d, T.row_tiles) ? all_row_tiles(d) : (int64_t)T.n_seqs * T.row_tiles);
    floats[t] = tiles[t] * T.split * (size_t)(kind == kAttnRows ? attn_row_slot(kind, d.head_dim) : 16 * attn_blocks(kind, d.head_dim) * (d.head_dim + 2));
    all_tiles += tiles[t];
    all_floats += floats[t];
  }
  p->totals.workspace_bytes = (int64_t)(all_tiles * 4 + all_floats * 4);
  if (p->totals.host_only || p->items.empty()) return ST_OK;
  const size_t off_items = up(n * sizeof(AttnDev)), off_status = off_items + up(p->items.size() * sizeof(AttnItem));
  const size_t off_counters = off_status + 256, off_ws = off_counters + up(all_tiles * 4);
  ST_HIP(hipGetDevice(&p->device));
  ST_HIP(hipMalloc((void**)&p->d_arena, off_ws + all_floats * 4));
  p->d_tenants = (AttnDev*)p->d_arena;
  p->d_items = (AttnItem*)(p->d_arena + off_items);
  p->d_status = (uint32_t*)(p->d_arena + off_status);
  size_t wf = off_ws, ct = off_counters;
  for (size_t t = 0; t < n; ++t) {
    AttnDev& T = p->tenants[t];
    T.status = p->d_status;
    T.ws = (float*)(p->d_arena + wf);
    T.counters = (uint32_t*)(p->d_arena + ct);
    wf += floats[t] * 4;
    ct += tiles[t] * 4;
  }
  std::vector<char> host(off_ws, 0);
  std::memcpy(host.data(), p->tenants.data(), n * sizeof(AttnDev));
  std::memcpy(host.data() + off_items, p->items.data(), p->items.size() * sizeof(AttnItem));
  ST_HIP(hipMemcpy(p->d_arena, host.data(), off_ws, hipMemcpyHostToDevice));
  return ST_OK;
}

st_status build(st_attn* p, const st_attn_desc* descs, int n, const st_plan_opts& o) {
  p->descs.assign(descs, descs + n);
  p->tenants.assign((size_t)n, AttnDev{});
  p->totals.n_tenants = n;
  p->totals.host_only = o.host_only;
  double tiles = 0, row_tiles = 0;      // of all tenants of either kind
  for (int t = 0; t < n; ++t) {
    const st_attn_desc& d = descs[t];
    const int kind = kind_of(d);
    AttnDev& T = p->tenants[t];
    set_pointers(T, d);
    T.heads = d.heads; T.kv_heads = d.kv_heads; T.group = d.heads / d.kv_heads;
    T.ldq = or_dense(d.ldq, (int64_t)d.heads * d.head_dim); T.ldo = or_dense(d.ldo, (int64_t)d.heads * d.head_dim);
    T.ldk = or_dense(d.ldk, (int64_t)d.kv_heads * d.head_dim); T.ldv = or_dense(d.ldv, (int64_t)d.kv_heads * d.head_dim);
    T.n_seqs = d.n_seqs; T.max_tokens = d.max_tokens; T.max_new = d.max_new; T.n_pages = d.n_pages;
    T.page_shift = __builtin_ctz((unsigned)d.page_tokens);
    T.page_bytes = page_bytes(d);
    T.table_pages = d.table_pages; T.window = window_of(d); T.causal = (d.flags & ST_ATTN_CAUSAL) != 0;
    // hidden tokens get the score -inf, which has to stay that under the scale: a negative one changes the queries' signs instead, and one of
    // 0, or so small, counts as 2^-100, under which all finite scores are equal, too
    const float twice = d.dtype == ST_DT_F16 ? 2.f : 1.f;      // keys are widened under half their scale there (see kHalved in st_attn.hip)
    T.scale = twice * std::min(std::max(std::fabs(d.scale) * 1.44269504088896340736f, 7.888609e-31f), 3.0e38f / twice);
    T.flip = d.scale < 0 ? 0x80008000u : 0u;
    T.row_tiles = cdiv(most_rows(d), (kind == kAttnRows ? attn_row_waves(d.head_dim) : 1) * 16 * attn_blocks(kind, d.head_dim));
    T.split = 1;
    if (d.max_tokens > 0 && d.n_seqs > 0 && kind != kAttnRows) tiles += (double)d.n_seqs * d.kv_heads * T.row_tiles;
    if (d.max_tokens > 0 && d.n_seqs > 0 && kind == kAttnRows) row_tiles += (double)std::min((int64_t)d.n_seqs * T.row_tiles, all_row_tiles(d)) * d.kv_heads;
  }
  int64_t n_items = 0, n_moves = 0;
  for (int t = 0; t < n; ++t) {
    const st_attn_desc& d = descs[t];
    AttnDev& T = p->tenants[t];
    if (d.n_seqs == 0 || d.max_tokens == 0) continue;
    const int steps = most_steps(d);
    if (kind_of(d) != kAttnRows) {
      // A stretch on every compute unit, not one more: that would share its unit with another (single tokens of 5, 10 and 20 sequences of 8192 in
      // 240 workgroups 16.2, 21.7 us and 160 38.2, in 280 to 320 20.4, 27.7, 44.8; 32 of 8000 with heads of 256, 128, 256, 512 workgroups:
      // 43.1, 28.4, 36.3), and more of them cost their set-up and their joining (one context of 131072 with 24, 32, 64 stretches: 35.3, 36.9, 42.9).  But none longer
      // than 192 steps where there are more sequences' heads than units, or a few long ones outlast the others (64 of up to 8192: 75.5 us in one
      // stretch each, 66.9 in two),
      // and short ones whole (a single sequence of 1000: 8.2 us whole, 9.1 in two; of 2000: 12.0 whole, 9.5 in four; of 4000: 19.9, 9.9 in eight).
      T.want = std::max(1, std::min(kAttnMaxSplit, (int)(kNumCUs / tiles)));
      const bool thirds = tiles > 0.5 * kNumCUs && 3 * tiles <= 2 * kNumCUs;      // 20 of 65536 in three 250 us, whole 272, in two 318; of 8192 36, 39, 45; of 2000 16.4, 14.5
      if (thirds) T.want = 3;
      T.whole = thirds ? 128 : 40; T.most = tiles > kNumCUs ? 192 : 8 * 192; T.least = 2 * kAttnTokenWaves;
      if (o.split_k > 0) T.want = std::min(o.split_k, kAttnMaxSplit), T.whole = 0, T.most = 1 << 30, T.least = 1;
      // ... as far as the table has no more room than is used: 2048 workgroups in all, as those of stretches that there are not take time, too
      const int parts = std::max(T.want, std::min({kAttnMaxSplit, cdiv(steps, T.most), (int)std::max(1.0, 2048 / tiles)}));
      T.split = steps <= T.whole ? 1 : std::min(parts, cdiv(steps, T.least));
      T.want = std::min(T.want, T.split);
      T.chunk = std::max(T.least, cdiv(steps, T.split));
    } else {
      row_stretches(T, d, row_tiles, steps / (kAttnRowTokens / kAttnStep) + 2);
      if (o.split_k > 0) T.split = T.want = T.most = std::min(o.split_k, kMostRowSplit), T.root = 1e12f, T.whole = 0, T.least = 1;
    }
    n_items += find_rows(d, T.row_tiles) ? all_row_tiles(d) * d.kv_heads * T.split + 1 : (int64_t)d.n_seqs * d.kv_heads * T.row_tiles * T.split;
    n_moves += find_moves(d) ? all_moves(d) + 1 : d.n_seqs * move_parts(d);
    if (n_items >= kMostWorkgroups || n_moves >= kMostWorkgroups) return fail(ST_ERR_UNSUPPORTED, "more than 2^23 workgroups");
  }
  for (int dtype : {ST_DT_BF16, ST_DT_F16})
    for (int dim : {64, 128, 256}) {
      for (int kind = 0; kind < kNumAttnKinds; ++kind) {
        const int64_t begin = (int64_t)p->items.size();
        for (int t = 0; t < n; ++t) {
          const st_attn_desc& d = descs[t];
          const AttnDev& T = p->tenants[t];
          if (d.dtype != dtype || d.head_dim != dim || (kind_of(d) == kAttnRows && T.split > 1 ? kAttnRowsSplit : kind_of(d)) != kind || d.n_seqs == 0 || d.max_tokens == 0) continue;
          if (find_rows(d, T.row_tiles)) {
            p->items.push_back({(uint32_t)t, kAttnCheck, 0u, 0u});
            for (int stretch = 0; stretch < T.split; ++stretch)
              for (int64_t tile = 0; tile < all_row_tiles(d); ++tile)
                for (int h = 0; h < d.kv_heads; ++h) p->items.push_back({(uint32_t)t, kAttnFind, (uint32_t)h, (uint32_t)(tile * T.split + stretch)});
            continue;
          }
          // a sequence's last rows see most; a key head's row tiles stay on one XCD where the heads divide well
          for (int stretch = 0; stretch < T.split; ++stretch)      // stretches that there are not, come last
            for (int tile = T.row_tiles - 1; tile >= 0; --tile)
              for (int s = 0; s < d.n_seqs; ++s)
                for (int h = 0; h < d.kv_heads; ++h) p->items.push_back({(uint32_t)t, (uint32_t)s, (uint32_t)h, (uint32_t)(tile * T.split + stretch)});
        }
        if ((int64_t)p->items.size() > begin) p->runs.push_back({dtype, dim, kind, begin, (int64_t)p->items.size() - begin});
      }
      p->totals.n_items = (int64_t)p->items.size();
    }
  p->totals.launches = (int32_t)p->runs.size();
  for (int dtype : {ST_DT_BF16, ST_DT_F16})
    for (int dim : {64, 128, 256})
      for (int many = 0; many < 2; ++many) {
        const int64_t begin = (int64_t)p->items.size();
        for (int t = 0; t < n; ++t) {
          const st_attn_desc& d = descs[t];
          if (d.dtype != dtype || d.head_dim != dim || moves_many(d) != (many != 0) || d.n_seqs == 0 || d.max_tokens == 0) continue;
          if (find_moves(d)) {
            p->items.push_back({(uint32_t)t, kAttnCheck, 0u, 0u});
            for (int64_t part = 0; part < all_moves(d); ++part) p->items.push_back({(uint32_t)t, kAttnFind, 0u, (uint32_t)part});
            continue;
          }
          const int parts = (int)move_parts(d);
          for (int s = 0; s < d.n_seqs; ++s)
            for (int part = 0; part < parts; ++part) p->items.push_back({(uint32_t)t, (uint32_t)s, 0u, (uint32_t)part});
        }
        if ((int64_t)p->items.size() > begin) p->moves.push_back({dtype, dim, many, begin, (int64_t)p->items.size() - begin});
      }
  return upload(p);
}

st_status check_runnable(const st_attn* plan) {
  if (!plan) return fail(ST_ERR_INVALID_ARG, "plan is NULL");
  if (plan->totals.host_only) return fail(ST_ERR_UNSUPPORTED, "plan was built host-only and cannot run");
  return ST_OK;
}

st_status move(const st_attn* plan, bool read, void* hip_stream) {
  const st_status s = check_runnable(plan);
  if (s != ST_OK) return s;
  if (!(read ? plan->can_read : plan->can_append)) return fail(ST_ERR_INVALID_ARG, read ? "k_out, v_out or a table is NULL" : "k, v or a table is NULL");
  if (plan->moves.empty()) return ST_OK;
  OnDevice on(plan->device);
  ST_HIP(on.error);
  for (const st_attn::Launch& l : plan->moves)
    ST_HIP((hipError_t)launch_attn_move(read, l.kind != 0, l.dtype, l.dim, plan->d_tenants, plan->d_items + l.begin, l.count, hip_stream));
  return ST_OK;
}

}  // namespace

extern "C" int64_t st_attn_page_bytes(const st_attn_desc* desc) { return desc && layout_ok(*desc) ? page_bytes(*desc) : -1; }

extern "C" st_status st_attn_plan(const st_attn_desc* descs, int32_t n_tenants, const st_plan_opts* opts, st_attn** out_plan) {
  if (!out_plan) return fail(ST_ERR_INVALID_ARG, "out_plan is NULL");
  *out_plan = nullptr;
  if (n_tenants < 0 || (n_tenants > 0 && !descs)) return fail(ST_ERR_INVALID_ARG, "descs is NULL or n_tenants negative");
  st_plan_opts o;
  std::memset(&o, 0, sizeof(o));
  if (opts) o = *opts;
  if (o.split_k < 0 || o.reserved != 0) return fail(ST_ERR_INVALID_ARG, "bad plan options");
  bool append = true, read = true, run = true;
  for (int t = 0; t < n_tenants; ++t) {
    st_status s = validate_sizes(descs[t], t);
    if (s == ST_OK) s = validate_pointers(descs[t], descs[t], t, &append, &read, &run);
    if (s != ST_OK) return s;
  }
  st_attn* p = new (std::nothrow) st_attn();
  if (!p) return fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  p->can_append = append; p->can_read = read; p->can_run = run;
  st_status s;
  try {
    s = build(p, descs, n_tenants, o);
  } catch (const std::exception&) {
    s = fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  }
  if (s != ST_OK) {
    st_attn_destroy(p);
    return s;
  }
  *out_plan = p;
  return ST_OK;
}

extern "C" st_status st_attn_append(const st_attn* plan, void* hip_stream) { return move(plan, false, hip_stream); }
extern "C" st_status st_attn_read(const st_attn* plan, void* hip_stream) { return move(plan, true, hip_stream); }

extern "C" st_status st_attn_run(const st_attn* plan, void* hip_stream) {
  const st_status s = check_runnable(plan);
  if (s != ST_OK) return s;
  if (!plan->can_run) return fail(ST_ERR_INVALID_ARG, "q, out or a table is NULL");
  if (plan->runs.empty()) return ST_OK;
  OnDevice on(plan->device);
  ST_HIP(on.error);
  for (const st_attn::Launch& l : plan->runs)
    ST_HIP((hipError_t)launch_attn(l.dtype, l.dim, l.kind, plan->d_tenants, plan->d_items + l.begin, l.count, hip_stream));
  return ST_OK;
}

extern "C" st_status st_attn_rebind_all(st_attn* plan, const st_attn_desc* descs, int32_t n_tenants, void* hip_stream) {
  if (!plan) return fail(ST_ERR_INVALID_ARG, "plan is NULL");
  if (n_tenants != (int32_t)plan->tenants.size()) return fail(ST_ERR_INVALID_ARG, "n_tenants differs from the plan's");
  if (n_tenants > 0 && !descs) return fail(ST_ERR_INVALID_ARG, "descs is NULL");
  bool append = true, read = true, run = true;
  for (int t = 0; t < n_tenants; ++t) {
    const st_status s = validate_pointers(plan->descs[t], descs[t], t, &append, &read, &run);
    if (s != ST_OK) return s;
  }
  std::vector<AttnDev> next;
  try {
    next = plan->tenants;
  } catch (const std::exception&) {
    return fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  }
  for (int t = 0; t < n_tenants; ++t) set_pointers(next[t], descs[t]);
  const bool same = n_tenants == 0 || std::memcmp(next.data(), plan->tenants.data(), next.size() * sizeof(AttnDev)) == 0;
  if (plan->d_tenants) {
    OnDevice on(plan->device);
    ST_HIP(on.error);
    bool captured = false;
    ST_HIP(is_captured(hip_stream, &captured));
    if (!same || captured || plan->graphs_rebind) ST_HIP((hipError_t)launch_poke(next.data(), (int64_t)(next.size() * sizeof(AttnDev)), plan->d_tenants, hip_stream));
    plan->graphs_rebind |= captured;
  }
  plan->tenants.swap(next);
  plan->can_append = append; plan->can_read = read; plan->can_run = run;
  for (int t = 0; t < n_tenants; ++t) {
    st_attn_desc& d = plan->descs[t];
    const st_attn_desc& f = descs[t];
    d.q = f.q; d.k = f.k; d.v = f.v; d.out = f.out; d.k_out = f.k_out; d.v_out = f.v_out;
    d.pages = f.pages; d.table = f.table; d.first = f.first; d.length = f.length;
  }
  return ST_OK;
}

extern "C" st_status st_attn_status(st_attn* plan, int32_t* bits) {
  if (!bits) return fail(ST_ERR_INVALID_ARG, "NULL argument");
  const st_status s = check_runnable(plan);
  if (s != ST_OK) return s;
  uint32_t found = 0;
  if (plan->d_status) {
    OnDevice on(plan->device);
    ST_HIP(on.error);
    ST_HIP(hipDeviceSynchronize());
    ST_HIP(hipMemcpy(&found, plan->d_status, 4, hipMemcpyDeviceToHost));
    const uint32_t none = 0;
    if (found) ST_HIP(hipMemcpy(plan->d_status, &none, 4, hipMemcpyHostToDevice));
  }
  *bits = (int32_t)found;
  return ST_OK;
}

extern "C" st_status st_attn_get_info(const st_attn* plan, st_attn_info* out) {
  if (!plan || !out) return fail(ST_ERR_INVALID_ARG, "NULL argument");
  *out = plan->totals;
  return ST_OK;
}

extern "C" void st_attn_destroy(st_attn* plan) {
  if (!plan) return;
  if (plan->d_arena) (void)hipFree(plan->d_arena);
  delete plan;
}
