// Matrix products of several tenants: validation, choice of tiles, work lists and the C ABI (include/st_lm.h).
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

struct st_matmul {
  std::vector<st_matmul_desc> descs;
  std::vector<st_matmul_tenant_info> info;
  std::vector<MatmulDev> tenants;      // host mirror of the device table
  struct Launch { int dtype, shape; int64_t begin, count; };
  std::vector<Launch> launches;
  std::vector<MatmulItem> items;       // of all launches, one after another
  st_matmul_plan_info totals = {};
  int device = 0;
  bool graphs_rebind = false;          // a graph may put other pointers into the device's table than the host's has
  char* d_arena = nullptr;             // the one device allocation: table, items, counters, partial tiles
  MatmulDev* d_tenants = nullptr;
  MatmulItem* d_items = nullptr;
};

namespace {

constexpr uint32_t kActs = ST_EPI_RELU | ST_EPI_GELU | ST_EPI_GELU_TANH | ST_EPI_SILU;
constexpr uint32_t kResiduals = ST_EPI_RESIDUAL | ST_EPI_RESIDUAL_LAST;

int64_t row_of(int64_t ld, int64_t dense) { return ld ? ld : dense; }

st_status validate_sizes(const st_matmul_desc& d, int t) {
  if (d.M < 0 || d.N <= 0 || d.K <= 0) return fail(ST_ERR_INVALID_ARG, "tenant %d: N and K must be positive and M not negative", t);
  if (d.in_dtype != ST_DT_F32 && d.in_dtype != ST_DT_BF16 && d.in_dtype != ST_DT_F16)
    return fail(ST_ERR_UNSUPPORTED, "tenant %d: unknown in_dtype %d", t, d.in_dtype);
  if (d.out_dtype != ST_DT_F32 && d.out_dtype != d.in_dtype)
    return fail(ST_ERR_UNSUPPORTED, "tenant %d: out_dtype must be f32 or equal to in_dtype", t);
  if (d.epilogue & ~(kActs | kResiduals | ST_EPI_BIAS)) return fail(ST_ERR_UNSUPPORTED, "tenant %d: unknown epilogue bits 0x%x", t, d.epilogue);
  if (__builtin_popcount(d.epilogue & kActs) > 1) return fail(ST_ERR_INVALID_ARG, "tenant %d: more than one activation", t);
  if ((d.epilogue & kResiduals) == kResiduals) return fail(ST_ERR_INVALID_ARG, "tenant %d: the residual is added once, before or after the activation", t);
  const bool res = (d.epilogue & kResiduals) != 0;
  if (d.ldx < 0 || d.ldw < 0 || d.ldy < 0 || d.ldr < 0 || (d.ldx && d.ldx < d.K) || (d.ldw && d.ldw < d.K) || (d.ldy && d.ldy < d.N) || (res && d.ldr && d.ldr < d.N))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: rows must not overlap the rows behind them", t);
  if (d.K > kMatmulMaxK || d.N > kMatmulMaxK || std::max(std::max(d.ldx, d.ldw), std::max(d.ldy, res ? d.ldr : 0)) > kMatmulMaxLd)
    return fail(ST_ERR_UNSUPPORTED, "tenant %d: rows of at most %d elements, at most %d apart", t, kMatmulMaxK, kMatmulMaxLd);
  return ST_OK;
}

st_status validate_pointers(const st_matmul_desc& d, const st_matmul_desc& p, int t) {      // sizes from d, pointers from p
  if (d.M == 0) return ST_OK;
  const bool res = (d.epilogue & kResiduals) != 0, bias = (d.epilogue & ST_EPI_BIAS) != 0;
  if (!p.x || !p.w || !p.y) return fail(ST_ERR_INVALID_ARG, "tenant %d: x, w and y must be non-NULL", t);
  if (bias && !p.bias) return fail(ST_ERR_INVALID_ARG, "tenant %d: ST_EPI_BIAS without a bias pointer", t);
  if (res && !p.residual) return fail(ST_ERR_INVALID_ARG, "tenant %d: a residual bit without a residual pointer", t);
  const int64_t es = elem_size(d.in_dtype), os = elem_size(d.out_dtype);
  if ((uintptr_t)p.x % es || (uintptr_t)p.w % es || (bias && (uintptr_t)p.bias % es) || (uintptr_t)p.y % os || (res && (uintptr_t)p.residual % os))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: a pointer is not a multiple of its element's size", t);
  const Span y = {(uintptr_t)p.y, d.M, d.N * os, row_of(d.ldy, d.N) * os};
  const Span x = {(uintptr_t)p.x, d.M, d.K * es, row_of(d.ldx, d.K) * es}, w = {(uintptr_t)p.w, d.N, d.K * es, row_of(d.ldw, d.K) * es};
  if (overlap(y, x) || overlap(y, w) || (bias && overlap(y, Span{(uintptr_t)p.bias, 1, d.N * es, d.N * es})))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: y must not overlap x, w or bias", t);
  const int64_t ldr = row_of(d.ldr, d.N);
  if (res && !(p.residual == p.y && ldr == row_of(d.ldy, d.N)) && overlap(y, Span{(uintptr_t)p.residual, d.M, d.N * os, ldr * os}))
    return fail(ST_ERR_INVALID_ARG, "tenant %d: residual must be y itself or not overlap it", t);
  return ST_OK;
}

void set_pointers(MatmulDev& T, const st_matmul_desc& d, const st_matmul_desc& p) {
  T.x = p.x; T.w = p.w; T.y = p.y;
  T.bias = (d.epilogue & ST_EPI_BIAS) ? p.bias : nullptr;
  T.res = (d.epilogue & kResiduals) ? p.residual : nullptr;
}

// ---- choice of a tile shape and of a division of the reduction -----------------------------------------------------------
// Microseconds of a launch of one shape: a workgroup alone takes first + steps step, a compute unit through which many pass busy_first +
// steps busy_step for each, some way towards whole rounds; a step costs `rough` more where rows are no multiple of 16 bytes; a divided reduction
// adds join and join_kb for each KiB of the tile's partial sums (and busy_kb per KiB of a slice); the operands come at 5 TB/s.  The largest of
// the three is the time, the others weigh a little.  Constants fitted to 523 products of 1 to 4096 rows, 64 to 8192 outputs and inputs, odd sizes among them, and
// 1 to 16 tenants, each measured with every shape and up to seven divisions: what it picks takes 0.8 % longer in the geometric mean
// than the fastest of them (2.3 % on 150 others).  [shape][fp32]
struct Cost { double first, step, busy_first, busy_step, join, join_kb, busy_kb, rounds, rough; };
constexpr Cost kCosts[kNumMatmulShapes][2] = {
    {{6.68, 0.797, 11.4, 1.3, 2.12, 0.0264, 0.0284, 0.425, 0.33}, {49.5, 26.1, 6.17, 0.758, 1.31, 0.0335, 0.0125, 1, 0.0134}},
    {{2.85, 0.531, 2.83, 0.441, 2.86, 0.00758, 0.0625, 0.494, 0.407}, {10.1, 1.15, 8.61, 1.61, 0.839, 0.00454, 0.0239, 0.312, 0.156}},
    {{0.886, 0.16, 1.06, 0.187, 1.45, 0.0124, 0.113, 0.758, 0.455}, {0.31, 0.562, 2.34, 0.446, 1.22, 0.0206, 0.0923, 1, 0.184}},
    {{12.2, 2.1, 3.21, 5.75, 6.99, 0.806, 0.00838, 0.431, 6.61}, {3.47, 0.329, 0.0943, 1.2, 0.784, 0.018, 0.0826, 1, 0.0131}},
    {{1.61, 0.112, 0.592, 0.794, 0.651, 0.0436, 0.238, 1, 3.13}, {4.09, 0.117, 0.333, 0.449, 0.772, 0.0156, 0.141, 1, 0.0545}},
    {{0.528, 0.231, 0.526, 0.326, 0.283, 0.0599, 0.522, 1, 0.731}, {0.139, 0.196, 0.472, 0.413, 0.52, 0.203, 0.0831, 0.661, 0.0649}},
    {{0.655, 0.1, 2, 0.108, 0.375, 0.194, 0.489, 0.831, 0.53}, {1.24, 0.0904, 1.78, 0.145, 0.7, 0.241, 0.213, 1, 0.00079}},
};
constexpr double kLaunchUs = 2.0;      // ... and what a launch takes beside them
constexpr int kMostSplit = 32;
// A tile's partial sums are reached by offsets of 32 bits of which 2^31 stands for none: a division that is asked for makes no more slices than this many bytes hold.
constexpr int64_t kMostPartialBytes = (int64_t)1 << 30;

int steps_of(const st_matmul_desc& d, int shape) {
  const int bytes = kMatmulShapes[shape].skinny ? kMatmulUnitBytes : kMatmulStepBytes;
  return cdiv((int64_t)(d.K / (16 / elem_size(d.in_dtype))) * 16, bytes);
}
// A tenant's least time, in the share of the chip that it needs of its launch: what it takes at the rates of the matrix cores and of memory.
double work_of(const st_matmul_desc& d) {
  const double es = elem_size(d.in_dtype), flops = 2.0 * d.M * d.N * d.K;
  return std::max(flops / (es == 4 ? 1.3e8 : 1.3e9), ((double)d.M * d.K + (double)d.N * d.K + (double)d.M * d.N) * es / 5e6);
}
double time_of(const st_matmul_desc& d, int shape, int split, double share) {
  const MatmulShape& S = kMatmulShapes[shape];
  const bool f32 = d.in_dtype == ST_DT_F32;
  const Cost& c = kCosts[shape][f32];
  const int steps = std::max(1, cdiv(std::max(1, steps_of(d, shape)), split * (S.skinny ? 4 : 1)));
  double items = (double)cdiv(d.M, S.MT) * cdiv(d.N, S.NT) * split / (kNumCUs * share);
  if (items > 1) items += c.rounds * (std::ceil(items) - items);
  const double kb = S.MT * S.NT * 4 / 1024.0, rough = (int64_t)d.K * elem_size(d.in_dtype) % 16 != 0 ? 1 + c.rough : 1;
  const double alone = c.first + steps * c.step * rough + (split > 1 ? c.join + c.join_kb * split * kb : 0.0);
  const double busy = items * (c.busy_first + steps * c.busy_step * rough + (split > 1 ? c.busy_kb * kb : 0.0));
  const double memory = ((double)d.N * d.K + (double)d.M * d.K) * elem_size(d.in_dtype) / (5e6 * share), most = std::max(alone, busy);
  return std::max(most, memory) + 0.25 * std::min(alone, busy) + 0.3 * std::min(memory, most);
}

struct Choice { int shape, split, per_split; };

// The division of the reduction that suits a tenant best in a shape, and its time.
Choice divide(const st_matmul_desc& d, int shape, double share, int forced, double* time) {
  const int steps = std::max(1, steps_of(d, shape));
  const MatmulShape& S = kMatmulShapes[shape];
  if (forced) forced = (int)std::min<int64_t>(forced, kMostPartialBytes / (S.MT * S.NT * 4));
  Choice best = {shape, 1, steps};
  *time = -1;
  for (int want = forced ? forced : 1; want <= (forced ? forced : kMostSplit); ++want) {
    const int per = cdiv(steps, std::min(want, steps)), split = cdiv(steps, per);
    const double t = time_of(d, shape, split, share);
    if (*time < 0 || t < *time) best = {shape, split, per}, *time = t;
  }
  return best;
}

// Shapes and divisions for tenants of one operand type.  Tenants of one shape go in one launch and share the chip by their work; launches run
// one after the other.  Either all take the same shape, whichever is best for them together, or each the one that is best for it alone.
double plan_together(const std::vector<st_matmul_desc>& descs, const std::vector<int>& who, const std::vector<int>& shape, int forced, std::vector<Choice>* out) {
  double total = 0;
  for (int s = 0; s < kNumMatmulShapes; ++s) {
    double work = 0, longest = -1;
    for (size_t i = 0; i < who.size(); ++i)
      if (shape[i] == s) work += work_of(descs[who[i]]);
    for (size_t i = 0; i < who.size(); ++i) {
      if (shape[i] != s) continue;
      double t;
      (*out)[i] = divide(descs[who[i]], s, std::max(work_of(descs[who[i]]) / work, 1e-4), forced, &t);
      longest = std::max(longest, t);
    }
    if (longest >= 0) total += kLaunchUs + longest;
  }
  return total;
}
// Skinny tiles are for tenants whose rows one of them holds.
bool holds_rows(const st_matmul_desc& d, int shape) { return !kMatmulShapes[shape].skinny || d.M <= kMatmulShapes[shape].MT; }
std::vector<Choice> choose(const std::vector<st_matmul_desc>& descs, const std::vector<int>& who, const st_plan_opts& o) {
  std::vector<Choice> best(who.size()), now(who.size());
  std::vector<int> shape(who.size());
  double least = -1;
  auto look = [&] {
    const double t = plan_together(descs, who, shape, o.split_k, &now);
    if (least < 0 || t < least) best = now, least = t;
  };
  for (int s = 0; s < kNumMatmulShapes; ++s) {
    if (o.tile_cfg && s != o.tile_cfg - 1) continue;
    std::fill(shape.begin(), shape.end(), s);
    if (o.tile_cfg || std::all_of(who.begin(), who.end(), [&](int t) { return holds_rows(descs[t], s); })) look();
  }
  if (!o.tile_cfg && who.size() > 1) {
    double work = 0;
    for (int t : who) work += work_of(descs[t]);
    for (size_t i = 0; i < who.size(); ++i) {
      double mine = -1, t;
      for (int s = 0; s < kNumMatmulShapes; ++s) {
        if (!holds_rows(descs[who[i]], s)) continue;
        divide(descs[who[i]], s, std::max(work_of(descs[who[i]]) / work, 1e-4), o.split_k, &t);
        if (mine < 0 || t < mine) shape[i] = s, mine = t;
      }
    }
    look();
  }
  return best;
}

// A tenant's items: blocks of 4 x 8 tiles, so that the workgroups that run side by side on an XCD share rows of x and w in its L2, cut
// into one stretch per XCD (workgroup b of a launch runs on XCD b mod 8).
void deal(int t, const st_matmul_tenant_info& ti, std::vector<MatmulItem> (&xcd)[kNumXCDs], int start) {
  std::vector<MatmulItem> all;
  all.reserve((size_t)ti.item_count);
  for (int bn = 0; bn < ti.tiles_n; bn += 8)
    for (int bm = 0; bm < ti.tiles_m; bm += 4)
      for (int n = bn; n < std::min(bn + 8, ti.tiles_n); ++n)
        for (int m = bm; m < std::min(bm + 4, ti.tiles_m); ++m)
          for (int s = 0; s < ti.split_k; ++s) all.push_back({(uint32_t)t, (uint32_t)m, (uint32_t)n, (uint32_t)s});
  const int64_t n = (int64_t)all.size();
  for (int x = 0; x < kNumXCDs; ++x)
    for (int64_t i = n * x / kNumXCDs; i < n * (x + 1) / kNumXCDs; ++i) xcd[(x + start) % kNumXCDs].push_back(all[(size_t)i]);
}

st_status upload(st_matmul* p) {
  const size_t n = p->tenants.size();
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  size_t ws = 0, counters = 0;
  for (size_t t = 0; t < n; ++t) {
    const st_matmul_tenant_info& ti = p->info[t];
    if (ti.split_k > 1) {
      ws += (size_t)ti.tiles_m * ti.tiles_n * ti.split_k * ti.MT * ti.NT * 4;
      counters += (size_t)ti.tiles_m * ti.tiles_n;
    }
  }
  p->totals.workspace_bytes = (int64_t)(ws + counters * 4);
  if (p->totals.host_only || p->items.empty()) return ST_OK;
  const size_t off_items = up(n * sizeof(MatmulDev)), off_counters = off_items + up(p->items.size() * sizeof(MatmulItem)), off_ws = off_counters + up(counters * 4);
  ST_HIP(hipGetDevice(&p->device));
  ST_HIP(hipMalloc((void**)&p->d_arena, off_ws + ws));
  p->d_tenants = (MatmulDev*)p->d_arena;
  p->d_items = (MatmulItem*)(p->d_arena + off_items);
  size_t wf = off_ws, ct = off_counters;
  for (size_t t = 0; t < n; ++t) {
    const st_matmul_tenant_info& ti = p->info[t];
    if (ti.split_k <= 1) continue;
    p->tenants[t].ws = (float*)(p->d_arena + wf);
    p->tenants[t].counters = (uint32_t*)(p->d_arena + ct);
    wf += (size_t)ti.tiles_m * ti.tiles_n * ti.split_k * ti.MT * ti.NT * 4;
    ct += (size_t)ti.tiles_m * ti.tiles_n * 4;
  }
  std::vector<char> host(off_ws, 0);
  std::memcpy(host.data(), p->tenants.data(), n * sizeof(MatmulDev));
  std::memcpy(host.data() + off_items, p->items.data(), p->items.size() * sizeof(MatmulItem));
  ST_HIP(hipMemcpy(p->d_arena, host.data(), off_ws, hipMemcpyHostToDevice));
  return ST_OK;
}

st_status build(st_matmul* p, const st_matmul_desc* descs, int n, const st_plan_opts& o) {
  p->descs.assign(descs, descs + n);
  p->info.assign((size_t)n, st_matmul_tenant_info{});
  p->tenants.assign((size_t)n, MatmulDev{});
  p->totals.n_tenants = n;
  p->totals.host_only = o.host_only;
  std::vector<Choice> choice((size_t)n, Choice{0, 1, 1});
  for (int dtype = 0; dtype < 3; ++dtype) {
    std::vector<int> who;
    for (int t = 0; t < n; ++t)
      if (descs[t].in_dtype == dtype && descs[t].M > 0) who.push_back(t);
    if (who.empty()) continue;
    const std::vector<Choice> c = choose(p->descs, who, o);
    for (size_t i = 0; i < who.size(); ++i) choice[(size_t)who[i]] = c[i];
  }
  for (int t = 0; t < n; ++t) {
    const st_matmul_desc& d = descs[t];
    const int64_t es = elem_size(d.in_dtype), os = elem_size(d.out_dtype);
    st_matmul_tenant_info& ti = p->info[t];
    MatmulDev& T = p->tenants[t];
    T.M = d.M; T.N = d.N; T.K = d.K;
    T.ldx = (int32_t)row_of(d.ldx, d.K); T.ldw = (int32_t)row_of(d.ldw, d.K); T.ldy = (int32_t)row_of(d.ldy, d.N); T.ldr = (int32_t)row_of(d.ldr, d.N);
    T.epilogue = d.epilogue;
    T.out_f32 = d.out_dtype == ST_DT_F32;
    set_pointers(T, d, d);
    const Choice& c = choice[(size_t)t];
    const MatmulShape& S = kMatmulShapes[c.shape];
    ti.tile_cfg = c.shape;
    ti.MT = S.MT; ti.NT = S.NT;
    ti.tiles_m = cdiv(d.M, S.MT); ti.tiles_n = cdiv(d.N, S.NT);
    ti.split_k = c.split;
    if ((double)ti.tiles_m * ti.tiles_n * ti.split_k >= 2147483648.0) return fail(ST_ERR_UNSUPPORTED, "tenant %d: more than 2^31 work items", t);
    ti.item_count = (int64_t)ti.tiles_m * ti.tiles_n * ti.split_k;
    T.tiles_n = ti.tiles_n; T.split = ti.split_k; T.per_split = c.per_split;
    p->totals.n_items += ti.item_count;
    if (d.M == 0) continue;
    p->totals.flops += 2 * (int64_t)d.M * d.N * d.K;
    p->totals.bytes += ((int64_t)d.M * d.K + (int64_t)d.N * d.K + ((d.epilogue & ST_EPI_BIAS) ? d.N : 0)) * es + (int64_t)d.M * d.N * os * ((d.epilogue & kResiduals) ? 2 : 1);
  }
  if (p->totals.n_items >= kMostWorkgroups) return fail(ST_ERR_UNSUPPORTED, "more than 2^23 workgroups");
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int shape = 0; shape < kNumMatmulShapes; ++shape) {
      std::vector<int> mine;
      for (int t = 0; t < n; ++t)
        if (p->info[t].item_count && descs[t].in_dtype == dtype && p->info[t].tile_cfg == shape) mine.push_back(t);
      if (mine.empty()) continue;
      // tenants whose items take longest come first
      std::stable_sort(mine.begin(), mine.end(), [&](int a, int b) { return p->tenants[a].per_split > p->tenants[b].per_split; });
      std::vector<MatmulItem> xcd[kNumXCDs];
      int start = 0;
      for (int t : mine) {
        deal(t, p->info[t], xcd, start);
        start = (int)((start + p->info[t].item_count) % kNumXCDs);
      }
      const int64_t begin = (int64_t)p->items.size();
      size_t most = 0;
      for (const auto& l : xcd) most = std::max(most, l.size());
      for (size_t i = 0; i < most; ++i)
        for (const auto& l : xcd)
          if (i < l.size()) p->items.push_back(l[i]);
      p->launches.push_back({dtype, shape, begin, (int64_t)p->items.size() - begin});
    }
  p->totals.launches = (int32_t)p->launches.size();
  return upload(p);
}

}  // namespace

extern "C" st_status st_matmul_plan(const st_matmul_desc* descs, int32_t n_tenants, const st_plan_opts* opts, st_matmul** out_plan) {
  if (!out_plan) return fail(ST_ERR_INVALID_ARG, "out_plan is NULL");
  *out_plan = nullptr;
  if (n_tenants < 0 || (n_tenants > 0 && !descs)) return fail(ST_ERR_INVALID_ARG, "descs is NULL or n_tenants negative");
  st_plan_opts o;
  std::memset(&o, 0, sizeof(o));
  if (opts) o = *opts;
  if (o.tile_cfg < 0 || o.tile_cfg > kNumMatmulShapes || o.split_k < 0 || o.reserved != 0) return fail(ST_ERR_INVALID_ARG, "bad plan options");
  for (int t = 0; t < n_tenants; ++t) {
    st_status s = validate_sizes(descs[t], t);
    if (s == ST_OK) s = validate_pointers(descs[t], descs[t], t);
    if (s != ST_OK) return s;
  }
  st_matmul* p = new (std::nothrow) st_matmul();
  if (!p) return fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  st_status s;
  try {
    s = build(p, descs, n_tenants, o);
  } catch (const std::exception&) {
    s = fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  }
  if (s != ST_OK) {
    st_matmul_destroy(p);
    return s;
  }
  *out_plan = p;
  return ST_OK;
}

extern "C" st_status st_matmul_run(const st_matmul* plan, void* hip_stream) {
  if (!plan) return fail(ST_ERR_INVALID_ARG, "plan is NULL");
  if (plan->totals.host_only) return fail(ST_ERR_UNSUPPORTED, "plan was built host-only and cannot run");
  if (plan->launches.empty()) return ST_OK;
  OnDevice on(plan->device);
  ST_HIP(on.error);
  for (const st_matmul::Launch& l : plan->launches)
    ST_HIP((hipError_t)launch_matmul(l.dtype, l.shape, plan->d_tenants, plan->d_items + l.begin, l.count, hip_stream));
  return ST_OK;
}

extern "C" st_status st_matmul_rebind_all(st_matmul* plan, const st_matmul_desc* descs, int32_t n_tenants, void* hip_stream) {
  if (!plan) return fail(ST_ERR_INVALID_ARG, "plan is NULL");
  if (n_tenants != (int32_t)plan->tenants.size()) return fail(ST_ERR_INVALID_ARG, "n_tenants differs from the plan's");
  if (n_tenants > 0 && !descs) return fail(ST_ERR_INVALID_ARG, "descs is NULL");
  for (int t = 0; t < n_tenants; ++t) {
    const st_status s = validate_pointers(plan->descs[t], descs[t], t);
    if (s != ST_OK) return s;
  }
  std::vector<MatmulDev> next;
  try {
    next = plan->tenants;
  } catch (const std::exception&) {
    return fail(ST_ERR_OUT_OF_MEMORY, "host allocation failed");
  }
  for (int t = 0; t < n_tenants; ++t) set_pointers(next[t], plan->descs[t], descs[t]);
  const bool same = n_tenants == 0 || std::memcmp(next.data(), plan->tenants.data(), next.size() * sizeof(MatmulDev)) == 0;
  if (!plan->totals.host_only && plan->d_tenants) {
    OnDevice on(plan->device);
    ST_HIP(on.error);
    bool captured = false;
    ST_HIP(is_captured(hip_stream, &captured));
    if (same && !captured && !plan->graphs_rebind) return ST_OK;
    ST_HIP((hipError_t)launch_poke(next.data(), (int64_t)(next.size() * sizeof(MatmulDev)), plan->d_tenants, hip_stream));
    plan->graphs_rebind |= captured;
  }
  plan->tenants.swap(next);
  for (int t = 0; t < n_tenants; ++t) {
    st_matmul_desc& d = plan->descs[t];
    d.x = descs[t].x; d.w = descs[t].w; d.bias = descs[t].bias; d.y = descs[t].y; d.residual = descs[t].residual;
  }
  return ST_OK;
}

extern "C" st_status st_matmul_get_info(const st_matmul* plan, st_matmul_plan_info* out) {
  if (!plan || !out) return fail(ST_ERR_INVALID_ARG, "NULL argument");
  *out = plan->totals;
  return ST_OK;
}

extern "C" st_status st_matmul_get_tenant_info(const st_matmul* plan, int32_t tenant, st_matmul_tenant_info* out) {
  if (!plan || !out) return fail(ST_ERR_INVALID_ARG, "NULL argument");
  if (tenant < 0 || (size_t)tenant >= plan->info.size()) return fail(ST_ERR_INVALID_ARG, "tenant index out of range");
  *out = plan->info[(size_t)tenant];
  return ST_OK;
}

extern "C" void st_matmul_destroy(st_matmul* plan) {
  if (!plan) return;
  if (plan->d_arena) (void)hipFree(plan->d_arena);
  delete plan;
}

extern "C" st_status st_matmul_tile_shape(int32_t index, int32_t* MT, int32_t* NT) {
  if (!MT || !NT) return fail(ST_ERR_INVALID_ARG, "NULL argument");
  if (index < 0 || index >= kNumMatmulShapes) return fail(ST_ERR_INVALID_ARG, "tile index out of range");
  *MT = kMatmulShapes[index].MT;
  *NT = kMatmulShapes[index].NT;
  return ST_OK;
}
extern "C" int32_t st_matmul_tile_count(void) { return kNumMatmulShapes; }
