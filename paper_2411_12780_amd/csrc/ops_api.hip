// C entry points of the operators that work on a caller's own buffers (include/ppll.h): argument checks on the host, the layout of the
// workspace, then the launches.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "ortho.h"
#include "rotary.h"

namespace ppll {

namespace {
constexpr int64_t FAR = (int64_t)1 << 40;          // offsets and strides below it: no sum of them passes 64 bits
constexpr int64_t MOST_ITEMS = (1 << 24) - 1;      // workgroups of 256 threads that a launch takes: under 2^32 threads

int64_t extent(const ppll_matrix_group& g) { return (int64_t)(g.rows - 1) * g.ld + g.cols; }
// A group as matrices one behind the other, each of `parts` blocks of columns `step` apart: matrices side by side are the blocks of one.
struct Run { int64_t offset, stride, ld, rows, count, cols, step, parts; };
Run run_of(const ppll_matrix_group& g) {
  if (g.count > 1 && g.stride < extent(g)) return {g.offset, 0, g.ld, g.rows, 1, g.cols, g.stride, g.count};
  return {g.offset, g.stride, g.ld, g.rows, g.count, g.cols, 0, 1};
}
// Whether one of a run's blocks of columns meets columns lo .. hi - 1
bool meets(const Run& a, int64_t lo, int64_t hi) {
  const int64_t i = a.parts > 1 && lo >= a.cols ? (lo - a.cols) / a.step + 1 : 0;      // the first block that ends behind lo
  return i < a.parts && i * a.step < hi && i * a.step + a.cols > lo;
}
// Whether matrices of two runs may share an element: their extents meet, and they are not different columns of rows of one length.
bool overlap(const Run& a, const Run& b) {
  auto length = [](const Run& r) { return (r.rows - 1) * r.ld + (r.parts - 1) * r.step + r.cols; };
  const int64_t ea = length(a), eb = length(b), apart = b.offset - a.offset;
  if (apart >= (a.count - 1) * a.stride + ea || -apart >= (b.count - 1) * b.stride + eb) return false;
  auto share = [&](int64_t from) {         // matrices that begin `from` elements from one another
    if (from >= ea || -from >= eb) return false;
    if (a.ld != b.ld) return true;
    const int64_t d = (from % a.ld + a.ld) % a.ld;
    // b's columns from d on, and a's from 0 and (the next row's) from ld on; block by block of the run that has fewer
    const bool by_a = a.parts < b.parts;
    for (int64_t j = 0; j < (by_a ? a.parts : b.parts); ++j) {
      const int64_t lo = by_a ? j * a.step - d : d + j * b.step, hi = lo + (by_a ? a.cols : b.cols), row = by_a ? a.ld : -a.ld;
      if (meets(by_a ? b : a, lo, hi) || meets(by_a ? b : a, lo + row, hi + row)) return true;
    }
    return false;
  };
  if (a.count == 1 || b.count == 1 || a.stride == b.stride) {
    // i-th and j-th begin apart + (j - i) stride from one another: j - i from where they first meet
    const int64_t stride = b.count > 1 ? b.stride : a.stride;
    int64_t k = a.count > 1 || b.count > 1 ? std::max<int64_t>(1 - a.count, (-eb - apart) / stride - 1) : 0;
    for (; k < b.count && apart + k * stride < ea; ++k)
      if (share(apart + k * stride)) return true;
    return false;
  }
  int64_t i = 0, j = 0;
  while (i < a.count && j < b.count) {
    const int64_t la = i * a.stride, lb = apart + j * b.stride;
    if (share(lb - la)) return true;
    if (la + ea < lb + eb) ++i;
    else ++j;
  }
  return false;
}
// Clocks that a workgroup spends on its part of a tile, two of them on a unit: those that every part costs (finding its place, the first copies' way,
// the epilogue), those of 64 k, and of a tile in pieces the way of its sums through memory.
double part_clocks(const OrthoGroup& g, int tile, int phase, int pieces) {
  const double stages = (phase == ORTHO_GRAM ? g.np : g.mp) / 64 / (double)pieces;
  return tile == 128 ? 10000 + stages * 3200 + (pieces > 1 ? 8000 + 2000 * pieces : 0) : 7000 + stages * 1150 + (pieces > 1 ? 4500 + 700 * pieces : 0);
}
int pieces_of(const OrthoGroup& g, int phase, int length) {
  const int k = phase == ORTHO_GRAM ? g.np : g.mp;
  return phase <= ORTHO_POLY ? std::max(1, (k + length / 2) / length) : 1;
}
// Tiles of one of the products, into how many pieces the k of each is split, and how the XCDs share them.  Taken is what fills rounds of 512 workgroups
// (two on a unit) in the least time: whole rounds, the last one filled up with the shortest part, and none shorter than the longest.  Measured, five
// steps: one matrix of 256 x 2048 (10 tiles of 64) 205 us whole, 145 in eight pieces; 512 x 512 160 and 168, so whole; two of 1536 x 6144 1893 in tiles
// of 64 (600, little more than a round), 1685 in tiles of 128 in three pieces (468).
void plan_product(OrthoPlan* p, int phase) {
  OrthoProduct& o = p->product[phase];
  int longest_k = 0, length = 1 << 20;
  for (int k = 0; k < p->n; ++k)
    if (!p->g[k].small) longest_k = std::max(longest_k, phase == ORTHO_GRAM ? p->g[k].np : p->g[k].mp);
  double best = 0;
  for (int tile : {128, 64})
    for (int most : {1, 2, 3, 4, 6, 8}) {
      if (most > 1 && (phase > ORTHO_POLY || longest_k < 128 * most)) break;
      const int len = most == 1 ? 1 << 20 : longest_k / most;
      double all = 0, longest = 0, parts = 0, last = 0;
      for (int k = 0; k < p->n; ++k) {
        const OrthoGroup& g = p->g[k];
        if (g.small) continue;
        const int pieces = pieces_of(g, phase, len);
        const double one = part_clocks(g, tile, phase, pieces), n = (double)g.count * tiles_of_matrix(g, tile, phase) * pieces;
        all += n * one;
        parts += n;
        longest = std::max(longest, one);
        last = last > 0 ? std::min(last, one) : one;
      }
      const double time = std::max((all + (std::ceil(parts / 512) * 512 - parts) * last) / 512, longest);
      if (best == 0 || time < best) { best = time; o.tile = tile; length = len; }
    }
  // shares of equal work, in whole parts
  double all = 0, before = 0;
  int32_t parts = 0, x = 0, split_tiles = 0;
  int64_t split_parts = 0;
  for (int k = 0; k < p->n; ++k) {
    OrthoProduct::Group& part = o.group[k];
    part.tiles = tiles_of_matrix(p->g[k], o.tile, phase);
    part.split = pieces_of(p->g[k], phase, length);
    part.each = part.tiles * part.split;
    part.tile_of = split_tiles;
    part.sums_of = 4 * (int64_t)o.tile * o.tile * split_parts;
    if (part.split > 1) { split_tiles += p->g[k].count * part.tiles; split_parts += (int64_t)p->g[k].count * part.each; }
    all += (double)p->g[k].count * part.each * part_clocks(p->g[k], o.tile, phase, part.split);
  }
  p->counters = std::max(p->counters, split_tiles);
  p->sums = std::max<int64_t>(p->sums, 4 * (int64_t)o.tile * o.tile * split_parts);
  o.first[0] = 0;
  for (int k = 0; k < p->n; ++k) {
    o.begin[k] = parts;
    const int32_t n = p->g[k].count * o.group[k].each;
    const double one = part_clocks(p->g[k], o.tile, phase, o.group[k].split);
    // the boundaries that fall into this group
    while (x < 7 && n > 0 && before + n * one >= all * (x + 1) / 8)
      o.first[++x] = parts + (int32_t)std::min<double>(n, std::ceil((all * (x + 1) / 8 - before) / one));
    before += n * one;
    parts += n;
  }
  for (int k = p->n; k < ORTHO_GROUPS; ++k) o.begin[k] = parts;
  while (x < 8) o.first[++x] = parts;
}
template <class EACH> void count_items(const OrthoPlan& p, OrthoItems* items, EACH each) {
  int32_t at = 0;
  for (int k = 0; k < ORTHO_GROUPS; ++k) {
    items->begin[k] = at;
    if (k >= p.n) continue;
    items->each[k] = each(p.g[k]);
    at += p.g[k].count * items->each[k];
  }
}
int64_t pad(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
}  // namespace

int ortho_plan(const ppll_matrix_group* groups, int32_t n_groups, OrthoPlan* plan) {
  if (n_groups < 0 || n_groups > ORTHO_GROUPS) { set_error("%d groups, 0 to %d are possible", n_groups, ORTHO_GROUPS); return PPLL_ERR_SHAPE; }
  if (n_groups > 0 && !groups) { set_error("groups is null"); return PPLL_ERR_NULL; }
  *plan = OrthoPlan{};
  Run runs[ORTHO_GROUPS];
  for (int k = 0; k < n_groups; ++k) {
    const ppll_matrix_group& g = groups[k];
    if (g.rows < 1 || g.cols < 1 || g.rows > ORTHO_SIDE || g.cols > ORTHO_SIDE) {
      set_error("group %d: %d x %d outside 1..%d", k, g.rows, g.cols, ORTHO_SIDE);
      return PPLL_ERR_SHAPE;
    }
    if (g.count < 0 || g.count > ORTHO_COUNT) { set_error("group %d: count %d outside 0..%d", k, g.count, ORTHO_COUNT); return PPLL_ERR_SHAPE; }
    if (g.reserved) { set_error("group %d: reserved is not 0", k); return PPLL_ERR_SHAPE; }
    if (g.offset < 0 || g.stride < 0 || g.offset >= FAR || g.stride >= FAR || g.ld < g.cols || g.ld >= FAR >> 13) {
      set_error("group %d: offset, stride or ld out of range", k);
      return PPLL_ERR_SHAPE;
    }
    if (g.count > 1 && g.stride < extent(g) && !(g.stride >= g.cols && (g.count - 1) * g.stride + g.cols <= g.ld)) {
      set_error("group %d: its matrices share elements", k);
      return PPLL_ERR_SHAPE;
    }
    if (!g.count) continue;
    runs[plan->n] = run_of(g);
    for (int i = 0; i < plan->n; ++i)
      if (overlap(runs[i], runs[plan->n])) { set_error("group %d shares elements with a group before it", k); return PPLL_ERR_SHAPE; }
    OrthoGroup& o = plan->g[plan->n++];
    o.offset = g.offset; o.stride = g.stride; o.ld = g.ld;
    o.rows = g.rows; o.cols = g.cols; o.count = g.count;
    o.tall = g.rows > g.cols;
    o.m = o.tall ? g.cols : g.rows; o.n = o.tall ? g.rows : g.cols;
    o.mp = (int32_t)pad(o.m, 32); o.np = (int32_t)pad(o.n, 32);
    o.small = small_room(o).bytes <= ORTHO_SMALL_LDS;
    if (!o.small) { o.mp = (int32_t)pad(o.m, 64); o.np = (int32_t)pad(o.n, 64); }
  }
  std::stable_sort(plan->g, plan->g + plan->n, [](const OrthoGroup& a, const OrthoGroup& b) { return a.np > b.np; });
  int64_t at = 0, pieces = 0, matrices = 0, squares = 0;
  auto take = [&](int64_t bytes) { const int64_t p = at; at = pad(at + bytes, 256); return p; };
  for (int k = 0; k < plan->n; ++k) {
    OrthoGroup& o = plan->g[k];
    if (o.small) continue;
    o.first = (int32_t)matrices; o.first_piece = (int32_t)pieces;
    matrices += o.count; pieces += (int64_t)o.count * o.pieces();
    squares += (int64_t)o.count * (o.mp / 64) * (o.np / 64);
    o.x[0] = take(o.count * 2 * 2 * o.plane_x());
    o.x[1] = take(o.count * 2 * 2 * o.plane_x());
    o.a = take(o.count * 2 * 2 * o.plane_a());
    o.b = take(o.count * 2 * 2 * o.plane_a());
    if (pieces > MOST_ITEMS || squares > MOST_ITEMS) { set_error("too many matrices for one call"); return PPLL_ERR_SHAPE; }
  }
  for (int phase = 0; phase < 3; ++phase) {
    plan_product(plan, phase);
    if (8 * (int64_t)plan->product[phase].longest() > MOST_ITEMS) { set_error("too many matrices for one call"); return PPLL_ERR_SHAPE; }
  }
  plan->sums = take(plan->sums);
  plan->arrived = take(plan->counters * (int64_t)sizeof(int32_t));
  count_items(*plan, &plan->pieces, [](const OrthoGroup& g) { return g.small ? 0 : g.pieces(); });
  count_items(*plan, &plan->squares, [](const OrthoGroup& g) { return g.small ? 0 : g.mp / 64 * (g.np / 64); });
  count_items(*plan, &plan->small, [](const OrthoGroup& g) { return g.small ? 1 : 0; });
  plan->partials = take(pieces * (int64_t)sizeof(double));
  plan->shrink = take(matrices * (int64_t)sizeof(float));
  plan->bytes = at;
  return PPLL_OK;
}

int rotary_plan(const ppll_rotary_config* c, RotaryPlan* p) {
  if (!c) { set_error("rotary config is null"); return PPLL_ERR_NULL; }
  auto bad = [](const char* what) { set_error("rotary config: %s", what); return PPLL_ERR_CONFIG; };
  if (c->struct_size != sizeof(ppll_rotary_config)) return bad("struct_size");
  if (c->precision != PPLL_FP32 && c->precision != PPLL_BF16) return bad("precision must be PPLL_FP32 or PPLL_BF16");
  if (c->rows < 0 || c->tokens < 1 || c->rows % c->tokens) return bad("rows must be a multiple of tokens >= 1");
  if (c->q_heads < 0 || c->k_heads < 0 || c->q_heads > 65536 || c->k_heads > 65536 || c->q_heads + c->k_heads < 1)
    return bad("heads outside 0..65536, or none");
  if (c->head_dim < 2 || c->head_dim > 2 * ROTARY_PAIRS || c->head_dim % 2) return bad("head_dim must be even, 2..256");
  if (c->axes < 1 || c->axes > 3) return bad("axes outside 1..3");
  if (!(c->base > 0.f) || !std::isfinite(c->base)) return bad("base must be positive and finite");
  p->rows = c->rows; p->tokens = c->tokens; p->heads[0] = c->q_heads; p->heads[1] = c->k_heads;
  p->hd = c->head_dim; p->axes = c->axes; p->neighbours = c->neighbours != 0; p->eps = c->norm_eps;
  // (exp2 takes a third of pow's time, of the 0.7 us of a call with 32 pairs; the exponent's rounding is a relative 1e-16 for each octave,
  // which a pair that turns less feels less; with a base below 1 pairs turn more, and far positions feel it)
  const double octaves = std::log2((double)c->base);
  int pairs = 0;
  for (int a = 0; a < 3; ++a) {
    const int n = a < c->axes ? c->pairs[a] : 0;
    if (n < 0 || n > c->head_dim / 2 - pairs) return bad("pairs of the axes: none negative, together head_dim / 2 at most");
    for (int i = 0; i < n; ++i) p->turns[pairs + i] = std::exp2(-octaves * i / n) / 6.283185307179586476925;
    pairs += n;
    p->end[a] = pairs;
  }
  p->pairs = pairs;
  return PPLL_OK;
}

namespace {
int check_side(const ppll_queries_keys* v, const RotaryPlan& p, int esz, const char* what) {
  if (!v) { set_error("%s is null", what); return PPLL_ERR_NULL; }
  for (int side = 0; side < 2; ++side) {
    if (!p.heads[side]) continue;
    const void* ptr = side ? v->k : v->q;
    const int64_t ld = side ? v->k_ld : v->q_ld;
    const char* name = side ? "k" : "q";
    if (!ptr) { set_error("%s: %s is null", what, name); return PPLL_ERR_NULL; }
    if (!aligned(ptr, esz)) { set_error("%s: %s is not aligned to its elements", what, name); return PPLL_ERR_SHAPE; }
    if (ld < (int64_t)p.heads[side] * p.hd || ld >= FAR >> 9) { set_error("%s: row stride of %s out of range", what, name); return PPLL_ERR_SHAPE; }
  }
  return PPLL_OK;
}
// Scales of the sides that have heads: all or none of them
int check_scales(const RotaryPlan& p, const float* q, const float* k, bool* norm) {
  const bool has_q = p.heads[0] && q, has_k = p.heads[1] && k;
  if ((p.heads[0] && p.heads[1] && has_q != has_k)) { set_error("one of the two scales is null"); return PPLL_ERR_NULL; }
  if ((has_q && !aligned(q, 4)) || (has_k && !aligned(k, 4))) { set_error("scales are not aligned to 4 bytes"); return PPLL_ERR_SHAPE; }
  *norm = has_q || has_k;
  if (*norm && (!(p.eps > 0.f) || !std::isfinite(p.eps))) { set_error("norm_eps must be positive and finite"); return PPLL_ERR_CONFIG; }
  return PPLL_OK;
}
int check_positions(const RotaryPlan& p, const int32_t* positions) {
  if (!positions) { set_error("positions_dev is null"); return PPLL_ERR_NULL; }
  if (!aligned(positions, 4)) { set_error("positions_dev is not aligned to 4 bytes"); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
RotarySide side_of(const RotaryPlan& p, int side, const ppll_queries_keys* x, const ppll_queries_keys* dy, const ppll_queries_keys* y,
                   const ppll_queries_keys* keep, const float* scale) {
  RotarySide s{};
  if (!p.heads[side]) return s;
  auto of = [&](const ppll_queries_keys* v) { return v ? (side ? v->k : v->q) : nullptr; };
  auto ld = [&](const ppll_queries_keys* v) { return v ? (side ? v->k_ld : v->q_ld) : 0; };
  s.x = of(x); s.dy = of(dy); s.y = of(y); s.keep = of(keep);
  s.x_ld = ld(x); s.dy_ld = ld(dy); s.y_ld = ld(y); s.keep_ld = ld(keep);
  s.scale = scale;
  return s;
}
int check_workspace(const void* ws, size_t have, size_t need) {
  if (!need) return PPLL_OK;
  if (!ws) { set_error("workspace_dev is null"); return PPLL_ERR_NULL; }
  if (!aligned(ws, 16)) { set_error("workspace_dev is not 16-byte aligned"); return PPLL_ERR_WORKSPACE; }
  if (have < need) { set_error("workspace has %zu bytes, %zu needed", have, need); return PPLL_ERR_WORKSPACE; }
  return PPLL_OK;
}
int check_blob(const void* p, const char* what) {
  if (!p) { set_error("%s is null", what); return PPLL_ERR_NULL; }
  if (!aligned(p, 16)) { set_error("%s is not 16-byte aligned", what); return PPLL_ERR_WORKSPACE; }
  return PPLL_OK;
}
int check_steps(int32_t steps) {
  if (steps >= 1 && steps <= ORTHO_STEPS) return PPLL_OK;
  set_error("%d Newton-Schulz steps, 1 to %d are possible", steps, ORTHO_STEPS);
  return PPLL_ERR_CONFIG;
}
}  // namespace
}  // namespace ppll

using namespace ppll;

extern "C" {

int ppll_orthogonalize_workspace_bytes(const ppll_matrix_group* groups, int32_t n_groups, size_t* bytes) {
  OrthoPlan p;
  PPLL_TRY(ortho_plan(groups, n_groups, &p));
  if (!bytes) { set_error("bytes is null"); return PPLL_ERR_NULL; }
  *bytes = (size_t)p.bytes;
  return PPLL_OK;
}

int ppll_orthogonalize(const ppll_matrix_group* groups, int32_t n_groups, int32_t precision, int32_t steps, const void* in_dev, void* out_dev,
                       void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  OrthoPlan p;
  PPLL_TRY(ortho_plan(groups, n_groups, &p));
  if (precision != PPLL_FP32 && precision != PPLL_BF16) { set_error("precision must be PPLL_FP32 or PPLL_BF16"); return PPLL_ERR_CONFIG; }
  PPLL_TRY(check_steps(steps));
  if (!p.n) return PPLL_OK;
  PPLL_TRY(check_blob(in_dev, "in_dev"));
  PPLL_TRY(check_blob(out_dev, "out_dev"));
  PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, (size_t)p.bytes));
  return launch_orthogonalize((hipStream_t)hip_stream, p, precision == PPLL_BF16 ? BF16 : F32, steps, in_dev, out_dev, (char*)workspace_dev);
}

int ppll_muon_step(const ppll_matrix_group* groups, int32_t n_groups, int32_t steps, const float* grads_dev, float* momentum_dev, float* params_dev,
                   void* shadow_dev, float lr, float momentum, int32_t nesterov, float weight_decay, void* workspace_dev, size_t workspace_bytes,
                   void* hip_stream) {
  OrthoPlan p;
  PPLL_TRY(ortho_plan(groups, n_groups, &p));
  PPLL_TRY(check_steps(steps));
  if (!(lr == lr) || !(momentum == momentum) || !(weight_decay == weight_decay)) { set_error("lr, momentum or weight_decay is NaN"); return PPLL_ERR_CONFIG; }
  if (!p.n) return PPLL_OK;
  PPLL_TRY(check_blob(grads_dev, "grads_dev"));
  PPLL_TRY(check_blob(momentum_dev, "momentum_dev"));
  PPLL_TRY(check_blob(params_dev, "params_dev"));
  if (shadow_dev) PPLL_TRY(check_blob(shadow_dev, "shadow_dev"));
  const void* blobs[] = {grads_dev, momentum_dev, params_dev, shadow_dev};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (blobs[i] == blobs[j]) { set_error("gradients, momentum, parameters and shadow need a blob each"); return PPLL_ERR_SHAPE; }
  PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, (size_t)p.bytes));
  return launch_muon((hipStream_t)hip_stream, p, steps, grads_dev, momentum_dev, params_dev, (uint16_t*)shadow_dev, lr, momentum, nesterov != 0,
                     weight_decay, (char*)workspace_dev);
}

int ppll_qk_rotary_forward(const ppll_rotary_config* cfg, const int32_t* positions_dev, const float* q_scale_dev, const float* k_scale_dev,
                           const ppll_queries_keys* in, const ppll_queries_keys* out, const ppll_queries_keys* keep, void* hip_stream) {
  RotaryPlan p;
  PPLL_TRY(rotary_plan(cfg, &p));
  bool norm;
  PPLL_TRY(check_scales(p, q_scale_dev, k_scale_dev, &norm));
  if (!p.rows) return PPLL_OK;
  const int dt = cfg->precision == PPLL_BF16 ? BF16 : F32, esz = (int)dtype_size(dt);
  PPLL_TRY(check_positions(p, positions_dev));
  PPLL_TRY(check_side(in, p, esz, "in"));
  PPLL_TRY(check_side(out, p, esz, "out"));
  if (keep) PPLL_TRY(check_side(keep, p, esz, "keep"));
  return launch_rotary_fwd((hipStream_t)hip_stream, p, dt, positions_dev, side_of(p, 0, in, nullptr, out, keep, norm ? q_scale_dev : nullptr),
                           side_of(p, 1, in, nullptr, out, keep, norm ? k_scale_dev : nullptr));
}

int ppll_qk_rotary_workspace_bytes(const ppll_rotary_config* cfg, size_t* bytes) {
  RotaryPlan p;
  PPLL_TRY(rotary_plan(cfg, &p));
  if (!bytes) { set_error("bytes is null"); return PPLL_ERR_NULL; }
  *bytes = rotary_partial_floats(p.hd) * sizeof(float);
  return PPLL_OK;
}

int ppll_qk_rotary_backward(const ppll_rotary_config* cfg, const int32_t* positions_dev, const float* q_scale_dev, const float* k_scale_dev,
                            const ppll_queries_keys* x, const ppll_queries_keys* dy, const ppll_queries_keys* dx, float* d_q_scale_dev,
                            float* d_k_scale_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  RotaryPlan p;
  PPLL_TRY(rotary_plan(cfg, &p));
  bool norm;
  PPLL_TRY(check_scales(p, q_scale_dev, k_scale_dev, &norm));
  const int dt = cfg->precision == PPLL_BF16 ? BF16 : F32, esz = (int)dtype_size(dt);
  const hipStream_t s = (hipStream_t)hip_stream;
  if (norm) {
    if ((p.heads[0] && !d_q_scale_dev) || (p.heads[1] && !d_k_scale_dev)) { set_error("a scale's gradient is null"); return PPLL_ERR_NULL; }
    if ((p.heads[0] && !aligned(d_q_scale_dev, 4)) || (p.heads[1] && !aligned(d_k_scale_dev, 4))) {
      set_error("scale gradients are not aligned to 4 bytes");
      return PPLL_ERR_SHAPE;
    }
  }
  if (p.rows) {
    PPLL_TRY(check_positions(p, positions_dev));
    PPLL_TRY(check_side(dy, p, esz, "dy"));
    PPLL_TRY(check_side(dx, p, esz, "dx"));
    if (norm) {
      PPLL_TRY(check_side(x, p, esz, "x"));
      PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, rotary_partial_floats(p.hd) * sizeof(float)));
    }
  }
  if (norm && p.heads[0] && p.heads[1]) {
    const uintptr_t dq = (uintptr_t)d_q_scale_dev, dk = (uintptr_t)d_k_scale_dev, bytes = p.hd * sizeof(float);
    if (dq < dk + bytes && dk < dq + bytes) { set_error("the gradients of the two scales share memory"); return PPLL_ERR_SHAPE; }
  }
  int rows = 0;
  if (p.rows)
    PPLL_TRY(launch_rotary_bwd(s, p, dt, positions_dev, side_of(p, 0, norm ? x : nullptr, dy, dx, nullptr, norm ? q_scale_dev : nullptr),
                               side_of(p, 1, norm ? x : nullptr, dy, dx, nullptr, norm ? k_scale_dev : nullptr),
                               norm ? (float*)workspace_dev : nullptr, &rows));
  if (!norm) return PPLL_OK;
  return launch_rotary_scales(s, (const float*)workspace_dev, rows, p.hd, p.heads[0] ? d_q_scale_dev : nullptr,
                              p.heads[1] ? d_k_scale_dev : nullptr);
}

}  // extern "C"
