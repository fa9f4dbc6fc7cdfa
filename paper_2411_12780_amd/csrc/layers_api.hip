// C entry points of rows of 8 bits, the linear layer on them and group norm (include/ppll.h): argument checks on the host, then the launches.
#include <cmath>

#include "bytes.h"

namespace ppll {

namespace {
constexpr int MOST_ROWS = 1 << 30;
// Tiles of 128 x 128 of a product.  A launch has under 2^32 threads: both gradients have 256 a tile, the forward pass leaves the kernel with 512 out where
// they are too many.
constexpr int64_t MOST_TILES = 1 << 23;

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
int esz(int32_t precision) { return precision == PPLL_BF16 ? 2 : 4; }
int type_of(int32_t precision) { return precision == PPLL_BF16 ? BF16 : F32; }

int check_precision(int32_t p) {
  if (p == PPLL_FP32 || p == PPLL_BF16) return PPLL_OK;
  set_error("precision must be PPLL_FP32 or PPLL_BF16");
  return PPLL_ERR_CONFIG;
}
int check_rows(const ppll_rows* r, int cols, int32_t precision, const char* what) {
  if (!r || !r->p) { set_error("%s is null", what); return PPLL_ERR_NULL; }
  if (!aligned(r->p, esz(precision))) { set_error("%s is not aligned to its elements", what); return PPLL_ERR_SHAPE; }
  if (r->ld < cols || r->ld >= ROW_LD) { set_error("row stride of %s out of range", what); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
int check_maybe(const ppll_rows* r, int cols, int32_t precision, const char* what) { return r ? check_rows(r, cols, precision, what) : PPLL_OK; }
// Buffers from one place, but where they may be one and the same
int check_apart(const ppll_rows* a, const ppll_rows* b, bool may_be_one, const char* what) {
  if (!a || !b || a->p != b->p || (may_be_one && a->ld == b->ld)) return PPLL_OK;
  set_error("%s share memory", what);
  return PPLL_ERR_SHAPE;
}
// rows of a linear layer, pixels of a map
int check_map(const ppll_rows* r, int cols, int32_t precision, const char* what) {
  PPLL_TRY(check_rows(r, cols, precision, what));
  if (r->ld > MAP_LD) { set_error("rows of %s more than 2^20 elements apart", what); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
int check_maybe_map(const ppll_rows* r, int cols, int32_t precision, const char* what) { return r ? check_map(r, cols, precision, what) : PPLL_OK; }
int check_bytes(const ppll_byte_rows* r, int cols, const char* what) {
  if (!r || !r->q || !r->e) { set_error("%s is null", what); return PPLL_ERR_NULL; }
  if (!aligned(r->q, 16)) { set_error("%s is not 16-byte aligned", what); return PPLL_ERR_SHAPE; }
  if (r->ld < cols || r->ld % 16 || r->ld > BYTE_LD) { set_error("row stride of %s: a multiple of 16 that holds the columns, 2^20 at most", what); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
int check_floats(const float* p, const char* what) {
  if (!p) { set_error("%s is null", what); return PPLL_ERR_NULL; }
  if (!aligned(p, 4)) { set_error("%s is not aligned to 4 bytes", what); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
int check_workspace(const void* ws, size_t have, size_t need) {
  if (!need) return PPLL_OK;
  if (!ws) { set_error("workspace_dev is null"); return PPLL_ERR_NULL; }
  if (!aligned(ws, 16)) { set_error("workspace_dev is not 16-byte aligned"); return PPLL_ERR_WORKSPACE; }
  if (have < need) { set_error("workspace has %zu bytes, %zu needed", have, need); return PPLL_ERR_WORKSPACE; }
  return PPLL_OK;
}
int check_matrix(int32_t rows, int32_t most_rows, int32_t cols, int32_t least_cols) {
  if (rows < 0 || rows > most_rows) { set_error("%d rows outside 0..%d", rows, most_rows); return PPLL_ERR_SHAPE; }
  if (cols < least_cols || cols > BYTE_COLS) { set_error("%d columns outside %d..%d", cols, least_cols, BYTE_COLS); return PPLL_ERR_SHAPE; }
  return PPLL_OK;
}
int64_t tiles(int64_t a, int64_t b) { return ((a + 127) / 128) * ((b + 127) / 128); }
ppll_rows given(const ppll_rows* r) { return r ? *r : ppll_rows{nullptr, 0}; }
ppll_byte_rows given(const ppll_byte_rows* r) { return r ? *r : ppll_byte_rows{nullptr, nullptr, 0}; }

int linear_of(const ppll_byte_linear_config* c, ByteLinear* l) {
  if (!c) { set_error("byte linear config is null"); return PPLL_ERR_NULL; }
  auto bad = [](const char* what) { set_error("byte linear config: %s", what); return PPLL_ERR_CONFIG; };
  if (c->struct_size != sizeof *c) return bad("struct_size");
  PPLL_TRY(check_precision(c->precision));
  if (c->rows < 0 || c->rows > MOST_ROWS) return bad("rows outside 0..2^30");
  if (c->in_dim < 1 || c->in_dim > BYTE_COLS || c->out_dim < 1 || c->out_dim > BYTE_COLS) return bad("in_dim, out_dim outside 1..65536");
  if (c->activation != PPLL_ACT_NONE && c->activation != PPLL_ACT_GELU) return bad("activation must be PPLL_ACT_NONE or PPLL_ACT_GELU");
  if (tiles(c->rows, c->in_dim) > MOST_TILES || tiles(c->rows, c->out_dim) > MOST_TILES) return bad("rows x in_dim or rows x out_dim is more than a launch holds");
  *l = {type_of(c->precision), c->rows, c->in_dim, c->out_dim, c->activation};
  return PPLL_OK;
}
int norm_of(const ppll_group_norm_config* c, GroupNorm* g) {
  if (!c) { set_error("group norm config is null"); return PPLL_ERR_NULL; }
  auto bad = [](const char* what) { set_error("group norm config: %s", what); return PPLL_ERR_CONFIG; };
  if (c->struct_size != sizeof *c) return bad("struct_size");
  PPLL_TRY(check_precision(c->precision));
  if (c->images < 0 || c->pixels < 1 || (int64_t)c->images * c->pixels > MOST_ROWS) return bad("images >= 0, pixels >= 1 and images * pixels <= 2^30 required");
  if (c->channels < 1 || c->channels > 4096) return bad("channels outside 1..4096");
  if (c->groups < 1 || c->channels % c->groups) return bad("groups must divide channels");
  if (c->activation < PPLL_ACT_NONE || c->activation > PPLL_ACT_GELU) return bad("activation must be one of PPLL_ACT_...");
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return bad("eps must be positive and finite");
  *g = {type_of(c->precision), c->images, c->pixels, c->channels, c->groups, c->activation, c->eps};
  return PPLL_OK;
}
}  // namespace
}  // namespace ppll

using namespace ppll;

extern "C" {

int ppll_byte_rows_pack(int32_t precision, int32_t rows, int32_t cols, const ppll_rows* in, const ppll_byte_rows* out, void* hip_stream) {
  PPLL_TRY(check_precision(precision));
  PPLL_TRY(check_matrix(rows, MOST_ROWS, cols, 1));
  if (!rows) return PPLL_OK;
  PPLL_TRY(check_rows(in, cols, precision, "in"));
  PPLL_TRY(check_bytes(out, cols, "out"));
  return launch_byte_rows_pack((hipStream_t)hip_stream, type_of(precision), rows, cols, *in, *out);
}

int ppll_byte_rows_pack_columns(int32_t precision, int32_t rows, int32_t cols, const ppll_rows* in, const ppll_byte_rows* out, void* hip_stream) {
  PPLL_TRY(check_precision(precision));
  PPLL_TRY(check_matrix(rows, BYTE_COLS, cols, 0));
  if (!rows) { set_error("no rows: columns of no values"); return PPLL_ERR_SHAPE; }
  if (!cols) return PPLL_OK;
  PPLL_TRY(check_rows(in, cols, precision, "in"));
  PPLL_TRY(check_bytes(out, rows, "out"));
  return launch_byte_rows_pack_columns((hipStream_t)hip_stream, type_of(precision), rows, cols, *in, *out);
}

int ppll_byte_rows_unpack(int32_t precision, int32_t rows, int32_t cols, const ppll_byte_rows* in, const ppll_rows* out, void* hip_stream) {
  PPLL_TRY(check_precision(precision));
  PPLL_TRY(check_matrix(rows, MOST_ROWS, cols, 1));
  if (!rows) return PPLL_OK;
  PPLL_TRY(check_bytes(in, cols, "in"));
  PPLL_TRY(check_rows(out, cols, precision, "out"));
  return launch_byte_rows_unpack((hipStream_t)hip_stream, type_of(precision), rows, cols, *in, *out);
}

int ppll_byte_linear_forward(const ppll_byte_linear_config* cfg, const ppll_byte_rows* x, const ppll_byte_rows* w, const float* bias_dev,
                             const ppll_rows* residual, const ppll_rows* y, const ppll_rows* slope, void* hip_stream) {
  ByteLinear l;
  PPLL_TRY(linear_of(cfg, &l));
  if (slope && l.activation != PPLL_ACT_GELU) { set_error("slope goes with PPLL_ACT_GELU"); return PPLL_ERR_CONFIG; }
  if (!l.rows) return PPLL_OK;
  PPLL_TRY(check_bytes(x, l.in, "x"));
  PPLL_TRY(check_bytes(w, l.in, "w"));
  if (bias_dev) PPLL_TRY(check_floats(bias_dev, "bias_dev"));
  PPLL_TRY(check_maybe_map(residual, l.out, cfg->precision, "residual"));
  PPLL_TRY(check_map(y, l.out, cfg->precision, "y"));
  PPLL_TRY(check_maybe_map(slope, l.out, cfg->precision, "slope"));
  PPLL_TRY(check_apart(y, residual, true, "y and residual of other strides"));
  PPLL_TRY(check_apart(y, slope, false, "y and slope"));
  PPLL_TRY(check_apart(slope, residual, false, "slope and residual"));
  return launch_byte_linear_fwd((hipStream_t)hip_stream, l, *x, *w, bias_dev, given(residual), *y, given(slope));
}

int ppll_byte_linear_workspace_bytes(const ppll_byte_linear_config* cfg, size_t* bytes) {
  ByteLinear l;
  PPLL_TRY(linear_of(cfg, &l));
  if (!bytes) { set_error("bytes is null"); return PPLL_ERR_NULL; }
  *bytes = byte_linear_workspace(l);
  return PPLL_OK;
}

int ppll_byte_linear_backward(const ppll_byte_linear_config* cfg, const ppll_byte_rows* x, const ppll_byte_rows* w, const ppll_rows* dy,
                              const ppll_rows* gate, const ppll_rows* dx, float* dw_dev, float* db_dev, void* workspace_dev, size_t workspace_bytes,
                              void* hip_stream) {
  ByteLinear l;
  PPLL_TRY(linear_of(cfg, &l));
  if (dw_dev) PPLL_TRY(check_floats(dw_dev, "dw_dev"));
  if (db_dev) PPLL_TRY(check_floats(db_dev, "db_dev"));
  if (!dx && gate) { set_error("gate goes with dx"); return PPLL_ERR_NULL; }
  if (l.rows) {
    if (!dx && !dw_dev && !db_dev) return PPLL_OK;
    PPLL_TRY(check_map(dy, l.out, cfg->precision, "dy"));
    if (dx) {
      PPLL_TRY(check_map(dx, l.in, cfg->precision, "dx"));
      PPLL_TRY(check_maybe_map(gate, l.in, cfg->precision, "gate"));
      PPLL_TRY(check_bytes(w, l.in, "w"));
    }
    if (dw_dev) PPLL_TRY(check_bytes(x, l.in, "x"));
    PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, byte_linear_workspace(l)));
    PPLL_TRY(check_apart(dx, gate, true, "dx and gate of other strides"));
    PPLL_TRY(check_apart(dx, dy, false, "dx and dy"));
  }
  return launch_byte_linear_bwd((hipStream_t)hip_stream, l, given(x), given(w), given(dy), given(gate), given(dx), dw_dev, db_dev, (char*)workspace_dev);
}

int ppll_group_norm_workspace_bytes(const ppll_group_norm_config* cfg, size_t* bytes) {
  GroupNorm g;
  PPLL_TRY(norm_of(cfg, &g));
  if (!bytes) { set_error("bytes is null"); return PPLL_ERR_NULL; }
  *bytes = group_norm_workspace(g);
  return PPLL_OK;
}

int ppll_group_norm_forward(const ppll_group_norm_config* cfg, const ppll_rows* x, const float* scale_dev, const float* shift_dev, const ppll_rows* residual,
                            const ppll_rows* y, float* stats_dev, const ppll_byte_rows* keep, void* workspace_dev, size_t workspace_bytes,
                            void* hip_stream) {
  GroupNorm g;
  PPLL_TRY(norm_of(cfg, &g));
  if (!g.images) return PPLL_OK;
  PPLL_TRY(check_map(x, g.channels, cfg->precision, "x"));
  PPLL_TRY(check_floats(scale_dev, "scale_dev"));
  PPLL_TRY(check_floats(shift_dev, "shift_dev"));
  PPLL_TRY(check_maybe_map(residual, g.channels, cfg->precision, "residual"));
  PPLL_TRY(check_map(y, g.channels, cfg->precision, "y"));
  if (stats_dev) PPLL_TRY(check_floats(stats_dev, "stats_dev"));
  if (keep) PPLL_TRY(check_bytes(keep, g.channels, "keep"));
  PPLL_TRY(check_apart(y, x, true, "y and x of other strides"));
  PPLL_TRY(check_apart(y, residual, true, "y and residual of other strides"));
  PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, group_norm_workspace(g)));
  return launch_group_norm_fwd((hipStream_t)hip_stream, g, *x, scale_dev, shift_dev, given(residual), *y, stats_dev, given(keep), (char*)workspace_dev);
}

int ppll_group_norm_backward(const ppll_group_norm_config* cfg, const ppll_rows* x, const ppll_byte_rows* x_bytes, const float* stats_dev,
                             const float* scale_dev, const float* shift_dev, const ppll_rows* residual, const ppll_rows* y, const ppll_rows* dy,
                             const ppll_rows* dx, const ppll_rows* d_residual, float* d_scale_dev, float* d_shift_dev, void* workspace_dev,
                             size_t workspace_bytes, void* hip_stream) {
  GroupNorm g;
  PPLL_TRY(norm_of(cfg, &g));
  PPLL_TRY(check_floats(d_scale_dev, "d_scale_dev"));
  PPLL_TRY(check_floats(d_shift_dev, "d_shift_dev"));
  const bool relu = g.activation == PPLL_ACT_RELU, curved = g.activation == PPLL_ACT_SILU || g.activation == PPLL_ACT_GELU;
  if (g.images) {
    if (x && x_bytes) { set_error("x is given twice"); return PPLL_ERR_SHAPE; }
    if (x_bytes) PPLL_TRY(check_bytes(x_bytes, g.channels, "x_bytes"));
    else PPLL_TRY(check_map(x, g.channels, cfg->precision, "x"));
    PPLL_TRY(check_floats(stats_dev, "stats_dev"));
    PPLL_TRY(check_floats(scale_dev, "scale_dev"));
    PPLL_TRY(check_floats(shift_dev, "shift_dev"));
    if (curved) PPLL_TRY(check_maybe_map(residual, g.channels, cfg->precision, "residual"));
    if (relu) PPLL_TRY(check_map(y, g.channels, cfg->precision, "y"));
    PPLL_TRY(check_map(dy, g.channels, cfg->precision, "dy"));
    PPLL_TRY(check_map(dx, g.channels, cfg->precision, "dx"));
    PPLL_TRY(check_maybe_map(d_residual, g.channels, cfg->precision, "d_residual"));
    PPLL_TRY(check_apart(dx, d_residual, false, "dx and d_residual"));
    PPLL_TRY(check_apart(dx, dy, true, "dx and dy of other strides"));
    PPLL_TRY(check_apart(d_residual, dy, true, "d_residual and dy of other strides"));
    if (!x_bytes) PPLL_TRY(check_apart(dx, x, false, "dx and x"));
    if (!x_bytes) PPLL_TRY(check_apart(d_residual, x, false, "d_residual and x"));
    PPLL_TRY(check_workspace(workspace_dev, workspace_bytes, group_norm_workspace(g)));
  }
  const uintptr_t a = (uintptr_t)d_scale_dev, b = (uintptr_t)d_shift_dev, bytes = g.channels * sizeof(float);
  if (a < b + bytes && b < a + bytes) { set_error("the gradients of scale and shift share memory"); return PPLL_ERR_SHAPE; }
  return launch_group_norm_bwd((hipStream_t)hip_stream, g, given(x), given(x_bytes), stats_dev, scale_dev, shift_dev, curved ? given(residual) : ppll_rows{},
                               relu ? given(y) : ppll_rows{}, given(dy), given(dx), given(d_residual), d_scale_dev, d_shift_dev, (char*)workspace_dev);
}

}  // extern "C"
