// Orthogonalised updates: what a call's matrices are, where their intermediates lie in the workspace.  Host arithmetic only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/ppll.h"

namespace ppll {

constexpr int ORTHO_GROUPS = 16;       // groups of a call
constexpr int ORTHO_SIDE = 8192;       // rows and columns of a matrix, at most
constexpr int ORTHO_COUNT = 65535;     // matrices of a group, at most
constexpr int ORTHO_STEPS = 16;        // Newton-Schulz steps, at most
constexpr int NORM_ROWS = 16, NORM_COLS = 256;   // piece of a matrix whose squares one workgroup adds up

constexpr int ORTHO_SMALL_LDS = 160 * 1024 - 256;   // what a workgroup of the small kernel may have (256 bytes are its own)

// A group as the kernels see it.  A matrix is worked on as X [m][n] with m <= n (transposed where rows > cols), padded with zeros to
// mp x np: zero rows and columns stay zero through every product, so no product has a border.  Each intermediate is two planes of fp16,
// one behind the other; offsets in bytes from the start of the workspace, those of matrix i of the group i times its size further.
struct OrthoGroup {
  int64_t offset, stride, ld;          // elements, in the caller's blobs
  int32_t rows, cols, count;
  int32_t m, n, mp, np, tall;
  int32_t small;                       // all steps in one workgroup (then mp and np are multiples of 32, of 64 else)
  int32_t first;                       // place of the group's first matrix among all of the call
  int32_t first_piece;                 // of its pieces among those of all groups
  int64_t x[2], a, b;
  __host__ __device__ int64_t plane_x() const { return (int64_t)mp * np; }      // elements
  __host__ __device__ int64_t plane_a() const { return (int64_t)mp * mp; }
  __host__ __device__ int pieces() const { return ((rows + NORM_ROWS - 1) / NORM_ROWS) * ((cols + NORM_COLS - 1) / NORM_COLS); }
};
// The small kernel's LDS: X and A, in whole tiles of 32 x 32 and at most four of them a side for A; where there is room a second X and a second
// A, and sums of shares of the k where A has few tiles.
struct SmallRoom { int64_t bytes; int32_t two_x, two_a, shares; };
__host__ __device__ inline SmallRoom small_room(const OrthoGroup& g) {
  const int64_t x = 4 * (int64_t)g.mp * (g.np + 8), a = 4 * (int64_t)g.mp * (g.mp + 8);
  SmallRoom r{x + a, 0, 0, 1};
  if (g.mp > 128) { r.bytes = (int64_t)1 << 40; return r; }
  const int shares = g.mp == 32 ? 8 : g.mp == 64 && g.np >= 192 ? 2 : 1, tiles = g.mp == 32 ? 1 : 4;
  if (shares > 1 && r.bytes + shares * tiles * 4096 <= ORTHO_SMALL_LDS) { r.shares = shares; r.bytes += shares * tiles * 4096; }
  if (r.bytes + a <= ORTHO_SMALL_LDS) { r.two_a = 1; r.bytes += a; }
  if (r.bytes + x <= ORTHO_SMALL_LDS) { r.two_x = 1; r.bytes += x; }
  return r;
}
// The products of a step: X X', then b A + c A A, then the product of that and X.
enum { ORTHO_GRAM = 0, ORTHO_POLY = 1, ORTHO_APPLY = 2 };
__host__ __device__ inline int tiles_of_matrix(const OrthoGroup& g, int tile, int phase) {
  if (g.small) return 0;
  const int down = (g.mp + tile - 1) / tile, across = (g.np + tile - 1) / tile;
  return phase <= ORTHO_POLY ? down * (down + 1) / 2 : down * across;      // of a symmetric result those on and under the diagonal
}
// Work items of a launch, `each` of a matrix: those of group k from begin[k] on (a group that has none begins where the next one does).  A kernel
// finds its group from one batch of loads, and what it needs of the group with the next: its arguments lie in memory, where a load takes half a
// microsecond, and a search that reads group by group is a chain of them.
struct OrthoItems { int32_t begin[ORTHO_GROUPS], each[ORTHO_GROUPS]; };
// The tiles of one product.  Workgroup w runs on XCD w % 8.  Each XCD has a run of the tiles, first[x] .. first[x + 1], with an eighth of the work:
// tiles of one matrix, which read the same rows at about the same time, meet in one L2.
struct OrthoProduct {
  int32_t tile;                        // 64 or 128
  int32_t first[9], begin[ORTHO_GROUPS];
  struct Group {
    int32_t each, tiles;               // parts and tiles of a matrix
    int32_t split;                     // parts of a tile, each with a piece of the k and a workgroup of its own
    int32_t tile_of;                   // the group's first tile among those in pieces
    int64_t sums_of;                   // and its first sums, in bytes
  } group[ORTHO_GROUPS];
  int longest() const {                // run of an XCD: a launch has eight times as many workgroups
    int most = 0;
    for (int x = 0; x < 8; ++x) most = first[x + 1] - first[x] > most ? first[x + 1] - first[x] : most;
    return most;
  }
};
struct OrthoPlan {
  OrthoGroup g[ORTHO_GROUPS];          // longest rows first: their tiles take the longest
  int32_t n;                           // groups with a matrix in them
  OrthoProduct product[3];
  OrthoItems pieces, squares, small;   // of the sums of squares, of the normalisation, matrices of the small kernel
  int64_t partials;                    // byte offset of the partial sums of squares, one double a piece
  int64_t shrink;                      // and of a float for each matrix (see k_ortho.hip)
  int64_t sums, arrived;               // of the tiles whose k is in pieces: sums of each piece, and how many of them are there (an int a tile)
  int32_t counters;                    // such tiles, of the product that has the most
  int64_t bytes;
};
static_assert(sizeof(OrthoPlan) <= 3900, "a kernel takes 4 KB of arguments");

// Checks the groups and lays the workspace out.  PPLL_OK, or an error with its text set.
int ortho_plan(const ppll_matrix_group* groups, int32_t n_groups, OrthoPlan* plan);

}  // namespace ppll
