// How the products are cut into tiles and shares of the contraction, and the workspace that follows from it.  Plain C++: launches, sizes and host
// tests take the same structures.
#pragma once
#include <cstddef>

namespace hpf {

constexpr int round_up64(int v) { return (v + 63) / 64 * 64; }
constexpr int slab_row(int n) { return (n + 7) & ~7; }       // rows of partial sums start on 32 bytes
constexpr size_t linear_align(size_t v) { return (v + 255) / 256 * 256; }

// How a bf16 product is cut (M x K x N, us):
// - 256 x 256 tiles where there are 160 (2560 x 4096 x 4096, 160 tiles: 84, with 128 x 128 ones 97; 2048 x 4096 x 4096, 128 tiles: 78 and 67);
// - 128 x 128 ones where there are 256 (2048 x 4096 x 2048, 256 tiles: 52, with 64 x 64 ones 61; 1536 x 4096 x 1536, 144 tiles: 42 and 37);
// - 64 x 64 ones, two work-groups of four stages per CU, with the contraction split until there is a work-group per CU;
// - k_linear_few for up to 16 rows of small weights, where a launch less counts most.  It reads K N weights once and x again for every 16
//   columns, K N M / 16, and takes up to 1.25 * 2^25 of both (4096 x 4096: 13.2 to 11.9 for 1 to 16 rows, with 64 x 64 tiles 14.5 to 13.9;
//   4096 x 8192: 13.0 and 14.6 for one row, 17.4 and 15.1 for 16; 4096 x 32000: 40 and 37, 58 and 37).
enum : int { CUT_LARGE, CUT_TILES, CUT_SPLIT, CUT_FEW };
struct Cut {
  int kind, splits, steps;      // steps (of 64, CUT_FEW: 32) per share
  unsigned rows, cols;          // tiles
};
// The contraction counts in whole steps of 64: an operand is read in place, K long, or from a copy whose rows are padded to 64, and either way the
// shares, and with them the workspace and the order of the sums, are the same.  (In steps of 32, K = 89760 has 2805 of them in place
// and 2806 padded: 85 shares of 33 and 83 of 34.)
inline Cut cut_of(int M, int N, int K, bool rows) {      // rows: of a ROWS product
  auto tiles = [&](int bm, int bn) { return (long)((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  Cut c;
  const int Kp = round_up64(K);
  const bool few = M <= 16 && !rows && (long)Kp * N * (16 + M) <= 20l << 25;
  c.kind = few ? CUT_FEW : tiles(256, 256) >= 160 ? CUT_LARGE : tiles(128, 128) >= 256 ? CUT_TILES : CUT_SPLIT;
  const int bm = c.kind == CUT_FEW ? 16 : c.kind == CUT_LARGE ? 256 : c.kind == CUT_TILES ? 128 : 64, bn = bm;
  c.rows = (unsigned)((M + bm - 1) / bm);
  c.cols = (unsigned)((N + bn - 1) / bn);
  const int k = Kp / (c.kind == CUT_FEW ? 32 : 64), least = c.kind == CUT_FEW ? 32 : 8;
  long want = c.kind == CUT_SPLIT || c.kind == CUT_FEW ? 256 / ((long)c.rows * c.cols) : 1;
  if (want > k / least) want = k / least;
  if (want < 1) want = 1;
  c.steps = (int)((k + want - 1) / want);
  c.splits = (k + c.steps - 1) / c.steps;
  return c;
}
// partial sums of a split product, [splits][M][slab_row(N)]
inline size_t slab_bytes(const Cut& c, int M, int N) {
  return c.splits > 1 ? linear_align((size_t)c.splits * M * slab_row(N) * sizeof(float)) : 0;
}

// Rows in a work-group of k_linear_rows: 64, or 16 while that gives no CU two work-groups (gradients of 1021 x 2049 x 1000: 47.8 us
// with 64, 43.6 with 16; of 8192 x 4096 x 4096, where 64 it is, no difference, but a quarter of the sums)
inline int group_of(int M, int width) { return (long)((M + 63) / 64) * ((width + 511) / 512) >= 512 ? 64 : 16; }

// The cuts of a call's products and its workspace.
// Forward: x [M][Kp] | shares of a split product
struct ForwardSpace {
  Cut y;
  size_t slabs, bytes;
  ForwardSpace(int M, int K, int N) : y(cut_of(M, N, K, false)) {
    slabs = linear_align((size_t)M * round_up64(K) * 2);
    bytes = slabs + slab_bytes(y, M, N);
  }
};
// Backward: dz [M][Np] | x [M][Kp] | sums of groups of rows [groups][N] | shares of a split product
struct BackwardSpace {
  Cut dx, dw;
  size_t dz, x, sums, slabs, bytes;
  int group, groups;            // rows of a sum; sums
  BackwardSpace(int M, int K, int N) : dx(cut_of(M, K, N, false)), dw(cut_of(K, N, M, true)) {
    const size_t Kp = round_up64(K), Np = round_up64(N);
    dz = 0;
    group = group_of(M, (int)Np);
    groups = (M + group - 1) / group;
    x = linear_align((size_t)M * Np * 2);
    sums = x + linear_align((size_t)M * Kp * 2);
    slabs = sums + linear_align((size_t)groups * N * 4);
    const size_t d = slab_bytes(dx, M, K), w = slab_bytes(dw, K, N);
    bytes = slabs + (d > w ? d : w);
  }
};

}  // namespace hpf
