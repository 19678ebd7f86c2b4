// Internal: the products of the training path (plain.hip): what they are, and the choice of the tile and of the ranges that
// each one's reduction is cut into.  Pure host arithmetic.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace ffsplit {

// What a product does with its sums (Z, U: sums of the gate and up columns, S: of the only ones):
//   EPI_OUT   C = S [+ resid] [+ C], in the storage type or fp32
//   EPI_GLU   H = silu(Z) U, and if D1 is set D1 = dH/dU = silu(Z), D2 = dH/dZ = U silu'(Z)
//   EPI_GELU  H = gelu(S), and if D1 is set D1 = gelu'(S)
//   EPI_GRAD  O1 = S * D1 and, with D2, O2 = S * D2
// H, D1, D2, O1, O2 are [M, ldi] matrices (bf16: rows rounded up to 16; H, O1 and O2 in blocks, D1 and D2 row-major) with
// n_store (N rounded up to 8) stored columns; those from N on are stored as zeros, so that a later reduction over
// them in whole 16-byte chunks adds nothing.
enum { EPI_OUT = 0, EPI_GLU = 1, EPI_GELU = 2, EPI_GRAD = 3 };

// How an operand's element (r, k) lies (see plain.hip): row-major with the reduction contiguous, r * ld + k, fetched a
// slab (KC) or two (KC2) at a time; row-major with the rows contiguous, k * ld + r (MC); in blocks of 16 x 32
// with r the token (BK) or k (BM).
enum { LAY_KC = 0, LAY_KC2 = 1, LAY_MC = 2, LAY_BK = 3, LAY_BM = 4 };

inline bool turned(int lay) { return lay == LAY_MC || lay == LAY_BM; }

// A product as the choice sees it: D[M, N] = sum over K; segs, twin: see PlainArgs; two: EPI_GRAD has a second output
struct PlainShape {
  int64_t M, N, K;
  int segs, twin, epi, two;
  int a_turned, b_turned;   // the operand's rows are contiguous
};

// The products of a layer's two passes on T tokens; planes: 2 if gated (of the weights' gradient: if both are wanted).
enum { DENSE_UP = 0, DENSE_DOWN = 1, DENSE_GRAD = 2, DENSE_DX = 3, DENSE_DUP = 4, DENSE_DDOWN = 5, DENSE_PRODUCTS = 6 };
inline PlainShape dense_product(int which, int64_t T, int d, int f, int planes) {
  switch (which) {
    case DENSE_UP: return {T, f, d, 1, 0, planes == 2 ? EPI_GLU : EPI_GELU, 0, 0, 1};   // X [Wg | W1]
    case DENSE_DOWN: return {T, d, f, 1, 0, EPI_OUT, 0, 0, 1};                          // H W2
    case DENSE_GRAD: return {T, f, d, 1, 0, EPI_GRAD, planes == 2, 0, 0};               // dY W2^T
    case DENSE_DX: return {T, d, f, planes, 0, EPI_OUT, 0, 0, 0};                       // dU W1^T + dG Wg^T
    case DENSE_DUP: return {d, f, T, 1, planes == 2, EPI_OUT, 0, 1, 1};                 // X^T [dU | dG]
    default: return {f, d, T, 1, 0, EPI_OUT, 0, 1, 1};                                  // H^T dY
  }
}

enum { PS_128x128 = 0, PS_256x256 = 1, PS_64x64 = 2, PS_256x128 = 3, PS_SHAPES = 4 };
struct PlainPlan { int shape, split; };

// Choice of the tile and of the ranges that the reduction is cut into, by estimated time (us).  Workgroups are counted in
// rounds of `round` on each of 256 CUs, the fullest of which sets the time: t[k - 1] a slab of k workgroups in the
// last round, `fixed` for filling the ring and storing.  (A CU holds two 64x64 workgroups at a time, so that their round of
// three, which is what the timings show, is two of them and one that follows.)  The figures are a least-squares fit to 6800
// timings of 460 products (1 to 6000 rows, the layers' widths from 256 to 5120, operands that no cache holds) on every tile and up to
// 16 ranges; the chosen one takes 1.2 % (bf16) and 0.3 % (fp32) longer than the best on average, 8 % and 2 % in the 95th percentile.
// What they show: an XCD's L2 hands its 32 CUs 64 bytes per channel and clock, 64 KB a us and CU, so that two 128x128 tiles (32 KB
// a slab) take as long as their MFMAs would twice over, and one 256x256 tile as long as its own.
struct ShapeCost { int bm, bn, round; float t[3], fixed; };
static const ShapeCost SHAPE_BF16[PS_SHAPES] = {{128, 128, 2, {0.252f, 0.477f}, 2.5f}, {256, 256, 1, {0.547f}, 4.2f},
                                                {64, 64, 3, {0.144f, 0.276f, 0.449f}, 1.8f}, {256, 128, 1, {0.355f}, 3.0f}};
static const ShapeCost SHAPE_BF16_GATED64 = {64, 128, 2, {0.203f, 0.433f}, 2.1f};
static const ShapeCost SHAPE_F32[PS_SHAPES] = {{128, 128, 2, {0.992f, 1.607f}, 1.7f}, {}, {64, 64, 3, {0.324f, 0.588f, 0.919f}, 0.5f}, {}};
struct ProductCost {
  float layout[3];        // factor of a slab: right operand turned round, neither, both
  float bw, overlap;      // bytes a us, and the share of the traffic's time that comes on top
  float sum, sum_range, sum_bw;   // adding ranges: a launch, each range, bytes a us
};
static const ProductCost COST_BF16 = {{1.0f, 1.07f, 1.11f}, 4.91e6f, 0.34f, 1.7f, 0.12f, 2.29e6f};
static const ProductCost COST_F32 = {{1.0f, 0.99f, 0.99f}, 2.20e6f, 0.22f, 2.0f, 0.10f, 1.70e6f};
constexpr size_t PLAIN_PART_ROOM = (size_t)64 << 20;   // scratch for ranges' sums, at most
constexpr int PLAIN_MAX_SPLIT = 16, PLAIN_MIN_SLABS = 4;   // ranges, and slabs of each

// Scratch for the ranges' sums of a product, whatever is chosen for it: as many ranges as its slabs allow, never less for a
// longer side.
inline size_t plain_part_bytes(const PlainShape& a, int bf16) {
  const int64_t bk = bf16 ? 32 : 16, most = a.segs * ((a.K + bk - 1) / bk) / PLAIN_MIN_SLABS;
  if (most < 2) return 0;
  const size_t bytes = (size_t)(most < PLAIN_MAX_SPLIT ? most : PLAIN_MAX_SPLIT) * (a.epi == EPI_GLU || a.twin ? 2 : 1) * a.M *
                       ((a.N + 7) / 8 * 8) * 4;
  return bytes < PLAIN_PART_ROOM ? bytes : PLAIN_PART_ROOM;
}

inline PlainPlan plain_plan(const PlainShape& a, int bf16) {
  const ProductCost& c = bf16 ? COST_BF16 : COST_F32;
  const int esz = bf16 ? 2 : 4, planes = a.epi == EPI_GLU || a.twin ? 2 : 1;
  const int64_t bk = bf16 ? 32 : 16, slabs = a.segs * ((a.K + bk - 1) / bk), n_store = (a.N + 7) / 8 * 8;
  const float layout = c.layout[a.a_turned ? 2 : a.b_turned ? 0 : 1];
  const int stored = a.epi == EPI_GLU ? 3 : a.epi == EPI_GELU ? 2 : a.epi == EPI_GRAD ? (a.two ? 4 : 2) : planes;
  const float bytes = (float)esz * ((float)a.M * a.K * a.segs + (float)a.N * a.K * (planes > a.segs ? planes : a.segs) +
                                    (float)stored * a.M * a.N);
  PlainPlan best = {PS_128x128, 1};
  float best_t = 1e30f;
  for (int s = 0; s < PS_SHAPES; ++s) {
    const ShapeCost& q = !bf16 ? SHAPE_F32[s] : s == PS_64x64 && a.epi == EPI_GLU ? SHAPE_BF16_GATED64 : SHAPE_BF16[s];
    if (q.bm == 0) continue;
    const int bn = a.epi == EPI_GLU ? q.bn / 2 : q.bn;
    const int64_t tiles = ((a.M + q.bm - 1) / q.bm) * ((n_store + bn - 1) / bn) * (a.twin ? 2 : 1);
    for (int split = 1; split <= PLAIN_MAX_SPLIT; split += split < 4 ? 1 : split < 8 ? 2 : 4) {
      const size_t part = (size_t)split * planes * a.M * n_store * 4;
      if (split > 1 && (part > PLAIN_PART_ROOM || tiles * split > 1024 || slabs / split < PLAIN_MIN_SLABS)) break;
      const int n = (int)((slabs + split - 1) / split);
      const int64_t load = (tiles * split + 255) / 256, full = load / q.round, rest = load % q.round;
      float t = (float)full * (n * q.t[q.round - 1] * layout + q.fixed);
      if (rest) t += n * q.t[rest - 1] * layout + q.fixed;
      t += c.overlap * bytes / c.bw;
      if (t < bytes / c.bw) t = bytes / c.bw;
      if (split > 1) t += c.sum + c.sum_range * split + (float)part / c.sum_bw;
      if (t < best_t) { best_t = t; best.shape = s; best.split = split; }
    }
  }
  return best;
}

}  // namespace ffsplit
