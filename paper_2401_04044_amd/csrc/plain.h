// Internal: products of the training path on plain row-major matrices (plain.hip), and what their
// launches store.
#pragma once
#include "common.h"
#include "plain_plan.h"

namespace ffsplit {

// bf16 activations of this path: element (t, j) of a [T, ldi] matrix.  Blocks of 16 tokens x 32 neurons, 1 KiB each,
// [token block][neuron block]; in a block the 16-byte chunk c of token r lies at 4 r + (c ^ f(r / 4)), f = 0 2 3 1.
// ldi a multiple of 32; T rounded up to 16, the rows behind the last token hold zeros.
inline __host__ __device__ int64_t blocked_at(int64_t t, int j, int64_t ldi) {
  const int r = (int)(t & 15), c = (j >> 3) & 3;
  return ((t >> 4) * (ldi >> 5) + (j >> 5)) * 512 + (4 * r + (c ^ ((0x78 >> (2 * (r >> 2))) & 3))) * 8 + (j & 7);
}

// D[m, n] = sum_k A(m, k) B(n, k), fp32 accumulation.  ld a multiple of 8 (blocks: 32), pointers 16-byte aligned; KC,
// KC2, BK: the elements from K to the next multiple of 8 are zero in at least one operand and finite in the other.
struct PlainArgs {
  const void* A[2];
  const void* B[2];
  int64_t lda, ldb;
  int64_t a_bytes, b_bytes;   // of each: nothing at or beyond is read
  int a_lay, b_lay;
  int M, N, K;
  // How the second operands take part:
  //   segs = 2   the reduction goes over A[0] B[0] and then A[1] B[1], K elements each
  //   twin       a second product A[0] B[1] beside the first, with its own destination C[1]
  //   EPI_GLU    B[0] gate columns, B[1] up columns, summed in the same tile
  int segs, twin;
  void* C[2];
  int64_t ldc;
  int out_f32, accumulate;
  const float* resid;
  const void* D1;
  const void* D2;
  void* O1;
  void* O2;
  void* H;
  int64_t ldi;
  int n_store;
  // The reduction cut into n_split ranges: fp32 sums [range][plane][M][ldp] that plain_reduce adds
  // (plane 1: up columns, or the twin product)
  float* part;
  int n_split, ldp;
  int group_m;   // row tiles per rasterisation group (set by the launcher)
};

// part: scratch of plain_part_bytes() of this product
int launch_plain(PlainArgs a, int epi, int bf16, float* part, hipStream_t st);
// dst[r][0 .. cols8) = src[r][0 .. cols), zeros behind, of one or two matrices; cols8 = cols rounded up to 8; rows a
// multiple of 8
int launch_pad_rows(const void* src0, const void* src1, void* dst0, void* dst1, int rows, int cols, int bf16, hipStream_t st);

}  // namespace ffsplit
