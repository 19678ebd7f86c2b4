// Products on plain row-major matrices in any orientation, with the store steps of the training path
// (plain.h), gfx950 only.
//
//   D[M, N] = sum_k A(m, k) B(n, k)
//
// A layer's forward and backward pass read the same matrices along different axes (X W1, dY W2^T,
// X^T dU, ...), and its weights change every step: a copy re-tiled for each use would cost 10 to 20 %
// of the products' time.  So one kernel takes each operand as it lies in memory:
//   KC   row-major, reduction contiguous, 64 bytes of a row per slab.  The 16-byte chunk c of row r sits in LDS at
//        4 r + (c ^ f(r / 4)), f = 0 2 3 1: the lane groups that a 16-byte LDS read serves at a time (lanes
//        0-3, 12-15, 20-27 and so on) then fall into different banks.
//   KC2  the same fetched two slabs at a time, 128 bytes of a row: half the requests.  (64 bytes a row cost the
//        memory pipeline up to a third of its rate: 4096 x 4096 x 22016 with both operands KC 614 us, with
//        contiguous ones 460, with one of them KC2 and the other contiguous 510.)  The ring needs one more pair, so that
//        LDS has room for only one operand of a product fetched this way.
//   MC   row-major, rows contiguous.  bf16 fragments are turned round on the way out of LDS (ds_read_b64_tr_b16:
//        lane j of 16 gets column j of four 16-column rows), fp32 ones are read element by element.  Pieces of the
//        LDS rows are exchanged by an XOR with the row number, so that the eight rows read at a time fall into
//        different banks.  As fast as contiguous loads.
//   BK, BM  this path's own activations in bf16 (H, dU, dG), stored in blocks of 16 tokens x 32 neurons (1 KiB)
//        whose chunks lie as KC has them in LDS: every load is a contiguous 1 KiB, whether the reduction goes
//        over the neurons (BK) or over the tokens (BM, turned round like MC).
// All go from global memory straight into rings of LDS stages (buffer loads with LDS destination).
// The buffers' bounds are exact: what lies behind an operand's end reads as zero, which is how a
// reduction that ends inside a slab and rows behind the last are handled, without masks in the loop.
#include "plain_epi.h"
#include "wave.h"
#include <atomic>
#include <algorithm>
#include <math.h>
#include <type_traits>

namespace ffsplit {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
template <typename T>
using lds_ptr = __attribute__((address_space(3))) T*;

union Frag {
  u32x4_t u;
  u32x2_t h[2];
  bf16x8_t v;
  f32x4_t f;
};

__device__ __forceinline__ uint32_t kc_swizzle(uint32_t r4) { return (0x78u >> (2 * (r4 & 3))) & 3; }   // 0 2 3 1

constexpr uint32_t NOWHERE = 0x80000000u;   // beyond every resource's end
constexpr uint32_t FAR = 1u << 30;          // a resource is set anew before a scalar offset passes this
// 16 bytes per lane from the buffer r at offset + soff (zeros beyond its end) straight into LDS, lane l to
// dst + 16 l; r, dst and soff in scalar registers.  In assembly because the compiler, when it sees a load
// into LDS, waits for all of them before every turned-round LDS read; here the counts are kept by hand.
// (dst goes into m0, which the compiler writes: it then knows what m0 holds.  The s_nop is the distance that a load needs
// from that write.)
__device__ __forceinline__ void load_to_lds(const u32x4_t& r, uint32_t dst, uint32_t offset, uint32_t soff) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, %3 offen lds"
               :
               : "v"(offset), "s"(r), "{m0}"(dst), "s"(soff)
               : "memory");
}
// A buffer resource for what lies from base on, `left` bytes, in scalar registers.  (The s_nop keeps the
// distance that a load needs from the v_readfirstlane that wrote them.)
__device__ __forceinline__ u32x4_t resource(const char* base, int64_t left) {
  const uint64_t b = (uint64_t)base;
  u32x4_t r;
  r[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  r[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32));
  const int hi = __builtin_amdgcn_readfirstlane((int)(left >> 31)), lo = __builtin_amdgcn_readfirstlane((int)left);
  r[2] = hi > 0 ? 0x7fffffffu : hi < 0 ? 0u : (uint32_t)lo;
  r[3] = 0x00027000u;
  asm volatile("s_nop 4" : "+s"(r));
  return r;
}
__device__ __forceinline__ uint32_t lds_offset(const char* q) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)q;
}

// One operand's side of the tile: R rows of one matrix.  Blocks of 1 KiB, one load instruction each: KC 16
// rows x 64 bytes; KC2 8 rows x 128 bytes; MC 1024 / P k-rows x P bytes, P the length of an LDS row (256 bytes, or the
// whole side if that is shorter); BK, BM a stored block.
template <typename T, int R, int LAY>
struct Side {
  static constexpr int EPC = 16 / sizeof(T);          // elements per 16-byte chunk
  static constexpr int BK = 4 * EPC;                  // depth of a slab
  static constexpr bool TURNED = LAY == LAY_MC || LAY == LAY_BM;
  static constexpr int UNIT = LAY == LAY_KC2 ? 2 : 1; // slabs fetched together
  static constexpr int UNIT_BYTES = UNIT * R * 64;
  static constexpr int P = R * (int)sizeof(T) < 256 ? R * (int)sizeof(T) : 256;
  static constexpr int SUB = P / (int)sizeof(T);      // MC: rows of the operand in one sub-block
  static constexpr int KPB = 1024 / P;                // MC: k-rows of one load
  static constexpr int BPS = BK / KPB;                // MC: loads of one sub-block
  static_assert(LAY != LAY_MC || P == 256 || P == 128, "the exchange of pieces is written for these");
  static_assert((LAY != LAY_BK && LAY != LAY_BM) || sizeof(T) == 2, "blocks are bf16");

  // MC: XOR on the chunk number within LDS row k.  bf16: a read serves rows 8 g + 0..3 of two groups g
  // with 32 bytes of each; fp32: rows 4 g + t of four groups with 64 bytes.
  static __device__ __forceinline__ uint32_t mc_swizzle(uint32_t k) {
    if (sizeof(T) == 2) {
      if (P == 256) return 2 * ((k & 3) + 4 * ((k >> 3) & 1));
      return 2 * (((k >> 1) & 1) + 2 * ((k >> 3) & 1));
    }
    if (P == 256) return 4 * ((k >> 2) & 3);
    return 4 * ((k >> 2) & 1);
  }
  // where the tile begins in the matrix (r0: its first row, a multiple of 32), and what a unit advances by, in bytes
  static __device__ __forceinline__ int64_t origin(int r0, int64_t ld) {
    if (LAY == LAY_MC) return (int64_t)r0 * (int)sizeof(T);
    if (LAY == LAY_BM) return (int64_t)(r0 / 32) * 1024;
    return (int64_t)r0 * ld * (int)sizeof(T);
  }
  static __device__ __forceinline__ uint32_t step(uint32_t ld) {
    return TURNED ? BK * ld * (uint32_t)sizeof(T) : LAY == LAY_BK ? 1024u : 64u * UNIT;
  }
  // byte offset of the lane's 16 bytes of block b of a unit; k: the first element of the reduction that they hold
  // (not TURNED)
  static __device__ __forceinline__ uint32_t source(int b, int lane, uint32_t ld, int* k) {
    if (LAY == LAY_MC) {
      constexpr int CPR = P / 16;   // chunks of an LDS row
      const uint32_t sub = b / BPS, kr = (b % BPS) * KPB + lane / CPR;
      const uint32_t c = (lane % CPR) ^ mc_swizzle(kr);
      return kr * ld * (uint32_t)sizeof(T) + sub * P + c * 16;
    }
    if (LAY == LAY_BM) return (b & 1) * 16 * ld * (uint32_t)sizeof(T) + (b >> 1) * 1024 + lane * 16;
    if (LAY == LAY_KC2) {
      const uint32_t r = (uint32_t)b * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
      *k = (int)c * EPC;
      return r * ld * (uint32_t)sizeof(T) + c * 16;
    }
    const uint32_t r = lane >> 2, c = (lane & 3) ^ kc_swizzle(r >> 2);
    *k = (int)c * EPC;
    if (LAY == LAY_BK) return (uint32_t)b * 16 * ld * (uint32_t)sizeof(T) + lane * 16;
    return ((uint32_t)b * 16 + r) * ld * (uint32_t)sizeof(T) + c * 16;
  }
  // where a wavefront's fragments begin, from the matrix's beginning in a stage: rows l & 15 of its first 16-row
  // tile x0 (a multiple of the number of its tiles), elements 8 (l >> 4) .. + 7 (fp32: 4 (l >> 4) .. + 3) of the slab
  static constexpr int TPS = SUB / 16;               // MC: tiles of a sub-block
  static constexpr uint32_t TB = 16 * sizeof(T);     // MC: bytes of a tile's piece of an LDS row
  static __device__ __forceinline__ uint32_t first(int x0, int lane) {
    const uint32_t g = lane >> 4, j = lane & 15;
    if (LAY == LAY_KC || LAY == LAY_BK) return x0 * 1024 + j * 64 + ((g ^ kc_swizzle(j >> 2)) * 16);
    if (LAY == LAY_KC2) return x0 * 2048 + j * 128 + ((g ^ ((j >> 1) & 7)) * 16);
    if (LAY == LAY_BM) {
      const uint32_t r = (8 * g + (j >> 2)) & 15;
      return (x0 / 2) * 2048 + (g >> 1) * 1024 + r * 64 + ((((j & 3) >> 1) ^ kc_swizzle(r >> 2)) * 16) + (j & 1) * 8;
    }
    uint32_t part;
    if (sizeof(T) == 2) {
      const uint32_t k = 8 * g + (j >> 2);
      part = k * P + ((((j & 3) >> 1) ^ mc_swizzle(k)) * 16) + (j & 1) * 8;
    } else {
      const uint32_t k = 4 * g;
      part = k * P + (((j >> 2) ^ mc_swizzle(k)) * 16) + (j & 3) * 4;
    }
    return (x0 / TPS) * (BK * P) + (part ^ ((uint32_t)(x0 % TPS) * TB));
  }
  // fragment of the tile x0 + i; at: that beginning in LDS; half: KC2, the slab of the pair
  static __device__ __forceinline__ void read(Frag& f, uint32_t at, int i, int half) {
    if (!TURNED) {
      f.u = *(lds_ptr<const u32x4_t>)(uintptr_t)((LAY == LAY_KC2 ? at ^ (half * 64u) : at) + i * 1024 * UNIT);
      return;
    }
    if constexpr (sizeof(T) == 2) {
      // (BM: four tokens on lie four rows down, with the pairs of chunks exchanged)
      const uint32_t a0 = LAY == LAY_BM ? (at ^ ((i & 1) * 32u)) + (i / 2) * 2048 : (at ^ ((uint32_t)(i % TPS) * TB)) + (i / TPS) * (BK * P);
      const uint32_t a1 = LAY == LAY_BM ? (at ^ ((i & 1) * 32u) ^ 288u) + (i / 2) * 2048 : a0 + 4 * P;
      f.h[0] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr<s16x4_t>)(uintptr_t)a0));
      f.h[1] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr<s16x4_t>)(uintptr_t)a1));
    } else {
      const uint32_t a = (at ^ ((uint32_t)(i % TPS) * TB)) + (i / TPS) * (BK * P);
#pragma unroll
      for (int t = 0; t < 4; ++t) f.f[t] = *(lds_ptr<const float>)(uintptr_t)(a + t * P);
    }
  }
  // LDS reads of one fragment (16-byte ones are not merged; fp32 rows may be)
  static constexpr int READS = TURNED ? (sizeof(T) == 2 ? 2 : 4) : 1;
};

// The walk of one operand's loads along the reduction: the next unit within its segment, as a scalar offset from where
// the resource begins.  Behind the last unit the resource is empty: the loads then put zeros into stages (which a
// reduction of an odd number of slabs multiplies once), and every step issues and awaits the same number of loads.
template <bool TWO>
struct Walk {
  const char *q0, *q1;   // the matrix, and that of the second segment (or, TWO, of the up columns)
  int64_t org, bytes;
  uint32_t unit;         // bytes of a unit's step
  int units, reach;      // units of a segment; units that one resource serves
  int next, todo, event; // units until the resource changes
  uint32_t soff;
  u32x4_t r0, r1;
  __device__ __forceinline__ void aim() {
    if (next == units) { next = 0; q0 = q1; }
    const int64_t off = org + next * (int64_t)unit;
    r0 = resource(q0 + off, todo > 0 ? bytes - off : 0);
    if (TWO) r1 = resource(q1 + off, todo > 0 ? bytes - off : 0);
    soff = 0;
    // (a resource's end and a lane's offset are 32-bit: it is left behind before the scalar offset passes FAR)
    event = todo > 0 ? min(min(todo, units - next), reach) : 0x7fffffff;
  }
  __device__ __forceinline__ void start(const void* p0, const void* p1, int64_t o, int64_t b, uint32_t step, int n, int at, int count) {
    q0 = (const char*)p0; q1 = (const char*)p1;
    org = o; bytes = b; unit = step; units = n;
    next = at; todo = count;
    if (next >= units) { next -= units; q0 = q1; }
    reach = __builtin_amdgcn_readfirstlane((int)(FAR / step));
    aim();
  }
  __device__ __forceinline__ void advance() {
    ++next; --todo; soff += unit;
    if (--event == 0) aim();
  }
};

// Bound by the MFMAs (at the clock that these products leave: 1.8 to 1.95 GHz on one card, 1.62 to 1.74 on another) and by
// what the L2 hands out, which overlap all but a fifth.  On the faster card: 256x256 tiles, 4096 tokens, us a slab: 0.75; without loads 0.65, without LDS reads 0.59, without MFMAs 0.53.
// At 4096 x 11008, 4096 tokens: X [Wg|W1] 600 us (1.23 PFLOP/s), H W2 259 (1.43), dY W2^T 354 (1.04), dU W1^T + dG Wg^T 509 (1.45),
// X^T [dU|dG] 631 (1.17), H^T dY 315 (1.17).
template <typename T, int BM, int BN, int WGM, int WGN, int STAGES, int LA_, int LB_, int EPI>
__global__ void __launch_bounds__(WGM* WGN * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
plain_kernel(const PlainArgs p) {
  constexpr bool PAIR = EPI == EPI_GLU;
  constexpr int NW = WGM * WGN;
  constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  constexpr int BNH = PAIR ? BN / 2 : BN;      // output columns of the tile
  using SA = Side<T, BM, LA_>;
  using SB = Side<T, BNH, LB_>;
  constexpr int BK = SA::BK;
  constexpr int A_BLK = BM / 16, B_BLK = BN / 16, HB = BNH / 16;   // blocks of a slab; HB: of one matrix's columns
  constexpr int LA = A_BLK / NW, LB = B_BLK / NW, LPW = LA + LB;   // loads of a wavefront and slab
  // a ring of STAGES slabs; pairs of slabs: one more pair
  constexpr bool PAIRED = SA::UNIT == 2 || SB::UNIT == 2;
  constexpr int NA = SA::UNIT == 2 ? STAGES / 2 + 1 : STAGES, NB = SB::UNIT == 2 ? STAGES / 2 + 1 : STAGES;
  constexpr int UA = SA::UNIT_BYTES, UB = SB::UNIT_BYTES * (PAIR ? 2 : 1), B_AT = NA * UA;
  static_assert(A_BLK % NW == 0 && B_BLK % NW == 0, "blocks divide over the wavefronts");
  static_assert(!PAIR || HB % NW == 0 || NW % HB == 0, "a load belongs to one matrix");
  static_assert(!PAIR || SB::UNIT == 1, "two matrices are fetched slab by slab");
  static_assert(STAGES >= 3 && (!PAIRED || STAGES % 2 == 0) && (STAGES + 1) * LPW <= 63, "loads in flight must fit the counter");
  static_assert(TM % 2 == 0 && (!PAIR || TN % 2 == 0), "row tiles are stored in pairs");

  extern __shared__ u32x4_t smem_v[];
  char* const smem = (char*)smem_v;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int tiles_n1 = (p.n_store + BNH - 1) / BNH, tiles_n = p.twin ? 2 * tiles_n1 : tiles_n1;
  const int tiles_m = (p.M + BM - 1) / BM;
  const int logical = xcd_remap(blockIdx.x, tiles_m * tiles_n);
  const int gsz = p.group_m * tiles_n;
  const int first_m = (logical / gsz) * p.group_m;
  const int gm = min(tiles_m - first_m, p.group_m);
  const int tm = first_m + (logical % gsz) % gm, tn2 = (logical % gsz) / gm;
  const int which = tn2 >= tiles_n1, tn = which ? tn2 - tiles_n1 : tn2;
  const int m0 = tm * BM, n0 = tn * BNH;

  // slabs: segs times ceil(K / BK), a whole number of pairs of them if pairs are fetched; this range's part
  constexpr int CUT = PAIRED ? 2 : 1;
  const int ns = (p.K + BK * CUT - 1) / (BK * CUT) * CUT;
  const int total = ns * p.segs;
  const int per = (total / CUT + p.n_split - 1) / p.n_split * CUT;
  const int s0 = blockIdx.y * per;
  const int nk = max(0, min(total, s0 + per) - s0);
  const int k_end = (p.K + SA::EPC - 1) / SA::EPC * SA::EPC;   // chunks of the reduction from here on read as zero

  uint32_t va[SA::UNIT][LA], vb[SB::UNIT][LB];
  int ka0 = 0, kb0 = 0;   // the lane's first element in a unit (the same for all its blocks)
#pragma unroll
  for (int h = 0; h < SA::UNIT; ++h)
#pragma unroll
    for (int i = 0; i < LA; ++i) va[h][i] = SA::source(wave + i * NW + h * A_BLK, lane, (uint32_t)p.lda, &ka0);
#pragma unroll
  for (int h = 0; h < SB::UNIT; ++h)
#pragma unroll
    for (int i = 0; i < LB; ++i) vb[h][i] = SB::source((wave + i * NW) % HB + h * HB, lane, (uint32_t)p.ldb, &kb0);
  const uint32_t lds0 = lds_offset((const char*)smem);
  const uint32_t lds_w = lds0 + wave * 1024;
  Walk<false> wa;
  Walk<PAIR> wb;
  wa.start(p.A[0], p.A[1], SA::origin(m0, p.lda), p.a_bytes, SA::step((uint32_t)p.lda), ns / SA::UNIT, s0 / SA::UNIT, nk / SA::UNIT);
  wb.start(which ? p.B[1] : p.B[0], p.B[1], SB::origin(n0, p.ldb), p.b_bytes, SB::step((uint32_t)p.ldb), ns / SB::UNIT,
           s0 / SB::UNIT, nk / SB::UNIT);

  // load number i of the left (right) operand's next unit into a stage; half: KC2, which half of its rows
  auto load_a = [&](int i, int stage, int half) {
    const uint32_t out = !SA::TURNED && ka0 >= k_end - wa.next * (BK * SA::UNIT) ? NOWHERE : 0u;
    load_to_lds(wa.r0, lds_w + stage * UA + (half * A_BLK + i * NW) * 1024, SA::TURNED ? va[half][i] : va[half][i] | out, wa.soff);
  };
  auto load_b = [&](int i, int stage, int half) {
    const uint32_t out = !SB::TURNED && kb0 >= k_end - wb.next * (BK * SB::UNIT) ? NOWHERE : 0u;
    // (gated: load i NW + wave belongs to the second matrix from HB on)
    const bool second = PAIR && (HB >= NW ? i * NW >= HB : (wave + i * NW) >= HB);
    load_to_lds(second ? wb.r1 : wb.r0, lds_w + B_AT + stage * UB + (half * HB + i * NW) * 1024,
                SB::TURNED ? vb[half][i] : vb[half][i] | out, wb.soff);
  };

  f32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  constexpr int TNH = PAIR ? TN / 2 : TN;   // column tiles of one matrix
  const uint32_t la = lds0 + SA::first(wm * TM, lane), lb = lds0 + B_AT + SB::first(wn * TNH, lane);
  // DBL: the left operand's fragments in two sets as well
  constexpr bool DBL = TM * TN <= 16;
  Frag fa[DBL ? 2 : 1][TM], fb[2][TN];
  auto read_a = [&](int set, int i, uint32_t st, int half) { SA::read(fa[DBL ? set : 0][i], la + st, i, half); };
  auto read_b = [&](int set, int j, uint32_t st, int half) {
    SB::read(fb[set][j], lb + st + (j / TNH) * (HB * 1024), j % TNH, half);
  };
  auto mma = [&](int set, int i, int j) {
    if constexpr (sizeof(T) == 2) {
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][j].v, fa[DBL ? set : 0][i].v, acc[i][j], 0, 0, 0);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[set][j].f[t], fa[DBL ? set : 0][i].f[t], acc[i][j], 0, 0, 0);
    }
  };
  // Step s multiplies slab s, whose fragments are in registers, reads those of slab s + 1 and has one
  // barrier, placed where the reads that it waits for were issued long before.
  //   DBL (small wavefront tiles): the reads are dealt out over the first five eighths of the MFMAs; the
  //     barrier after three quarters retires slab s + 1, which is in registers then, and publishes slab s + 2;
  //     the loads of slab s + 1 + STAGES go out behind it.
  //   otherwise: the left operand's fragment i is overwritten as soon as the MFMAs that use it are issued; the
  //     barrier in the middle retires slab s and publishes slab s + 2; the loads of slab s + STAGES follow.
  // An operand fetched in pairs of slabs retires a pair in every second step, and half of the rows of the next
  // pair go out in each: one half is under way before the first step, and then a pair is as many steps under
  // way as a slab.
#pragma unroll
  for (int m = 0; m < STAGES + (PAIRED ? 1 : 0); ++m) {
    const int t = PAIRED ? m - 1 : m;   // slab
    if (SA::UNIT == 2) {
#pragma unroll
      for (int i = 0; i < LA; ++i) load_a(i, m / 2, m & 1);
      if (m & 1) wa.advance();
    } else if (t >= 0) {
#pragma unroll
      for (int i = 0; i < LA; ++i) load_a(i, t, 0);
      wa.advance();
    }
    if (SB::UNIT == 2) {
#pragma unroll
      for (int i = 0; i < LB; ++i) load_b(i, m / 2, m & 1);
      if (m & 1) wb.advance();
    } else if (t >= 0) {
#pragma unroll
      for (int i = 0; i < LB; ++i) load_b(i, t, 0);
      wb.advance();
    }
  }
  wait_vmcnt<(STAGES - 2) * LPW>();   // slabs 0 and 1
  lds_barrier();
#pragma unroll
  for (int j = 0; j < TN; ++j) read_b(0, j, 0, 0);
#pragma unroll
  for (int i = 0; i < TM; ++i) read_a(0, i, 0, 0);
  if (DBL) {
    wait_lgkmcnt<0>();
    lds_barrier();
#pragma unroll
    for (int i = 0; i < LA; ++i) load_a(i, SA::UNIT == 2 ? NA - 1 : 0, SA::UNIT == 2);
    wa.advance();
#pragma unroll
    for (int i = 0; i < LB; ++i) load_b(i, SB::UNIT == 2 ? NB - 1 : 0, SB::UNIT == 2);
    wb.advance();
  }
  int sta = 0, stb = 0;   // the stages of slab s
  auto step = [&](auto setc) {
    constexpr int set = decltype(setc)::value;   // s mod 2
    const int na = sta + 1 == NA ? 0 : sta + 1, nb = stb + 1 == NB ? 0 : stb + 1;
    // where slab s + 1 is read, and where the loads of this step go
    const uint32_t xa = (SA::UNIT == 2 && set == 0 ? sta : na) * UA, xb = (SB::UNIT == 2 && set == 0 ? stb : nb) * UB;
    const int ha = SA::UNIT == 2 && set == 0, hb = SB::UNIT == 2 && set == 0;
    const int pa = SA::UNIT == 2 ? (!DBL && set == 0 ? (sta == 0 ? NA - 1 : sta - 1) : sta) : DBL ? na : sta;
    const int pb = SB::UNIT == 2 ? (!DBL && set == 0 ? (stb == 0 ? NB - 1 : stb - 1) : stb) : DBL ? nb : stb;
    constexpr int ga = SA::UNIT == 2 ? (DBL ? set : 1 - set) : 0, gb = SB::UNIT == 2 ? (DBL ? set : 1 - set) : 0;
    auto issue = [&](int l) {
      if (l < LA) load_a(l, pa, ga);
      else load_b(l - LA, pb, gb);
    };
    FFS_ORDER;
    if constexpr (DBL) {
      constexpr int NM = TM * TN, NR = TM + TN, RD = NM * 5 / 8, SYNC = NM * 3 / 4;
#pragma unroll
      for (int q = 0; q < NM; ++q) {
        const int i = q / TN, j = (i & 1) ? TN - 1 - q % TN : q % TN;
        mma(set, i, j);
        FFS_ORDER;
#pragma unroll
        for (int r = 0; r < NR; ++r)
          if (r * RD / NR == q) {
            if (r < TN) read_b(set ^ 1, r, xb, hb);
            else read_a(set ^ 1, r - TN, xa, ha);
          }
        FFS_ORDER;
        if (q == SYNC - 1) {
          wait_vmcnt<(STAGES - 2) * LPW>();
          wait_lgkmcnt<0>();
          lds_barrier();
          FFS_ORDER;
        }
#pragma unroll
        for (int l = 0; l < LPW; ++l)
          if (SYNC + l * (NM - SYNC) / LPW == q) issue(l);
        FFS_ORDER;
      }
    } else {
      constexpr int RB = TM / 2 - 1;                  // the barrier follows this row
      // reads of this step issued in front of the barrier
      constexpr int YOUNGER = sizeof(T) == 2 ? (RB + 1) * SA::READS + ((RB + 1) * TN + TM - 1) / TM * SB::READS : 0;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int jj = 0; jj < TN; ++jj) {
          mma(set, i, (i & 1) ? TN - 1 - jj : jj);
          FFS_ORDER;
#pragma unroll
          for (int q = 0; q < TN; ++q)
            if (q * TM == i * TN + jj) read_b(set ^ 1, q, xb, hb);
          FFS_ORDER;
        }
        read_a(0, i, xa, ha);
        FFS_ORDER;
        if (i == RB) {
          wait_vmcnt<(STAGES - 3) * LPW>();
          wait_lgkmcnt<YOUNGER>();
          lds_barrier();
          FFS_ORDER;
        }
        if (i > RB) {
#pragma unroll
          for (int l = 0; l < LPW; ++l)
            if (l * (TM - RB - 1) / LPW == i - RB - 1) issue(l);
          FFS_ORDER;
        }
      }
    }
    if (SA::UNIT == 1 || ga == 1) wa.advance();
    if (SB::UNIT == 1 || gb == 1) wb.advance();
    if (SA::UNIT == 1 || set == 1) sta = na;
    if (SB::UNIT == 1 || set == 1) stb = nb;
  };
  for (int s = 0; s < nk; s += 2) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  }
  wait_vmcnt<0>();

  // Store.  A lane holds columns 4 (l >> 4) .. + 3 of row l & 15 of each 16x16 tile.  Each wavefront turns 32
  // rows at a time round in a piece of LDS of its own, so that eight lanes (gated: four) hold 64 (32)
  // consecutive columns of a row: whole cache lines, and the kept derivatives are read in the same shape, a
  // group of 32 rows ahead.
  constexpr int OW = PAIR ? WN / 2 : WN;             // output columns of a wavefront
  constexpr int LPR = OW / 8, RP = 64 / LPR, NP = 32 / RP;
  constexpr int PITCH = WN * 4 + 16;
  static_assert(NW * 32 * PITCH <= B_AT + NB * UB, "the stages' memory is used");
  wait_lgkmcnt<0>();
  lds_barrier();   // every wavefront is done with the stages
  char* const own = smem + wave * (32 * PITCH);
  const int col = n0 + wn * OW + (lane % LPR) * 8;
  const int64_t row0 = m0 + wm * WM + lane / LPR;
  const int rows = stored_rows<T, EPI>(p);
  using KT = kept_t<T>;
  Raw8<KT> ka[2][EPI == EPI_GRAD ? NP : 1], kb[2][EPI == EPI_GRAD ? NP : 1];
  auto fetch = [&](int set, int ip) {
    if constexpr (EPI == EPI_GRAD) {
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        const int64_t row = row0 + ip * 16 + q * RP;
        if (row < rows && col < p.n_store && p.part == nullptr) {
          ka[set][q].load(p.D1, row * p.ldi + col);
          if (p.D2 != nullptr) kb[set][q].load(p.D2, row * p.ldi + col);
        }
      }
    }
  };
  fetch(0, 0);
#pragma unroll
  for (int ip = 0; ip < TM; ip += 2) {
    constexpr int last = TM - 2;
    if (ip < last) fetch((ip / 2 + 1) & 1, ip + 2);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *(f32x4_t*)(own + (h * 16 + (lane & 15)) * PITCH + (j * 16 + 4 * (lane >> 4)) * 4) = acc[ip + h][j];
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const char* const at = own + (q * RP + lane / LPR) * PITCH + (lane % LPR) * 32;
      float v[8], u[8];
      load8<float>(at, 0, v);
      if (PAIR) load8<float>(at + OW * 4, 0, u);
      const int64_t row = row0 + ip * 16 + q * RP;
      if (row >= (p.part != nullptr ? p.M : rows) || col >= p.n_store) continue;
      if (p.part != nullptr) {
        const int planes = PAIR || p.twin ? 2 : 1;
        const int64_t to = (((int64_t)blockIdx.y * planes + which) * p.M + row) * p.ldp + col;
        store8<float>(p.part, to, v);
        if (PAIR) store8<float>(p.part, to + (int64_t)p.M * p.ldp, u);
      } else if constexpr (EPI == EPI_GRAD) {
        float a[8], b[8];
        ka[(ip / 2) & 1][q].get(a);
        kb[(ip / 2) & 1][q].get(b);
        grad8<T>(p, row, col, v, a, b);
      } else {
        emit8<T, EPI>(p, which, row, col, v, u);
      }
    }
  }
}

// Sum of the ranges' fp32 sums in range order, and the store step.  One thread per row, plane of a twin
// product and eight columns; four ranges are read at a time.
template <typename T, int EPI>
__global__ void __launch_bounds__(64) plain_reduce_kernel(const PlainArgs p) {
  constexpr bool PAIR = EPI == EPI_GLU;
  const int cpr = p.n_store / 8;
  const int64_t id = (int64_t)blockIdx.x * 64 + threadIdx.x;
  const int64_t per_plane = (int64_t)stored_rows<T, EPI>(p) * cpr;
  const int which = p.twin && id >= per_plane;
  const int64_t in = which ? id - per_plane : id;
  if (in >= per_plane) return;
  const int64_t row = in / cpr;
  const int col = (int)(in % cpr) * 8;
  const int planes = PAIR || p.twin ? 2 : 1;
  const int64_t plane = (int64_t)p.M * p.ldp;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int s0 = 0; row < p.M && s0 < p.n_split; s0 += 4) {
    float w[4][8], x[PAIR ? 4 : 1][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = min(s0 + i, p.n_split - 1);
      const int64_t at = ((int64_t)s * planes + which) * plane + row * p.ldp + col;
      load8<float>(p.part, at, w[i]);
      if (PAIR) load8<float>(p.part, at + plane, x[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s0 + i < p.n_split)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] += w[i][e];
          if (PAIR) u[e] += x[i][e];
        }
  }
  emit8<T, EPI>(p, which, row, col, v, u);
}

// The weights' gradients of at most 32 tokens: a reduction of one slab, so that the output's traffic is all there is.
// The kernel above then spends its time on starting workgroups (180 of four wavefronts a us) and on one dependent
// round trip each.  Here three workgroups a CU walk over the 128x128 tiles and fetch the next one's operands before
// they multiply and store the present one.  4096 x 11008, 8 tokens: dW1 and dWg 65 -> 38 us (180 MB), dW2 39 -> 23.
// (Both operands turned round, bf16.)
template <int LA_, int LB_>
__global__ void __launch_bounds__(256) outer_kernel(const PlainArgs p, int tiles_m, int tiles_n1, int tiles) {
  using SA = Side<uint16_t, 128, LA_>;
  using SB = Side<uint16_t, 128, LB_>;
  constexpr int BUF = 16 * 1024, PITCH = 64 * 4 + 16;   // a slab of both operands; staging of 16 rows a wavefront
  __shared__ __attribute__((aligned(16))) char smem[2 * BUF + 4 * 16 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t lds0 = lds_offset(smem);
  int k = 0;
  uint32_t va[2], vb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    va[i] = SA::source(wave + i * 4, lane, (uint32_t)p.lda, &k);
    vb[i] = SB::source(wave + i * 4, lane, (uint32_t)p.ldb, &k);
  }
  struct Where { int m0, n0, which; };
  auto where = [&](int t) {
    const int tn2 = t / tiles_m, which = tn2 >= tiles_n1;
    return Where{(t - tn2 * tiles_m) * 128, (which ? tn2 - tiles_n1 : tn2) * 128, which};
  };
  auto fetch = [&](const Where& w, int buf) {
    const int64_t ao = SA::origin(w.m0, p.lda), bo = SB::origin(w.n0, p.ldb);
    const u32x4_t ra = resource((const char*)p.A[0] + ao, p.a_bytes - ao);
    const u32x4_t rb = resource((const char*)(w.which ? p.B[1] : p.B[0]) + bo, p.b_bytes - bo);
    const uint32_t st = lds0 + buf * BUF + wave * 1024;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_to_lds(ra, st + i * 4096, va[i], 0);
      load_to_lds(rb, st + 8192 + i * 4096, vb[i], 0);
    }
  };
  const uint32_t la = lds0 + SA::first(wm * 4, lane), lb = lds0 + 8192 + SB::first(wn * 4, lane);
  char* const own = smem + 2 * BUF + wave * (16 * PITCH);
  int t = blockIdx.x, buf = 0;
  if (t >= tiles) return;
  Where w = where(t);
  fetch(w, 0);
  while (true) {
    wait_vmcnt<0>();
    wait_lgkmcnt<0>();
    lds_barrier();   // this tile's operands are there for all; all are done with the other buffer
    const int tn = t + gridDim.x;
    const Where next = where(tn < tiles ? tn : t);
    if (tn < tiles) fetch(next, buf ^ 1);
    Frag fa[4], fb[4];
    f32x4_t acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) SB::read(fb[j], lb + buf * BUF, j, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) SA::read(fa[i], la + buf * BUF, i, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j].v, fa[i].v, f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    const int col = w.n0 + wn * 64 + (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) *(f32x4_t*)(own + (lane & 15) * PITCH + (j * 16 + 4 * (lane >> 4)) * 4) = acc[i][j];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int r = q * 8 + (lane >> 3);
        float v[8], u[8];
        load8<float>(own + r * PITCH + (lane & 7) * 32, 0, v);
        const int64_t row = w.m0 + wm * 64 + i * 16 + r;
        if (row < p.M && col < p.n_store) emit8<uint16_t, EPI_OUT>(p, w.which, row, col, v, u);
      }
    }
    if (tn >= tiles) break;
    t = tn;
    w = next;
    buf ^= 1;
  }
}

// A workgroup per row, in 32-bit words: neighbouring lanes on neighbouring ones, AT of a thread's under way.  (A row of
// an odd number of bf16 begins in the middle of a word in every second row.  The matrix has a multiple of 8 rows, so
// that each word with an element of it is whole.)  blockIdx.y: which of the two matrices.  Bound by memory: two bf16
// matrices of 4096 x 11007, 360 MB, in 71 us (5.1 TB/s); by elements, eight to a thread, 97.
template <bool BF16>
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint32_t* src0, const uint32_t* src1, uint32_t* dst0, uint32_t* dst1,
                                                       int cols, int words) {
  constexpr int AT = 4, PER = BF16 ? 2 : 1;   // PER: elements of a word
  const int64_t first = (int64_t)blockIdx.x * cols;
  const uint32_t* const src = (blockIdx.y ? src1 : src0) + first / PER;
  uint32_t* const dst = (blockIdx.y ? dst1 : dst0) + (int64_t)blockIdx.x * words;
  const bool odd = BF16 && (first & 1);
  for (int i0 = threadIdx.x; i0 < words; i0 += AT * 256) {
    uint32_t v[AT], w[AT];
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      const int i = i0 + a * 256;
      v[a] = i * PER < cols ? src[i] : 0u;
      w[a] = odd && i * PER + 1 < cols ? src[i + 1] : 0u;
    }
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      const int i = i0 + a * 256;
      if (odd) v[a] = (v[a] >> 16) | (w[a] << 16);
      else if (BF16 && i * PER + 1 >= cols) v[a] &= 0xffffu;
      if (i < words) dst[i] = v[a];
    }
  }
}

template <typename T, int BM, int BN, int WGM, int WGN, int STAGES, int LA_, int LB_, int EPI>
static int launch_tile(const PlainArgs& a, hipStream_t st) {
  constexpr auto ring = [](int rows, int lay) { return (size_t)rows * (lay == LAY_KC2 ? (STAGES / 2 + 1) * 128 : STAGES * 64); };
  constexpr size_t lds = ring(BM, LA_) + ring(BN, LB_);
  static_assert(lds <= 160 * 1024, "LDS budget of a CU");
  auto kern = plain_kernel<T, BM, BN, WGM, WGN, STAGES, LA_, LB_, EPI>;
  // (a set-once note per device that the limit of dynamic LDS has been raised; racing first calls both
  // set it, which is harmless)
  static std::atomic<uint64_t> configured{0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return -1;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev >= 64 || !(configured.load(std::memory_order_acquire) & bit)) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return -1;
    if (dev < 64) configured.fetch_or(bit, std::memory_order_release);
  }
  const int bnh = EPI == EPI_GLU ? BN / 2 : BN;
  const int tiles_m = (a.M + BM - 1) / BM;
  const int64_t tiles = (int64_t)tiles_m * ((a.n_store + bnh - 1) / bnh) * (a.twin ? 2 : 1);
  if (tiles * (WGM * WGN * 64) > 0xffffffffll) return -1;   // threads of a launch
  PlainArgs g = a;
  // as many row tiles per group as make an XCD's tiles read the fewest rows of both operands
  const int per_cu = lds <= 80 * 1024 ? 2 : 1;
  const int r = (int)std::max<int64_t>(1, std::min<int64_t>(32 * per_cu, tiles / 8));
  g.group_m = std::max(1, std::min(tiles_m, (int)(sqrt((double)r * BN / BM) + 0.5)));
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles, a.n_split), dim3(WGM * WGN * 64), lds, st, g);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <typename T, int LA_, int LB_, int EPI>
static int launch_shape(const PlainArgs& a, int shape, hipStream_t st) {
  constexpr bool BF = sizeof(T) == 2, PAIRED = LA_ == LAY_KC2 || LB_ == LAY_KC2;
  if (a.a_lay != LA_ || a.b_lay != LB_) return -1;
  switch (shape) {
    case PS_128x128: return launch_tile<T, 128, 128, 2, 2, PAIRED ? 4 : 5, LA_, LB_, EPI>(a, st);
    case PS_64x64:   // (bf16 gated: 64 x 64 of each matrix)
      return launch_tile<T, 64, BF && EPI == EPI_GLU ? 128 : 64, 2, 2, BF && EPI == EPI_GLU ? 6 : 8, LA_, LB_, EPI>(a, st);
  }
  if constexpr (BF) {
    if (shape == PS_256x256) return launch_tile<T, 256, 256, 2, 4, 4, LA_, LB_, EPI>(a, st);
    if (shape == PS_256x128) return launch_tile<T, 256, 128, 4, 2, 4, LA_, LB_, EPI>(a, st);
  }
  return -1;
}

template <typename T, int EPI>
static int launch_reduce(const PlainArgs& a, hipStream_t st) {
  const int64_t n = (int64_t)stored_rows<T, EPI>(a) * (a.n_store / 8) * (a.twin ? 2 : 1);
  hipLaunchKernelGGL((plain_reduce_kernel<T, EPI>), dim3((unsigned)((n + 63) / 64)), dim3(64), 0, st, a);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <typename T, int LA_, int LB_, int EPI>
static int launch_whole(const PlainArgs& a, int shape, hipStream_t st) {
  const int rc = launch_shape<T, LA_, LB_, EPI>(a, shape, st);
  return rc == 0 && a.part ? launch_reduce<T, EPI>(a, st) : rc;
}

template <int LA_, int LB_>
static int launch_outer(const PlainArgs& a, hipStream_t st) {
  const int64_t tiles_m = (a.M + 127) / 128, tiles_n1 = (a.n_store + 127) / 128, tiles = tiles_m * tiles_n1 * (a.twin ? 2 : 1);
  if (tiles > 0x3fffffff) return -1;
  hipLaunchKernelGGL((outer_kernel<LA_, LB_>), dim3((unsigned)std::min<int64_t>(tiles, 3 * 256)), dim3(256), 0, st, a, (int)tiles_m,
                     (int)tiles_n1, (int)tiles);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

// The products of the two passes and the way their operands lie.
template <typename T>
static int launch_typed(const PlainArgs& a, int epi, int shape, hipStream_t st) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int ACT_K = BF ? LAY_BK : LAY_KC2, ACT_M = BF ? LAY_BM : LAY_MC;   // this path's activations
  switch (epi) {
    case EPI_GLU: return launch_whole<T, LAY_KC2, LAY_MC, EPI_GLU>(a, shape, st);
    case EPI_GELU: return launch_whole<T, LAY_KC2, LAY_MC, EPI_GELU>(a, shape, st);
    case EPI_GRAD: return launch_whole<T, LAY_KC2, LAY_KC, EPI_GRAD>(a, shape, st);
    case EPI_OUT:
      if (!turned(a.a_lay) && turned(a.b_lay)) return launch_whole<T, ACT_K, LAY_MC, EPI_OUT>(a, shape, st);        // H W2
      if (!turned(a.a_lay)) return launch_whole<T, ACT_K, BF ? LAY_KC2 : LAY_KC, EPI_OUT>(a, shape, st);            // dU W1^T
      if constexpr (BF)
        if (a.K <= 32 && !a.part) return a.a_lay == LAY_MC ? launch_outer<LAY_MC, LAY_BM>(a, st) : launch_outer<LAY_BM, LAY_MC>(a, st);
      if (a.a_lay == LAY_MC) return launch_whole<T, LAY_MC, ACT_M, EPI_OUT>(a, shape, st);                          // X^T dU
      return launch_whole<T, ACT_M, LAY_MC, EPI_OUT>(a, shape, st);                                                 // H^T dY
  }
  return -1;
}

static PlainShape shape_of(const PlainArgs& a, int epi) {
  return {a.M, a.N, a.K, a.segs, a.twin, epi, a.D2 != nullptr, turned(a.a_lay), turned(a.b_lay)};
}

int launch_plain(PlainArgs a, int epi, int bf16, float* part, hipStream_t st) {
  if (a.M <= 0 || a.N <= 0) return 0;
  if ((a.lda & 7) || (a.ldb & 7) || (a.segs != 1 && a.segs != 2) || a.n_store < a.N) return -1;
  // a lane's offset inside a tile stays below 2 GiB
  if (a.lda > (1 << 20) || a.ldb > (1 << 20)) return -1;
  const PlainPlan pl = plain_plan(shape_of(a, epi), bf16);
  a.n_split = pl.split;
  a.part = pl.split > 1 ? part : nullptr;
  a.ldp = a.n_store;
  return bf16 ? launch_typed<uint16_t>(a, epi, pl.shape, st) : launch_typed<float>(a, epi, pl.shape, st);
}

int launch_pad_rows(const void* src0, const void* src1, void* dst0, void* dst1, int rows, int cols, int bf16, hipStream_t st) {
  if (rows <= 0 || cols <= 0) return 0;
  if (rows & 7) return -1;
  const dim3 grid(rows, src1 ? 2 : 1);
  const int words = (cols + 7) / 8 * (bf16 ? 4 : 8);
  const uint32_t *s0 = (const uint32_t*)src0, *s1 = (const uint32_t*)src1;
  if (bf16) hipLaunchKernelGGL(pad_rows_kernel<true>, grid, dim3(256), 0, st, s0, s1, (uint32_t*)dst0, (uint32_t*)dst1, cols, words);
  else hipLaunchKernelGGL(pad_rows_kernel<false>, grid, dim3(256), 0, st, s0, s1, (uint32_t*)dst0, (uint32_t*)dst1, cols, words);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace ffsplit
