// C ABI of the training calls (declared in include/ffsplit.h): host-side validation, layouts of the kept
// activations and of the scratch, launch sequences.
#include "../../include/ffsplit.h"
#include "layout.h"
#include "plain.h"
#include "prep.h"
#include "grad.h"
#include "train.h"
#include <math.h>

using namespace ffsplit;

namespace {

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
inline bool misaligned256(const void* p) { return ((uintptr_t)p & 255u) != 0; }

#define FFS_TRY(expr)                      \
  do {                                     \
    if ((expr) != 0) return FFSPLIT_E_HIP; \
  } while (0)

// (widths: a lane's byte offset inside a tile of a product fits 31 bits; tokens: counts of rows, rounded up to
// a tile's, and of workgroups fit theirs)
constexpr int MAX_WIDTH = 1 << 20;
constexpr int64_t MAX_TOKENS = (int64_t)1 << 28;
int check_dense(const ffsplit_desc_t* d, int64_t T) {
  if (!d) return FFSPLIT_E_NULLPTR;
  if (d->d_model <= 0 || d->d_ff <= 0) return FFSPLIT_E_BADDESC;
  if (d->act != FFSPLIT_ACT_GELU && d->act != FFSPLIT_ACT_SWIGLU) return FFSPLIT_E_BADDESC;
  if (d->dtype != FFSPLIT_F32 && d->dtype != FFSPLIT_BF16) return FFSPLIT_E_BADDESC;
  if (d->d_model % 8 != 0 || T < 0 || T > MAX_TOKENS) return FFSPLIT_E_BADSHAPE;
  if (d->d_model > MAX_WIDTH || d->d_ff > MAX_WIDTH - 64) return FFSPLIT_E_BADSHAPE;
  return FFSPLIT_OK;
}

// Everything the calls below need to know about a layer and T tokens.
struct Dense {
  int bf16, gated, d, f, f8, ldi, planes;
  int64_t T, esz;
  int64_t rows;          // of the activations below: T, in bf16 rounded up to the blocks' 16
  size_t act_bytes;      // of H, D1, D2, dU or dG: [rows, ldi]
  size_t pad_bytes;      // of an aligned copy of W1 or Wg (0: rows are aligned as they are)
};

Dense dense_of(const ffsplit_desc_t& d, int64_t T) {
  Dense s = {};
  s.bf16 = d.dtype == FFSPLIT_BF16;
  s.gated = d.act == FFSPLIT_ACT_SWIGLU;
  s.planes = s.gated ? 2 : 1;
  s.d = d.d_model; s.f = d.d_ff; s.f8 = round_up(d.d_ff, 8); s.ldi = round_up(d.d_ff, 64);
  s.T = T; s.esz = s.bf16 ? 2 : 4;
  s.rows = s.bf16 ? (T + 15) / 16 * 16 : T;
  s.act_bytes = align256((size_t)s.rows * s.ldi * s.esz);
  s.pad_bytes = s.f8 == s.f ? 0 : align256((size_t)s.d * s.f8 * s.esz);
  return s;
}

// scratch for the ranges' sums of any of a pass's products, one after the other
size_t part_room(const Dense& s, int first, int last) {
  size_t room = 0;
  for (int which = first; which <= last; ++which) {
    const size_t n = plain_part_bytes(dense_product(which, s.T, s.d, s.f, s.planes), s.bf16);
    if (n > room) room = n;
  }
  return align256(room);
}
size_t forward_ws(const ffsplit_desc_t& d, int64_t T) {
  const Dense s = dense_of(d, T);
  return s.planes * s.pad_bytes + s.act_bytes + part_room(s, DENSE_UP, DENSE_DOWN);
}
size_t backward_ws(const ffsplit_desc_t& d, int64_t T) {
  const Dense s = dense_of(d, T);
  return s.planes * s.pad_bytes + s.planes * s.act_bytes + part_room(s, DENSE_GRAD, DENSE_DDOWN);
}
size_t kept_bytes(const Dense& s) { return (1 + s.planes) * s.act_bytes; }

// W1 (and Wg) with rows of a multiple of 8 elements: as they are, or copied to ws
int aligned_weights(const Dense& s, const void* W1, const void* Wg, char* ws, const void** u, const void** g, hipStream_t st) {
  *u = W1; *g = Wg;
  if (!s.pad_bytes) return 0;
  *u = ws;
  if (s.gated) *g = ws + s.pad_bytes;
  return launch_pad_rows(W1, s.gated ? Wg : nullptr, ws, ws + s.pad_bytes, s.d, s.f, s.bf16, st);
}

PlainArgs product(const Dense& s, int which, int planes) {
  const PlainShape q = dense_product(which, s.T, s.d, s.f, planes);
  PlainArgs a = {};
  a.M = (int)q.M; a.N = (int)q.N; a.K = (int)q.K; a.n_store = round_up((int)q.N, 8);
  a.segs = q.segs; a.twin = q.twin;
  a.a_lay = LAY_KC2; a.b_lay = LAY_MC;
  return a;
}
// bytes of a row-major operand: rows of len elements, ld apart
inline int64_t extent(int64_t rows, int64_t ld, int64_t len, int64_t esz) { return ((rows - 1) * ld + len) * esz; }

// an activation's layout with the reduction over the neurons or the tokens, and its bytes
inline int act_k(const Dense& s) { return s.bf16 ? LAY_BK : LAY_KC2; }
inline int act_m(const Dense& s) { return s.bf16 ? LAY_BM : LAY_MC; }
inline int64_t act_extent(const Dense& s) { return s.bf16 ? s.rows * s.ldi * s.esz : extent(s.T, s.ldi, s.f8, s.esz); }

int dense_forward(const Dense& s, const void* X, const void* W1, const void* Wg, const void* W2, void* Y,
                  const float* residual, int y_f32, void* kept, char* ws, hipStream_t st) {
  const void *u, *g;
  if (aligned_weights(s, W1, Wg, ws, &u, &g, st)) return -1;
  char* at = ws + s.planes * s.pad_bytes;
  char* const H = kept ? (char*)kept : at;
  if (!kept) at += s.act_bytes;
  float* const part = (float*)at;
  PlainArgs a = product(s, DENSE_UP, s.planes);
  a.A[0] = X; a.lda = s.d; a.a_bytes = extent(s.T, s.d, s.d, s.esz);
  a.B[0] = s.gated ? g : u; a.B[1] = u; a.ldb = s.f8; a.b_bytes = extent(s.d, s.f8, s.f8, s.esz);
  a.H = H; a.ldi = s.ldi;
  if (kept) { a.D1 = H + s.act_bytes; a.D2 = H + 2 * s.act_bytes; }
  if (launch_plain(a, s.gated ? EPI_GLU : EPI_GELU, s.bf16, part, st)) return -1;
  a = product(s, DENSE_DOWN, s.planes);
  a.A[0] = H; a.lda = s.ldi; a.a_lay = act_k(s); a.a_bytes = act_extent(s);
  a.B[0] = W2; a.ldb = s.d; a.b_bytes = extent(s.f, s.d, s.d, s.esz);
  a.C[0] = Y; a.ldc = s.d; a.resid = residual; a.out_f32 = y_f32;
  return launch_plain(a, EPI_OUT, s.bf16, part, st);
}

int dense_backward(const Dense& s, const void* X, const void* W1, const void* Wg, const void* W2, const void* kept,
                   const void* dY, void* dX, void* dW1, void* dWg, void* dW2, int grad_f32, int accumulate, char* ws,
                   hipStream_t st) {
  const void *u, *g;
  if (dX && aligned_weights(s, W1, Wg, ws, &u, &g, st)) return -1;
  char* at = ws + s.planes * s.pad_bytes;
  char* const dU = at;                                  // (un-gated: the only one)
  char* const dG = s.gated ? dU + s.act_bytes : nullptr;
  at += s.planes * s.act_bytes;
  float* const part = (float*)at;
  const char* const H = (const char*)kept;
  const int64_t act_ext = act_extent(s), x_ext = extent(s.T, s.d, s.d, s.esz);
  PlainArgs a;
  if (dX || dW1 || dWg) {
    // dU = (dY W2^T) D1, dG = (dY W2^T) D2
    a = product(s, DENSE_GRAD, s.planes);
    a.A[0] = dY; a.lda = s.d; a.a_bytes = x_ext;
    a.B[0] = W2; a.ldb = s.d; a.b_lay = LAY_KC; a.b_bytes = extent(s.f, s.d, s.d, s.esz);
    a.D1 = H + s.act_bytes; a.O1 = dU; a.ldi = s.ldi;
    if (s.gated) { a.D2 = H + 2 * s.act_bytes; a.O2 = dG; }
    if (launch_plain(a, EPI_GRAD, s.bf16, part, st)) return -1;
  }
  if (dX) {
    // dX = dU W1^T + dG Wg^T
    a = product(s, DENSE_DX, s.planes);
    a.A[0] = dU; a.A[1] = dG; a.lda = s.ldi; a.a_lay = act_k(s); a.a_bytes = act_ext;
    a.B[0] = u; a.B[1] = g; a.ldb = s.f8; a.b_lay = s.bf16 ? LAY_KC2 : LAY_KC; a.b_bytes = extent(s.d, s.f8, s.f8, s.esz);
    a.C[0] = dX; a.ldc = s.d;
    if (launch_plain(a, EPI_OUT, s.bf16, part, st)) return -1;
  }
  if (dW1 || dWg) {
    // dW1 = X^T dU, dWg = X^T dG: one launch if both are wanted
    a = product(s, DENSE_DUP, dW1 && dWg ? 2 : 1);
    a.A[0] = X; a.lda = s.d; a.a_lay = LAY_MC; a.a_bytes = x_ext;
    a.B[0] = dW1 ? dU : dG; a.B[1] = dG; a.ldb = s.ldi; a.b_lay = act_m(s); a.b_bytes = act_ext;
    a.C[0] = dW1 ? dW1 : dWg; a.C[1] = dWg; a.ldc = s.f;
    a.out_f32 = grad_f32; a.accumulate = accumulate;
    if (launch_plain(a, EPI_OUT, s.bf16, part, st)) return -1;
  }
  if (dW2) {
    // dW2 = H^T dY
    a = product(s, DENSE_DDOWN, s.planes);
    a.A[0] = H; a.lda = s.ldi; a.a_lay = act_m(s); a.a_bytes = act_ext;
    a.B[0] = dY; a.ldb = s.d; a.b_lay = LAY_MC; a.b_bytes = x_ext;
    a.C[0] = dW2; a.ldc = s.d;
    a.out_f32 = grad_f32; a.accumulate = accumulate;
    if (launch_plain(a, EPI_OUT, s.bf16, part, st)) return -1;
  }
  return 0;
}

// One layer of the stack's kept state: its input stream (fp32), the normalised tokens, the layer's own.
struct StackKept { size_t off_n, off_layer, bytes; };
StackKept stack_kept(const Dense& s) {
  StackKept k;
  k.off_n = align256((size_t)s.T * s.d * 4);
  k.off_layer = k.off_n + align256((size_t)s.T * s.d * s.esz);
  k.bytes = k.off_layer + kept_bytes(s);
  return k;
}
// Scratch of the stack's two passes: normalised tokens (forward without kept state) or the two gradients
// between a layer and its norm, then the layer's own.  The norm's sums lie in the same place behind them: room for those of
// NORM_LAYERS layers whatever the layers' size (4.3 MB).
constexpr int64_t NORM_LAYERS = 4096;
size_t stack_ws(const ffsplit_desc_t& d, int64_t T) {
  const Dense s = dense_of(d, T);
  const size_t f = forward_ws(d, T), b = backward_ws(d, T), n = align256(grad_norm_ws_bytes(3 * NORM_LAYERS));
  const size_t layers = 2 * align256((size_t)T * s.d * s.esz) + (f > b ? f : b);
  return layers > n ? layers : n;
}

}  // namespace

namespace ffsplit {

size_t train_workspace_bytes(const ffsplit_desc_t* d, int32_t call_id, int64_t T) {
  if (call_id == FFSPLIT_WS_GRAD_NORM) return T < 0 ? 0 : grad_norm_ws_bytes(T);
  if (check_dense(d, T) != FFSPLIT_OK) return 0;
  if (call_id == FFSPLIT_WS_DENSE_FORWARD) return forward_ws(*d, T);
  if (call_id == FFSPLIT_WS_DENSE_BACKWARD) return backward_ws(*d, T);
  if (call_id == FFSPLIT_WS_DENSE_STACK) return stack_ws(*d, T);
  return 0;
}

}  // namespace ffsplit

extern "C" {

size_t ffsplit_dense_kept_bytes(const ffsplit_desc_t* d, int64_t T) {
  if (check_dense(d, T) != FFSPLIT_OK) return 0;
  return kept_bytes(dense_of(*d, T));
}

int ffsplit_dense_forward(const ffsplit_desc_t* d, const void* X, int64_t T, const void* W1, const void* Wg, const void* W2,
                          void* Y, const float* residual, int32_t y_f32, void* kept, void* workspace,
                          size_t workspace_bytes, void* stream) {
  const int rc = check_dense(d, T);
  if (rc) return rc;
  if (T == 0) return FFSPLIT_OK;
  const Dense s = dense_of(*d, T);
  if (!X || !W1 || !W2 || (s.gated && !Wg) || !Y) return FFSPLIT_E_NULLPTR;
  if (misaligned(X) || misaligned(W1) || misaligned(W2) || misaligned(Wg) || misaligned(Y) || misaligned(residual) ||
      misaligned256(kept))
    return FFSPLIT_E_ALIGN;
  if (!workspace || workspace_bytes < forward_ws(*d, T)) return FFSPLIT_E_WORKSPACE;
  if (misaligned256(workspace)) return FFSPLIT_E_ALIGN;
  FFS_TRY(dense_forward(s, X, W1, Wg, W2, Y, residual, y_f32 != 0, kept, (char*)workspace, (hipStream_t)stream));
  return FFSPLIT_OK;
}

int ffsplit_dense_backward(const ffsplit_desc_t* d, const void* X, int64_t T, const void* W1, const void* Wg, const void* W2,
                           const void* kept, const void* dY, void* dX, void* dW1, void* dWg, void* dW2, int32_t flags,
                           void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_dense(d, T);
  if (rc) return rc;
  if (flags & ~(FFSPLIT_GRAD_F32 | FFSPLIT_GRAD_ACCUMULATE)) return FFSPLIT_E_BADDESC;
  const Dense s = dense_of(*d, T);
  const int accumulate = (flags & FFSPLIT_GRAD_ACCUMULATE) != 0, f32 = (flags & FFSPLIT_GRAD_F32) != 0;
  if (!s.gated && dWg) return FFSPLIT_E_BADDESC;
  if (misaligned(dW1) || misaligned(dWg) || misaligned(dW2)) return FFSPLIT_E_ALIGN;
  hipStream_t st = (hipStream_t)stream;
  if (T == 0) {   // no token: the gradients are zero
    const size_t bytes = (size_t)s.d * s.f * (f32 ? 4 : s.esz);
    for (void* g : {dW1, dWg, dW2})
      if (g && !accumulate) FFS_TRY(launch_fill_zero(g, bytes, st));
    return FFSPLIT_OK;
  }
  if (!X || !W1 || !W2 || (s.gated && !Wg) || !kept || !dY) return FFSPLIT_E_NULLPTR;
  if (misaligned(X) || misaligned(W1) || misaligned(W2) || misaligned(Wg) || misaligned(dY) || misaligned(dX) ||
      misaligned256(kept))
    return FFSPLIT_E_ALIGN;
  if (!workspace || workspace_bytes < backward_ws(*d, T)) return FFSPLIT_E_WORKSPACE;
  if (misaligned256(workspace)) return FFSPLIT_E_ALIGN;
  FFS_TRY(dense_backward(s, X, W1, Wg, W2, kept, dY, dX, dW1, dWg, dW2, f32, accumulate, (char*)workspace, st));
  return FFSPLIT_OK;
}

int ffsplit_token_rmsnorm_backward(const float* x, const void* dn, int64_t T, int32_t d_model, float eps, int32_t dtype,
                                   const float* residual, float* dx, void* dx_cast, void* stream) {
  if (d_model <= 0 || d_model % 8 != 0 || d_model > MAX_WIDTH || T < 0 || T > 0x7fffffff) return FFSPLIT_E_BADSHAPE;
  if (dtype != FFSPLIT_F32 && dtype != FFSPLIT_BF16) return FFSPLIT_E_BADDESC;
  if (T == 0) return FFSPLIT_OK;
  if (!x || !dn || !dx) return FFSPLIT_E_NULLPTR;
  if (misaligned(x) || misaligned(dn) || misaligned(residual) || misaligned(dx) || misaligned(dx_cast)) return FFSPLIT_E_ALIGN;
  FFS_TRY(launch_rmsnorm_backward(x, dn, T, d_model, eps, dtype == FFSPLIT_BF16, residual, dx, dx_cast, (hipStream_t)stream));
  return FFSPLIT_OK;
}

static int check_grads(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes) {
  if (n < 0) return FFSPLIT_E_BADSHAPE;
  if (n == 0) return FFSPLIT_OK;
  if (!grads || !counts || !dtypes) return FFSPLIT_E_NULLPTR;
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] < 0) return FFSPLIT_E_BADSHAPE;
    if (dtypes[i] != FFSPLIT_F32 && dtypes[i] != FFSPLIT_BF16) return FFSPLIT_E_BADDESC;
    if (counts[i] > 0 && !grads[i]) return FFSPLIT_E_NULLPTR;
    if (misaligned(grads[i])) return FFSPLIT_E_ALIGN;
  }
  return FFSPLIT_OK;
}

int ffsplit_grad_norm(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, float* norm,
                      int32_t* nonfinite, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_grads(n, grads, counts, dtypes);
  if (rc) return rc;
  if (!norm) return FFSPLIT_E_NULLPTR;
  if (((uintptr_t)norm & 3u) || ((uintptr_t)nonfinite & 3u)) return FFSPLIT_E_ALIGN;
  if (!workspace || workspace_bytes < grad_norm_ws_bytes(n)) return FFSPLIT_E_WORKSPACE;
  if (misaligned(workspace)) return FFSPLIT_E_ALIGN;
  GradSet g = {};
  g.n = n; g.src = grads; g.counts = counts; g.dtypes = dtypes;
  FFS_TRY(launch_grad_norm(g, norm, nonfinite, (double*)workspace, (hipStream_t)stream));
  return FFSPLIT_OK;
}

int ffsplit_grad_clip(int32_t n, const void* const* grads, const int64_t* counts, const int32_t* dtypes, const float* norm,
                      float max_norm, void* const* out, void* stream) {
  const int rc = check_grads(n, grads, counts, dtypes);
  if (rc) return rc;
  if (!(max_norm > 0.f)) return FFSPLIT_E_BADSHAPE;
  if (n == 0) return FFSPLIT_OK;
  if (!norm || !out) return FFSPLIT_E_NULLPTR;
  if ((uintptr_t)norm & 3u) return FFSPLIT_E_ALIGN;
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] > 0 && !out[i]) return FFSPLIT_E_NULLPTR;
    if (misaligned(out[i])) return FFSPLIT_E_ALIGN;
  }
  GradSet g = {};
  g.n = n; g.src = grads; g.dst = out; g.counts = counts; g.dtypes = dtypes;
  FFS_TRY(launch_grad_clip(g, norm, max_norm, (hipStream_t)stream));
  return FFSPLIT_OK;
}

size_t ffsplit_dense_stack_kept_bytes(const ffsplit_desc_t* d, int32_t n_layers, int64_t T) {
  if (check_dense(d, T) != FFSPLIT_OK || n_layers < 0) return 0;
  return (size_t)n_layers * stack_kept(dense_of(*d, T)).bytes;
}

static int check_stack(const ffsplit_desc_t* d, int32_t n_layers, const void* const* W1, const void* const* Wg,
                       const void* const* W2, int64_t T) {
  const int rc = check_dense(d, T);
  if (rc) return rc;
  if (n_layers < 0) return FFSPLIT_E_BADSHAPE;
  if (n_layers == 0) return FFSPLIT_OK;
  const bool gated = d->act == FFSPLIT_ACT_SWIGLU;
  if (!W1 || !W2 || (gated && !Wg)) return FFSPLIT_E_NULLPTR;
  for (int32_t l = 0; l < n_layers; ++l) {
    if (!W1[l] || !W2[l] || (gated && !Wg[l])) return FFSPLIT_E_NULLPTR;
    if (misaligned(W1[l]) || misaligned(W2[l]) || (gated && misaligned(Wg[l]))) return FFSPLIT_E_ALIGN;
  }
  return FFSPLIT_OK;
}

int ffsplit_dense_stack_forward(const ffsplit_desc_t* d, int32_t n_layers, const void* const* W1, const void* const* Wg,
                                const void* const* W2, float* x, int64_t T, float eps, void* kept, void* workspace,
                                size_t workspace_bytes, void* stream) {
  int rc = check_stack(d, n_layers, W1, Wg, W2, T);
  if (rc) return rc;
  if (n_layers == 0 || T == 0) return FFSPLIT_OK;
  if (!x) return FFSPLIT_E_NULLPTR;
  if (misaligned(x) || misaligned256(kept)) return FFSPLIT_E_ALIGN;
  if (!workspace || workspace_bytes < stack_ws(*d, T)) return FFSPLIT_E_WORKSPACE;
  if (misaligned256(workspace)) return FFSPLIT_E_ALIGN;
  hipStream_t st = (hipStream_t)stream;
  const Dense s = dense_of(*d, T);
  const StackKept k = stack_kept(s);
  const size_t nb = align256((size_t)T * s.d * s.esz);
  char* const ws = (char*)workspace;
  char* kl = (char*)kept;
  if (kept) FFS_TRY(launch_cast(x, T * s.d, 0, kl, st));   // the first layer's input
  for (int32_t l = 0; l < n_layers; ++l) {
    // with kept state a layer reads its input there and writes the next one's (the last: x)
    const float* in = kept ? (const float*)kl : x;
    float* out = kept && l + 1 < n_layers ? (float*)(kl + k.bytes) : x;
    char* const n = kept ? kl + k.off_n : ws;
    FFS_TRY(launch_token_rmsnorm(in, T, s.d, eps, s.bf16, n, st));
    FFS_TRY(dense_forward(s, n, W1[l], s.gated ? Wg[l] : nullptr, W2[l], out, in, 1, kept ? kl + k.off_layer : nullptr,
                          ws + nb, st));
    if (kept) kl += k.bytes;
  }
  return FFSPLIT_OK;
}

int ffsplit_dense_stack_backward(const ffsplit_desc_t* d, int32_t n_layers, const void* const* W1, const void* const* Wg,
                                 const void* const* W2, const void* kept, float* dx, int64_t T, float eps,
                                 void* const* dW1, void* const* dWg, void* const* dW2, int32_t flags, float max_norm,
                                 float* norm, int32_t* nonfinite, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_stack(d, n_layers, W1, Wg, W2, T);
  if (rc) return rc;
  if (flags & ~(FFSPLIT_GRAD_F32 | FFSPLIT_GRAD_ACCUMULATE)) return FFSPLIT_E_BADDESC;
  if (((uintptr_t)norm & 3u) || ((uintptr_t)nonfinite & 3u)) return FFSPLIT_E_ALIGN;
  if (n_layers > 0x7fffffff / 3 || max_norm != max_norm) return FFSPLIT_E_BADSHAPE;
  // (the norm's partial sums lie where the layers' scratch was)
  if (!workspace || workspace_bytes < stack_ws(*d, T) ||
      (norm && workspace_bytes < grad_norm_ws_bytes((int64_t)3 * n_layers)))
    return FFSPLIT_E_WORKSPACE;
  if (misaligned256(workspace)) return FFSPLIT_E_ALIGN;
  const bool gated = d->act == FFSPLIT_ACT_SWIGLU;
  if (n_layers > 0 && (!dW1 || !dW2 || (gated && !dWg))) return FFSPLIT_E_NULLPTR;
  for (int32_t l = 0; l < n_layers; ++l) {
    if (!dW1[l] || !dW2[l] || (gated && !dWg[l])) return FFSPLIT_E_NULLPTR;
    if (misaligned(dW1[l]) || misaligned(dW2[l]) || (gated && misaligned(dWg[l]))) return FFSPLIT_E_ALIGN;
  }
  if (T > 0 && n_layers > 0) {
    if (!kept || !dx) return FFSPLIT_E_NULLPTR;
    if (misaligned(dx) || misaligned256(kept)) return FFSPLIT_E_ALIGN;
  }
  hipStream_t st = (hipStream_t)stream;
  const Dense s = dense_of(*d, T);
  const int f32 = (flags & FFSPLIT_GRAD_F32) != 0, accumulate = (flags & FFSPLIT_GRAD_ACCUMULATE) != 0;
  if (T == 0) {
    for (int32_t l = 0; l < n_layers; ++l) {
      rc = ffsplit_dense_backward(d, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, dW1[l],
                                  gated ? dWg[l] : nullptr, dW2[l], flags, nullptr, 0, stream);
      if (rc) return rc;
    }
  } else if (n_layers > 0) {
    const StackKept k = stack_kept(s);
    const size_t nb = align256((size_t)T * s.d * s.esz);
    char* const dY = (char*)workspace;       // the stream's gradient in bf16 (fp32 layers read the stream's itself)
    char* const dn = dY + nb;
    char* const ws = dn + nb;
    if (s.bf16) FFS_TRY(launch_cast(dx, T * s.d, 1, dY, st));
    for (int32_t l = n_layers - 1; l >= 0; --l) {
      const char* const kl = (const char*)kept + l * k.bytes;
      FFS_TRY(dense_backward(s, kl + k.off_n, W1[l], gated ? Wg[l] : nullptr, W2[l], kl + k.off_layer, s.bf16 ? (void*)dY : dx,
                             dn, dW1[l], gated ? dWg[l] : nullptr, dW2[l], f32, accumulate, ws, st));
      FFS_TRY(launch_rmsnorm_backward((const float*)kl, dn, T, s.d, eps, s.bf16, dx, dx, s.bf16 && l > 0 ? dY : nullptr, st));
    }
  }
  if (norm) {
    GradSet g = {};
    g.n_mats = gated ? 3 : 2;
    g.n = n_layers * g.n_mats;
    g.mats[0] = dW1; g.mats[1] = dW2; g.mats[2] = dWg;
    g.count = (int64_t)s.d * s.f; g.f32 = f32 || !s.bf16;
    FFS_TRY(launch_grad_norm(g, norm, nonfinite, (double*)workspace, st));
    if (max_norm > 0.f) FFS_TRY(launch_grad_clip(g, norm, max_norm, st));
  }
  return FFSPLIT_OK;
}

}  // extern "C"
