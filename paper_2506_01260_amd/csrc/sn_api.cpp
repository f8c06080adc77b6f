// The C ABI: host-side argument validation and dispatch to the kernels.
// Every check runs before anything is launched; see include/sn.h for the
// contract of each entry point.
#include "sn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <exception>
#include <iterator>
#include <vector>

#include "sn_internal.h"

namespace {

thread_local char g_err[512] = "";

int32_t fail(int32_t st, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

int32_t ok() {
  g_err[0] = '\0';
  return SN_OK;
}

}  // namespace


namespace sn {

int32_t set_error(int32_t st, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

}  // namespace sn

namespace {

int32_t hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return ok();
  return fail(SN_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

size_t elem_size(int32_t dt) { return dt == SN_F32 ? 4 : 2; }

bool dtype_ok(int32_t dt) { return dt == SN_F32 || dt == SN_BF16; }

bool elem_aligned(const void *p, int32_t dt) {
  return (reinterpret_cast<uintptr_t>(p) & (elem_size(dt) - 1)) == 0;
}

// Byte range [lo, hi) covered by a rows x cols matrix with row stride ld.
struct Span {
  uintptr_t lo = 0, hi = 0;
};

Span span(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t es) {
  Span s;
  if (!p || rows <= 0 || cols <= 0) return s;
  s.lo = reinterpret_cast<uintptr_t>(p);
  s.hi = s.lo + (static_cast<uintptr_t>(rows - 1) * ld + cols) * es;
  return s;
}

bool overlap(Span a, Span b) { return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi; }

constexpr int64_t kMaxDim = int64_t(1) << 31;  // rows, columns and strides stay below 2^31
constexpr int64_t kMaxElems = int64_t(1) << 40;  // elements of the tensors of a clipping call

int32_t check_basis(const void *basis, int64_t d, int64_t k, int32_t dt) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  if (!basis) return fail(SN_ERR_NULL, "basis is NULL");
  if (reinterpret_cast<uintptr_t>(basis) & 255)
    return fail(SN_ERR_ALIGN, "packed basis must be 256-byte aligned");
  if (d < 1 || d >= kMaxDim) return fail(SN_ERR_SHAPE, "d = %lld out of range", (long long)d);
  if (k < 1 || k > d) return fail(SN_ERR_SHAPE, "k = %lld must satisfy 1 <= k <= d", (long long)k);
  if (k > SN_MAX_K) return fail(SN_ERR_UNSUPPORTED, "k = %lld > SN_MAX_K", (long long)k);
  return SN_OK;
}

// Validates the id / table arguments shared by compress and decompress.
int32_t check_ids(int64_t N, int64_t d, int32_t dt, const int32_t *tok, const void *E,
                  int64_t vocab, int64_t lde, const int32_t *pos, const void *P, int64_t n_pos,
                  int64_t ldp, int64_t seq_len) {
  if (E) {
    if (vocab < 1 || vocab >= kMaxDim)
      return fail(SN_ERR_SHAPE, "vocab = %lld out of range", (long long)vocab);
    if (lde < d || lde >= kMaxDim) return fail(SN_ERR_SHAPE, "lde must be >= d");
    if (N > 0 && !tok) return fail(SN_ERR_NULL, "tok is NULL but E is given");
    if (!elem_aligned(E, dt)) return fail(SN_ERR_ALIGN, "E not aligned to its element size");
    if (tok && (reinterpret_cast<uintptr_t>(tok) & 3))
      return fail(SN_ERR_ALIGN, "tok not 4-byte aligned");
  }
  if (P) {
    if (n_pos < 1 || n_pos >= kMaxDim)
      return fail(SN_ERR_SHAPE, "n_pos = %lld out of range", (long long)n_pos);
    if (ldp < d || ldp >= kMaxDim) return fail(SN_ERR_SHAPE, "ldp must be >= d");
    if (!pos && (seq_len < 1 || seq_len > n_pos))
      return fail(SN_ERR_SHAPE, "pos is NULL: need 1 <= seq_len <= n_pos (seq_len = %lld)",
                  (long long)seq_len);
    if (!elem_aligned(P, dt)) return fail(SN_ERR_ALIGN, "P not aligned to its element size");
    if (pos && (reinterpret_cast<uintptr_t>(pos) & 3))
      return fail(SN_ERR_ALIGN, "pos not 4-byte aligned");
  }
  return SN_OK;
}

// The output span must not overlap any input span.
int32_t check_out_alias(Span out, const void *basis, size_t basis_bytes, Span in, int64_t N,
                        const int32_t *tok, const void *E, int64_t vocab, int64_t lde,
                        const int32_t *pos, const void *P, int64_t n_pos, int64_t ldp,
                        int64_t d, size_t es) {
  Span b;
  b.lo = reinterpret_cast<uintptr_t>(basis);
  b.hi = b.lo + basis_bytes;
  if (overlap(out, b)) return fail(SN_ERR_ALIAS, "output overlaps the packed basis");
  if (overlap(out, in)) return fail(SN_ERR_ALIAS, "output overlaps the input matrix");
  if (E && overlap(out, span(E, vocab, d, lde, es)))
    return fail(SN_ERR_ALIAS, "output overlaps E");
  if (P && overlap(out, span(P, n_pos, d, ldp, es)))
    return fail(SN_ERR_ALIAS, "output overlaps P");
  if (E && tok && overlap(out, span(tok, 1, N, N, 4)))
    return fail(SN_ERR_ALIAS, "output overlaps tok");
  if (P && pos && overlap(out, span(pos, 1, N, N, 4)))
    return fail(SN_ERR_ALIAS, "output overlaps pos");
  return SN_OK;
}

Span bytes_span(const void *p, size_t n) {
  Span s;
  if (!p || n == 0) return s;
  s.lo = reinterpret_cast<uintptr_t>(p);
  s.hi = s.lo + n;
  return s;
}

int32_t check_state(const void *state, int64_t d, int64_t k) {
  if (!state) return fail(SN_ERR_NULL, "state is NULL");
  if (reinterpret_cast<uintptr_t>(state) & 255)
    return fail(SN_ERR_ALIGN, "state must be 256-byte aligned");
  if (k > sn::kGrassMaxK)
    return fail(SN_ERR_UNSUPPORTED, "subspace update needs k <= %d", sn::kGrassMaxK);
  (void)d;
  return SN_OK;
}

int32_t check_workspace(const void *ws, size_t have, size_t need) {
  if (!ws) return fail(SN_ERR_NULL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) & 255)
    return fail(SN_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (have < need) return fail(SN_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", have, need);
  return SN_OK;
}

sn::IdArgs make_ids(const int32_t *tok, const void *E, int64_t vocab, int64_t lde,
                    const int32_t *pos, const void *P, int64_t n_pos, int64_t ldp,
                    int64_t seq_len, int32_t *err_flag) {
  sn::IdArgs a;
  a.E = E;
  a.tok = E ? tok : nullptr;
  a.vocab = vocab;
  a.lde = lde;
  a.P = P;
  a.pos = P ? pos : nullptr;
  a.n_pos = n_pos;
  a.ldp = ldp;
  a.seq_len = (P && !pos) ? seq_len : 1;
  a.err_flag = err_flag;
  return a;
}

}  // namespace

namespace sn {

int32_t project_args_check(const void *basis, int64_t d, int64_t k, int32_t dt, const void *W,
                           int64_t m, int64_t ldw) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (m < 0 || m >= kMaxDim) return fail(SN_ERR_SHAPE, "m out of range");
  if (ldw < m || ldw >= kMaxDim) return fail(SN_ERR_SHAPE, "ldw must be >= m");
  if (m == 0) return ok();
  if (!W) return fail(SN_ERR_NULL, "W is NULL");
  if (!elem_aligned(W, dt)) return fail(SN_ERR_ALIGN, "W not aligned to its element size");
  return ok();
}

}  // namespace sn

extern "C" {

size_t sn_basis_packed_bytes(int64_t d, int64_t k, int32_t dt) {
  if (!dtype_ok(dt) || d < 1 || d >= kMaxDim || k < 1 || k > d || k > SN_MAX_K) return 0;
  return sn::pack_layout(d, k, dt).total;
}

int32_t sn_basis_pack(const void *U, int64_t d, int64_t k, int64_t ldu, int32_t dt, void *packed,
                      size_t packed_bytes, sn_stream stream) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  if (!U || !packed) return fail(SN_ERR_NULL, "U or packed is NULL");
  if (d < 1 || d >= kMaxDim) return fail(SN_ERR_SHAPE, "d out of range");
  if (k < 1 || k > d) return fail(SN_ERR_SHAPE, "need 1 <= k <= d");
  if (k > SN_MAX_K) return fail(SN_ERR_UNSUPPORTED, "k > SN_MAX_K");
  if (ldu < k || ldu >= kMaxDim) return fail(SN_ERR_SHAPE, "ldu must be >= k");
  if (!elem_aligned(U, dt)) return fail(SN_ERR_ALIGN, "U not aligned to its element size");
  if (reinterpret_cast<uintptr_t>(packed) & 255)
    return fail(SN_ERR_ALIGN, "packed must be 256-byte aligned");
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  if (packed_bytes < L.total)
    return fail(SN_ERR_WORKSPACE, "packed buffer has %zu bytes, needs %zu", packed_bytes, L.total);
  Span pu;
  pu.lo = reinterpret_cast<uintptr_t>(packed);
  pu.hi = pu.lo + L.total;
  if (overlap(pu, span(U, d, k, ldu, elem_size(dt))))
    return fail(SN_ERR_ALIAS, "packed overlaps U");
  return hip_status(sn::launch_pack(L, U, ldu, packed, static_cast<hipStream_t>(stream)),
                    "sn_basis_pack launch");
}

int32_t sn_compress(const void *basis, int64_t d, int64_t k, int32_t dt, const void *X, int64_t N,
                    int64_t ldx, const int32_t *tok, const void *E, int64_t vocab, int64_t lde,
                    const int32_t *pos, const void *P, int64_t n_pos, int64_t ldp,
                    int64_t seq_len, void *C, int64_t ldc, int32_t *err_flag, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (ldx < d || ldx >= kMaxDim) return fail(SN_ERR_SHAPE, "ldx must be >= d");
  if (ldc < k || ldc >= kMaxDim) return fail(SN_ERR_SHAPE, "ldc must be >= k");
  if ((st = check_ids(N, d, dt, tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len))) return st;
  if (N == 0) return ok();
  if (!X || !C) return fail(SN_ERR_NULL, "X or C is NULL");
  if (!elem_aligned(X, dt) || !elem_aligned(C, dt))
    return fail(SN_ERR_ALIGN, "X or C not aligned to its element size");
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  if ((st = check_out_alias(span(C, N, k, ldc, es), basis, L.total, span(X, N, d, ldx, es), N,
                            tok, E, vocab, lde, pos, P, n_pos, ldp, d, es)))
    return st;
  const sn::IdArgs ids = make_ids(tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len, err_flag);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(sn::launch_compress(L, basis, X, N, ldx, ids, C, ldc, s),
                    "sn_compress launch");
}

int32_t sn_decompress(const void *basis, int64_t d, int64_t k, int32_t dt, const void *C,
                      int64_t N, int64_t ldc, const int32_t *tok, const void *E, int64_t vocab,
                      int64_t lde, const int32_t *pos, const void *P, int64_t n_pos, int64_t ldp,
                      int64_t seq_len, void *X, int64_t ldx, int32_t *err_flag,
                      sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (ldx < d || ldx >= kMaxDim) return fail(SN_ERR_SHAPE, "ldx must be >= d");
  if (ldc < k || ldc >= kMaxDim) return fail(SN_ERR_SHAPE, "ldc must be >= k");
  if ((st = check_ids(N, d, dt, tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len))) return st;
  if (N == 0) return ok();
  if (!X || !C) return fail(SN_ERR_NULL, "X or C is NULL");
  if (!elem_aligned(X, dt) || !elem_aligned(C, dt))
    return fail(SN_ERR_ALIGN, "X or C not aligned to its element size");
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  if ((st = check_out_alias(span(X, N, d, ldx, es), basis, L.total, span(C, N, k, ldc, es), N,
                            tok, E, vocab, lde, pos, P, n_pos, ldp, d, es)))
    return st;
  const sn::IdArgs ids = make_ids(tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len, err_flag);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (sn::decompress_mfma_ok(L, X, ldx, ids))
    return hip_status(sn::launch_decompress_mfma(L, basis, C, N, ldc, ids, X, ldx, s),
                      "sn_decompress launch");
  return hip_status(sn::launch_decompress_generic(L, basis, C, N, ldc, ids, X, ldx, s),
                    "sn_decompress launch");
}

int32_t sn_grad_compress(const void *basis, int64_t d, int64_t k, int32_t dt, const void *G,
                         int64_t N, int64_t ldg, void *Cg, int64_t ldc, sn_stream stream) {
  return sn_compress(basis, d, k, dt, G, N, ldg, nullptr, nullptr, 0, 0, nullptr, nullptr, 0, 0,
                     0, Cg, ldc, nullptr, stream);
}

size_t sn_embed_projected_bytes(int64_t k, int64_t vocab, int64_t n_pos) {
  if (k < 1 || k > SN_MAX_K || vocab < 0 || vocab >= kMaxDim || n_pos < 0 || n_pos >= kMaxDim)
    return 0;
  return sn::proj_layout(k, vocab, n_pos).total;
}

int32_t sn_embed_project(const void *basis, int64_t d, int64_t k, int32_t dt, const void *E,
                         int64_t vocab, int64_t lde, const void *P, int64_t n_pos, int64_t ldp,
                         void *proj, size_t proj_bytes, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (vocab < 0 || vocab >= kMaxDim) return fail(SN_ERR_SHAPE, "vocab out of range");
  if (n_pos < 0 || n_pos >= kMaxDim) return fail(SN_ERR_SHAPE, "n_pos out of range");
  if ((vocab > 0) != (E != nullptr)) return fail(SN_ERR_NULL, "E must be given iff vocab > 0");
  if ((n_pos > 0) != (P != nullptr)) return fail(SN_ERR_NULL, "P must be given iff n_pos > 0");
  if (E && (lde < d || lde >= kMaxDim)) return fail(SN_ERR_SHAPE, "lde must be >= d");
  if (P && (ldp < d || ldp >= kMaxDim)) return fail(SN_ERR_SHAPE, "ldp must be >= d");
  if ((E && !elem_aligned(E, dt)) || (P && !elem_aligned(P, dt)))
    return fail(SN_ERR_ALIGN, "E or P not aligned to its element size");
  const sn::ProjLayout PL = sn::proj_layout(k, vocab, n_pos);
  if (PL.total == 0) return ok();
  if (!proj) return fail(SN_ERR_NULL, "proj is NULL");
  if (reinterpret_cast<uintptr_t>(proj) & 255)
    return fail(SN_ERR_ALIGN, "proj must be 256-byte aligned");
  if (proj_bytes < PL.total)
    return fail(SN_ERR_WORKSPACE, "proj has %zu bytes, needs %zu", proj_bytes, PL.total);
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  Span out;
  out.lo = reinterpret_cast<uintptr_t>(proj);
  out.hi = out.lo + PL.total;
  Span b;
  b.lo = reinterpret_cast<uintptr_t>(basis);
  b.hi = b.lo + L.total;
  if (overlap(out, b) || overlap(out, span(E, vocab, d, lde, es)) ||
      overlap(out, span(P, n_pos, d, ldp, es)))
    return fail(SN_ERR_ALIAS, "proj overlaps the basis, E or P");
  hipStream_t s = static_cast<hipStream_t>(stream);
  char *base = static_cast<char *>(proj);
  const struct {
    const void *t;
    int64_t rows, ld;
    size_t off;
  } parts[2] = {{E, vocab, lde, PL.off_eu}, {P, n_pos, ldp, PL.off_pu}};
  for (const auto &pt : parts) {
    if (pt.rows == 0) continue;
    float *o = reinterpret_cast<float *>(base + pt.off);
    const hipError_t e =
        sn::launch_table_project(L, basis, pt.t, pt.rows, pt.ld, o, PL.kp, s);
    if (e != hipSuccess) return hip_status(e, "sn_embed_project launch");
  }
  return ok();
}

int32_t sn_compress_projected(const void *basis, int64_t d, int64_t k, int32_t dt, const void *X,
                              int64_t N, int64_t ldx, const int32_t *tok, const int32_t *pos,
                              int64_t seq_len, const void *proj, int64_t vocab, int64_t n_pos,
                              void *C, int64_t ldc, int32_t *err_flag, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (ldx < d || ldx >= kMaxDim) return fail(SN_ERR_SHAPE, "ldx must be >= d");
  if (ldc < k || ldc >= kMaxDim) return fail(SN_ERR_SHAPE, "ldc must be >= k");
  if (vocab < 0 || vocab >= kMaxDim) return fail(SN_ERR_SHAPE, "vocab out of range");
  if (n_pos < 0 || n_pos >= kMaxDim) return fail(SN_ERR_SHAPE, "n_pos out of range");
  if ((vocab > 0 || n_pos > 0) && !proj) return fail(SN_ERR_NULL, "proj is NULL");
  if (proj && (reinterpret_cast<uintptr_t>(proj) & 255))
    return fail(SN_ERR_ALIGN, "proj must be 256-byte aligned");
  if (n_pos > 0 && !pos && (seq_len < 1 || seq_len > n_pos))
    return fail(SN_ERR_SHAPE, "pos is NULL: need 1 <= seq_len <= n_pos (seq_len = %lld)",
                (long long)seq_len);
  if ((tok && (reinterpret_cast<uintptr_t>(tok) & 3)) ||
      (pos && (reinterpret_cast<uintptr_t>(pos) & 3)))
    return fail(SN_ERR_ALIGN, "tok / pos not 4-byte aligned");
  if (N == 0) return ok();
  if (vocab > 0 && !tok) return fail(SN_ERR_NULL, "tok is NULL but vocab > 0");
  if (!X || !C) return fail(SN_ERR_NULL, "X or C is NULL");
  if (!elem_aligned(X, dt) || !elem_aligned(C, dt))
    return fail(SN_ERR_ALIGN, "X or C not aligned to its element size");
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const sn::ProjLayout PL = sn::proj_layout(k, vocab, n_pos);
  const Span out = span(C, N, k, ldc, es);
  Span b;
  b.lo = reinterpret_cast<uintptr_t>(basis);
  b.hi = b.lo + L.total;
  Span pj;
  if (proj) {
    pj.lo = reinterpret_cast<uintptr_t>(proj);
    pj.hi = pj.lo + PL.total;
  }
  if (overlap(out, b) || overlap(out, pj) || overlap(out, span(X, N, d, ldx, es)) ||
      (vocab > 0 && overlap(out, span(tok, 1, N, N, 4))) ||
      (n_pos > 0 && pos && overlap(out, span(pos, 1, N, N, 4))))
    return fail(SN_ERR_ALIAS, "C overlaps an input");
  const char *pb = static_cast<const char *>(proj);
  sn::ProjArgs pa{};
  pa.tok = vocab > 0 ? tok : nullptr;
  pa.eu = vocab > 0 ? reinterpret_cast<const float *>(pb + PL.off_eu) : nullptr;
  pa.vocab = vocab;
  pa.pos = n_pos > 0 ? pos : nullptr;
  pa.pu = n_pos > 0 ? reinterpret_cast<const float *>(pb + PL.off_pu) : nullptr;
  pa.n_pos = n_pos;
  pa.seq_len = (n_pos > 0 && !pos) ? seq_len : 1;
  pa.kp = PL.kp;
  pa.err_flag = err_flag;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(sn::launch_compress_projected(L, basis, X, N, ldx, pa, C, ldc, s),
                    "sn_compress_projected launch");
}

size_t sn_project_weights_workspace_bytes(int64_t d, int64_t k, int32_t dt, int64_t m) {
  if (!dtype_ok(dt) || d < 1 || d >= kMaxDim || k < 1 || k > d || k > SN_MAX_K || m < 0 ||
      m >= kMaxDim)
    return 0;
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  size_t a = sn::project_workspace_generic(d, k, m);
  size_t b = L.mfma ? sn::project_workspace_mfma(d, k, m) : 0;
  return sn::align256(a > b ? a : b);
}

int32_t sn_project_weights(const void *basis, int64_t d, int64_t k, int32_t dt, void *W,
                           int64_t m, int64_t ldw, void *workspace, size_t workspace_bytes,
                           sn_stream stream) {
  int32_t st = sn::project_args_check(basis, d, k, dt, W, m, ldw);
  if (st) return st;
  if (m == 0) return ok();
  if (!workspace) return fail(SN_ERR_NULL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255)
    return fail(SN_ERR_ALIGN, "workspace must be 256-byte aligned");
  const size_t need = sn_project_weights_workspace_bytes(d, k, dt, m);
  if (workspace_bytes < need)
    return fail(SN_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  Span w = span(W, d, m, ldw, elem_size(dt));
  Span ws;
  ws.lo = reinterpret_cast<uintptr_t>(workspace);
  ws.hi = ws.lo + need;
  Span b;
  b.lo = reinterpret_cast<uintptr_t>(basis);
  b.hi = b.lo + L.total;
  if (overlap(w, ws) || overlap(w, b) || overlap(ws, b))
    return fail(SN_ERR_ALIAS, "W, workspace and basis must not overlap");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (L.mfma && sn::project_mfma_ok(L, W, m, ldw))
    return hip_status(sn::launch_project_mfma(L, basis, W, m, ldw, workspace, s),
                      "sn_project_weights launch");
  return hip_status(sn::launch_project_generic(L, basis, W, m, ldw, workspace, s),
                    "sn_project_weights launch");
}

size_t sn_grassmann_state_bytes(int64_t d, int64_t k) {
  if (d < 1 || d >= kMaxDim || k < 1 || k > d || k > sn::kGrassMaxK) return 0;
  return sn::grass_state_bytes(d, k);
}

size_t sn_grassmann_workspace_bytes(int64_t d, int64_t k, int32_t dt, int64_t N) {
  if (!dtype_ok(dt) || d < 1 || d >= kMaxDim || k < 1 || k > d || k > sn::kGrassMaxK || N < 0 ||
      N >= kMaxDim)
    return 0;
  return sn::grass_workspace_bytes(sn::pack_layout(d, k, dt), N);
}

int32_t sn_grassmann_reset(void *state, int64_t d, int64_t k, sn_stream stream) {
  if (d < 1 || d >= kMaxDim || k < 1 || k > d) return fail(SN_ERR_SHAPE, "need 1 <= k <= d");
  int32_t st = check_state(state, d, k);
  if (st) return st;
  return hip_status(sn::launch_grass_reset(state, d, k, static_cast<hipStream_t>(stream)),
                    "sn_grassmann_reset launch");
}

int32_t sn_grassmann_accumulate(const void *basis, int64_t d, int64_t k, int32_t dt, const void *G,
                                int64_t N, int64_t ldg, void *Cg, int64_t ldc, int32_t with_su,
                                void *state, void *workspace, size_t workspace_bytes,
                                sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if ((st = check_state(state, d, k))) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N = %lld out of range", (long long)N);
  if (ldg < d || ldg >= kMaxDim) return fail(SN_ERR_SHAPE, "ldg must be >= d");
  if (Cg && (ldc < k || ldc >= kMaxDim)) return fail(SN_ERR_SHAPE, "ldc must be >= k");
  if (N == 0) return ok();
  if (!G) return fail(SN_ERR_NULL, "G is NULL");
  if (!elem_aligned(G, dt) || (Cg && !elem_aligned(Cg, dt)))
    return fail(SN_ERR_ALIGN, "G or Cg not aligned to its element size");
  const size_t need = sn_grassmann_workspace_bytes(d, k, dt, N);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const Span g = span(G, N, d, ldg, es), c = span(Cg, N, k, ldc, es);
  const Span b = bytes_span(basis, L.total), sb = bytes_span(state, sn::grass_state_bytes(d, k));
  const Span w = bytes_span(workspace, need);
  if (overlap(c, g) || overlap(c, b) || overlap(c, sb) || overlap(c, w))
    return fail(SN_ERR_ALIAS, "Cg overlaps an input, the state or the workspace");
  if (overlap(sb, g) || overlap(sb, b) || overlap(sb, w))
    return fail(SN_ERR_ALIAS, "state overlaps G, the basis or the workspace");
  if (overlap(w, g) || overlap(w, b))
    return fail(SN_ERR_ALIAS, "workspace overlaps G or the basis");
  return hip_status(sn::launch_grass_accumulate(L, basis, G, N, ldg, Cg, ldc, with_su != 0, state,
                                                workspace, static_cast<hipStream_t>(stream)),
                    "sn_grassmann_accumulate launch");
}

int32_t sn_grassmann_step(const void *basis, int64_t d, int64_t k, int32_t dt, const void *state,
                          double eta, void *U_new, int64_t ldu, int32_t out_dt, void *workspace,
                          size_t workspace_bytes, int32_t *err_flag, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if ((st = check_state(state, d, k))) return st;
  if (!dtype_ok(out_dt)) return fail(SN_ERR_DTYPE, "unknown out_dt %d", out_dt);
  if (!(eta >= 0.0) || eta > 1e300) return fail(SN_ERR_SHAPE, "eta must be finite and >= 0");
  if (!U_new) return fail(SN_ERR_NULL, "U_new is NULL");
  if (ldu < k || ldu >= kMaxDim) return fail(SN_ERR_SHAPE, "ldu must be >= k");
  if (!elem_aligned(U_new, out_dt)) return fail(SN_ERR_ALIGN, "U_new not aligned");
  if (err_flag && (reinterpret_cast<uintptr_t>(err_flag) & 3))
    return fail(SN_ERR_ALIGN, "err_flag not 4-byte aligned");
  const size_t need = sn_grassmann_workspace_bytes(d, k, dt, 0);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const Span u = span(U_new, d, k, ldu, elem_size(out_dt));
  const Span b = bytes_span(basis, L.total), sb = bytes_span(state, sn::grass_state_bytes(d, k));
  const Span w = bytes_span(workspace, need);
  if (overlap(u, b) || overlap(u, sb) || overlap(u, w))
    return fail(SN_ERR_ALIAS, "U_new overlaps the basis, the state or the workspace");
  if (overlap(w, b) || overlap(w, sb))
    return fail(SN_ERR_ALIAS, "workspace overlaps the basis or the state");
  return hip_status(sn::launch_grass_step(L, basis, state, eta, U_new, ldu, out_dt, workspace,
                                          err_flag, static_cast<hipStream_t>(stream)),
                    "sn_grassmann_step launch");
}

size_t sn_embed_lowrank_workspace_bytes(int64_t d, int64_t k, int32_t dt, int64_t N,
                                        int64_t vocab) {
  if (!dtype_ok(dt) || d < 1 || d >= kMaxDim || k < 1 || k > d || k > SN_MAX_K || N < 0 ||
      N >= kMaxDim || vocab < 1 || vocab >= kMaxDim)
    return 0;
  return sn::embed_workspace_bytes(k, dt, N, vocab);
}

int32_t sn_embed_lowrank_forward(const void *basis, int64_t d, int64_t k, int32_t dt,
                                 const void *CS, int64_t vocab, int64_t ldcs, const int32_t *tok,
                                 const void *E, int64_t lde, const int32_t *pos, const void *P,
                                 int64_t n_pos, int64_t ldp, int64_t seq_len, void *X0,
                                 int64_t N, int64_t ldx, int32_t *err_flag, void *workspace,
                                 size_t workspace_bytes, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N out of range");
  if (vocab < 1 || vocab >= kMaxDim) return fail(SN_ERR_SHAPE, "vocab out of range");
  if (ldcs < k || ldcs >= kMaxDim) return fail(SN_ERR_SHAPE, "ldcs must be >= k");
  if (ldx < d || ldx >= kMaxDim) return fail(SN_ERR_SHAPE, "ldx must be >= d");
  if ((st = check_ids(N, d, dt, tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len))) return st;
  if (N == 0) return ok();
  if (!CS || !tok || !X0) return fail(SN_ERR_NULL, "CS, tok and X0 are required");
  if (!elem_aligned(CS, dt) || !elem_aligned(X0, dt) || (reinterpret_cast<uintptr_t>(tok) & 3))
    return fail(SN_ERR_ALIGN, "CS, X0 or tok misaligned");
  const size_t need = sn_embed_lowrank_workspace_bytes(d, k, dt, N, vocab);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  const size_t es = elem_size(dt);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const Span x = span(X0, N, d, ldx, es), w = bytes_span(workspace, need);
  if ((st = check_out_alias(x, basis, L.total, span(CS, vocab, k, ldcs, es), N, tok, E, vocab,
                            lde, pos, P, n_pos, ldp, d, es)))
    return st;
  if (overlap(x, span(tok, 1, N, N, 4)) || overlap(x, w) || overlap(w, span(CS, vocab, k, ldcs, es)) ||
      overlap(w, span(tok, 1, N, N, 4)) || overlap(w, bytes_span(basis, L.total)) ||
      (E && overlap(w, span(E, vocab, d, lde, es))) || (P && overlap(w, span(P, n_pos, d, ldp, es))))
    return fail(SN_ERR_ALIAS, "X0 or the workspace overlaps an input");
  const sn::IdArgs ids = make_ids(tok, E, vocab, lde, pos, P, n_pos, ldp, seq_len, err_flag);
  return hip_status(sn::launch_embed_forward(L, basis, CS, vocab, ldcs, tok, ids, N, X0, ldx,
                                             workspace, static_cast<hipStream_t>(stream)),
                    "sn_embed_lowrank_forward launch");
}

int32_t sn_embed_lowrank_backward(const void *basis, int64_t d, int64_t k, int32_t dt,
                                  const void *dX0, int64_t N, int64_t ldg, const int32_t *tok,
                                  int64_t vocab, float *gCS, int64_t ldgc, int32_t *err_flag,
                                  void *workspace, size_t workspace_bytes, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (N < 0 || N >= kMaxDim) return fail(SN_ERR_SHAPE, "N out of range");
  if (vocab < 1 || vocab >= kMaxDim) return fail(SN_ERR_SHAPE, "vocab out of range");
  if (ldg < d || ldg >= kMaxDim) return fail(SN_ERR_SHAPE, "ldg must be >= d");
  if (ldgc < k || ldgc >= kMaxDim) return fail(SN_ERR_SHAPE, "ldgc must be >= k");
  if (vocab >= (int64_t(1) << 21))
    return fail(SN_ERR_UNSUPPORTED, "the gradient scatter sorts ids below 2^21 (vocab = %lld)",
                (long long)vocab);
  if (N == 0) return ok();
  if (!dX0 || !tok || !gCS) return fail(SN_ERR_NULL, "dX0, tok and gCS are required");
  if (!elem_aligned(dX0, dt) || !elem_aligned(gCS, SN_F32) ||
      (reinterpret_cast<uintptr_t>(tok) & 3))
    return fail(SN_ERR_ALIGN, "dX0, gCS or tok misaligned");
  const size_t need = sn_embed_lowrank_workspace_bytes(d, k, dt, N, vocab);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const Span g = span(gCS, vocab, k, ldgc, 4), w = bytes_span(workspace, need);
  const Span x = span(dX0, N, d, ldg, elem_size(dt)), t = span(tok, 1, N, N, 4);
  const Span b = bytes_span(basis, L.total);
  if (overlap(g, x) || overlap(g, t) || overlap(g, w) || overlap(g, b) || overlap(w, x) ||
      overlap(w, t) || overlap(w, b))
    return fail(SN_ERR_ALIAS, "gCS, the workspace and the inputs must not overlap");
  return hip_status(sn::launch_embed_backward(L, basis, dX0, N, ldg, tok, vocab, gCS, ldgc,
                                              err_flag, workspace,
                                              static_cast<hipStream_t>(stream)),
                    "sn_embed_lowrank_backward launch");
}

size_t sn_adamw_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || rows >= kMaxDim || cols < 0 || cols >= kMaxDim) return 0;
  return sn::adamw_workspace_bytes(rows, cols);
}

int32_t sn_adamw_step(void *W, int64_t ldw, const void *G, int64_t ldg, int32_t dt, float *M,
                      float *V, int64_t ldm, int64_t rows, int64_t cols, int64_t t, double lr,
                      double beta1, double beta2, double eps, double weight_decay,
                      int32_t subspace, void *workspace, size_t workspace_bytes,
                      sn_stream stream) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  if (rows < 0 || rows >= kMaxDim || cols < 0 || cols >= kMaxDim)
    return fail(SN_ERR_SHAPE, "rows / cols out of range");
  if (t < 1) return fail(SN_ERR_SHAPE, "t counts steps from 1 (t = %lld)", (long long)t);
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(SN_ERR_SHAPE, "betas must lie in [0, 1)");
  if (!(eps >= 0.0 && eps <= 1e30) || !(lr >= 0.0 && lr <= 1e30) ||
      !(weight_decay >= 0.0 && weight_decay <= 1e30))
    return fail(SN_ERR_SHAPE, "lr, eps and weight_decay must be finite and >= 0");
  if (rows == 0 || cols == 0) return ok();
  if (ldw < cols || ldg < cols || ldm < cols || ldw >= kMaxDim || ldg >= kMaxDim ||
      ldm >= kMaxDim)
    return fail(SN_ERR_SHAPE, "row strides must be >= cols");
  if (!W || !G || !M || !V) return fail(SN_ERR_NULL, "W, G, M and V are required");
  if (!elem_aligned(W, dt) || !elem_aligned(G, dt) || !elem_aligned(M, SN_F32) ||
      !elem_aligned(V, SN_F32))
    return fail(SN_ERR_ALIGN, "W, G, M or V not aligned to its element size");
  int32_t st;
  const size_t need = subspace ? sn_adamw_workspace_bytes(rows, cols) : 0;
  if (subspace && (st = check_workspace(workspace, workspace_bytes, need))) return st;
  const size_t es = elem_size(dt);
  const Span w = span(W, rows, cols, ldw, es), g = span(G, rows, cols, ldg, es);
  const Span m = span(M, rows, cols, ldm, 4), v = span(V, rows, cols, ldm, 4);
  const Span ws = subspace ? bytes_span(workspace, need) : Span{};
  const Span all[5] = {w, g, m, v, ws};
  for (int i = 0; i < 5; ++i)
    for (int j = i + 1; j < 5; ++j)
      if (overlap(all[i], all[j]))
        return fail(SN_ERR_ALIAS, "W, G, M, V and the workspace must not overlap");
  return hip_status(sn::launch_adamw(dt, W, ldw, G, ldg, M, V, ldm, rows, cols, t, lr, beta1,
                                     beta2, eps, weight_decay, subspace != 0, workspace,
                                     static_cast<hipStream_t>(stream)),
                    "sn_adamw_step launch");
}

namespace {

// The segmented (one set of launches) form applies when every matrix meets
// the MFMA path's conditions with a width that is a multiple of 256.
bool multi_segmented(const sn::PackLayout &L, int32_t count, void *const *W, const int64_t *m,
                     const int64_t *ldw) {
  if (!L.mfma || L.ks2 == 0 || count < 1 || count > sn::kMaxSeg) return false;
  for (int32_t i = 0; i < count; ++i)
    if (m[i] % 256 != 0 || !sn::project_mfma_ok(L, W[i], m[i], ldw[i])) return false;
  return true;
}

}  // namespace

size_t sn_project_weights_multi_workspace_bytes(int64_t d, int64_t k, int32_t dt, int32_t count,
                                                const int64_t *m) {
  if (!dtype_ok(dt) || d < 1 || d >= kMaxDim || k < 1 || k > d || k > SN_MAX_K || count < 0 ||
      count > SN_PROJECT_MAX_MATRICES || (count > 0 && !m))
    return 0;
  size_t best = 0;
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (m[i] < 0 || m[i] >= kMaxDim) return 0;
    const size_t one = sn_project_weights_workspace_bytes(d, k, dt, m[i]);
    best = one > best ? one : best;
    total += m[i];
  }
  if (total >= kMaxDim) return 0;
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  if (L.mfma && total > 0) {
    const size_t seg = sn::align256(sn::project_workspace_mfma(d, k, total));
    best = seg > best ? seg : best;
  }
  return best;
}

int32_t sn_project_weights_multi(const void *basis, int64_t d, int64_t k, int32_t dt, int32_t count,
                                 void *const *W, const int64_t *m, const int64_t *ldw,
                                 void *workspace, size_t workspace_bytes, sn_stream stream) {
  int32_t st = check_basis(basis, d, k, dt);
  if (st) return st;
  if (count < 0 || count > SN_PROJECT_MAX_MATRICES)
    return fail(SN_ERR_SHAPE, "count must lie in [0, %d]", SN_PROJECT_MAX_MATRICES);
  if (count == 0) return ok();
  if (!W || !m || !ldw) return fail(SN_ERR_NULL, "W, m and ldw arrays are required");
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (m[i] < 0 || m[i] >= kMaxDim) return fail(SN_ERR_SHAPE, "m[%d] out of range", i);
    if (ldw[i] < m[i] || ldw[i] >= kMaxDim) return fail(SN_ERR_SHAPE, "ldw[%d] must be >= m[%d]", i, i);
    if (m[i] > 0 && !W[i]) return fail(SN_ERR_NULL, "W[%d] is NULL", i);
    if (m[i] > 0 && !elem_aligned(W[i], dt)) return fail(SN_ERR_ALIGN, "W[%d] misaligned", i);
    total += m[i];
  }
  if (total >= kMaxDim) return fail(SN_ERR_SHAPE, "total width out of range");
  if (total == 0) return ok();
  if (!workspace) return fail(SN_ERR_NULL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255)
    return fail(SN_ERR_ALIGN, "workspace must be 256-byte aligned");
  const size_t need = sn_project_weights_multi_workspace_bytes(d, k, dt, count, m);
  if (workspace_bytes < need)
    return fail(SN_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
  const sn::PackLayout L = sn::pack_layout(d, k, dt);
  const size_t es = elem_size(dt);
  const Span ws = bytes_span(workspace, need), b = bytes_span(basis, L.total);
  if (overlap(ws, b)) return fail(SN_ERR_ALIAS, "workspace overlaps the basis");
  for (int32_t i = 0; i < count; ++i) {
    const Span wi = span(W[i], d, m[i], ldw[i], es);
    if (overlap(wi, ws) || overlap(wi, b))
      return fail(SN_ERR_ALIAS, "W[%d] overlaps the workspace or the basis", i);
    for (int32_t j = 0; j < i; ++j)
      if (overlap(wi, span(W[j], d, m[j], ldw[j], es)))
        return fail(SN_ERR_ALIAS, "W[%d] overlaps W[%d]", i, j);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (multi_segmented(L, count, W, m, ldw)) {
    sn::ColSegs cs;
    cs.n = 0;
    int64_t c0 = 0;
    for (int32_t i = 0; i < count; ++i) {
      if (m[i] == 0) continue;
      cs.c0[cs.n] = c0;
      cs.base[cs.n] = W[i];
      cs.ld[cs.n] = ldw[i];
      ++cs.n;
      c0 += m[i];
    }
    cs.c0[cs.n] = c0;
    return hip_status(sn::launch_project_mfma_segs(L, basis, cs, workspace, s),
                      "sn_project_weights_multi launch");
  }
  for (int32_t i = 0; i < count; ++i) {  // one after another, sharing the workspace
    if (m[i] == 0) continue;
    if ((st = sn_project_weights(basis, d, k, dt, W[i], m[i], ldw[i], workspace, workspace_bytes,
                                 stream)))
      return st;
  }
  return ok();
}

}  // extern "C"

// ---- token log probabilities, norms, gradient clipping ---------------------

namespace {

int32_t check_rows(const char *name, int64_t n, int64_t cols, int64_t ld) {
  if (n < 0 || n >= kMaxDim || cols < 1 || cols >= kMaxDim)
    return fail(SN_ERR_SHAPE, "%s: %lld x %lld out of range", name, (long long)n, (long long)cols);
  if (ld < cols || ld >= kMaxDim)
    return fail(SN_ERR_SHAPE, "%s: the row stride must be >= the columns", name);
  return SN_OK;
}

int32_t check_scale(double scale) {
  if (!(scale >= 0x1p-20 && scale <= 0x1p20))
    return fail(SN_ERR_SHAPE, "scale must lie in [2^-20, 2^20]");
  return SN_OK;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The buffers of a call, for the checks that no output overlaps another buffer.
struct Buffers {
  static constexpr int kMost = 16;
  Span in[kMost], out[kMost];
  int ins = 0, outs = 0;
  void read(Span s) { in[ins++] = s; }
  void write(Span s) { out[outs++] = s; }
  int32_t check(const char *call) const {
    for (int i = 0; i < outs; ++i) {
      for (int j = 0; j < ins; ++j)
        if (overlap(out[i], in[j])) return fail(SN_ERR_ALIAS, "%s: an output overlaps an input", call);
      for (int j = 0; j < i; ++j)
        if (overlap(out[i], out[j])) return fail(SN_ERR_ALIAS, "%s: two outputs overlap", call);
    }
    return SN_OK;
  }
};

// What the calls on logits share.
int32_t check_logits(const void *Z, int64_t N, int64_t V, int64_t ldz, int32_t dt, double scale,
                     const int32_t *tok) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  int32_t st = check_rows("Z", N, V, ldz);
  if (st || (st = check_scale(scale))) return st;
  if (N == 0) return SN_OK;
  if (!Z) return fail(SN_ERR_NULL, "Z is NULL");
  if (!elem_aligned(Z, dt)) return fail(SN_ERR_ALIGN, "Z not aligned to its element size");
  if (!aligned(tok, 4)) return fail(SN_ERR_ALIGN, "tok not 4-byte aligned");
  return SN_OK;
}

int32_t check_dlogits(const void *Z, int64_t N, int64_t V, int64_t ldz, int32_t dt, void *dZ,
                      int64_t lddz, Buffers &b) {
  if (lddz < V || lddz >= kMaxDim) return fail(SN_ERR_SHAPE, "lddz must be >= V");
  if (N == 0) return SN_OK;
  if (!dZ) return fail(SN_ERR_NULL, "dZ is NULL");
  if (!elem_aligned(dZ, dt)) return fail(SN_ERR_ALIGN, "dZ not aligned to its element size");
  b.write(span(dZ, N, V, lddz, elem_size(dt)));
  if (dZ != Z || lddz != ldz) b.read(span(Z, N, V, ldz, elem_size(dt)));
  return SN_OK;
}

// H, X, R and w of the norm's forward calls; adds them to the buffers.
int32_t check_norm(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt, const void *R,
                   int64_t ldr, const void *w, double eps, void *H, int64_t ldh, Buffers &b) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  int32_t st = check_rows("X", N, d, ldx);
  if (st || (R && (st = check_rows("R", N, d, ldr))) || (H && (st = check_rows("H", N, d, ldh))))
    return st;
  if (!(eps >= 0.0 && eps <= 3.0e38)) return fail(SN_ERR_SHAPE, "eps must be finite and >= 0");
  if (N == 0) return SN_OK;
  if (!X) return fail(SN_ERR_NULL, "X is NULL");
  if (!elem_aligned(X, dt) || !elem_aligned(R, dt) || !elem_aligned(w, dt) || !elem_aligned(H, dt))
    return fail(SN_ERR_ALIGN, "X, R, w or H not aligned to its element size");
  const size_t es = elem_size(dt);
  const bool on_x = H == X && ldh == ldx, on_r = H == R && ldh == ldr;
  if (H) b.write(span(H, N, d, ldh, es));
  if (!H || !on_x) b.read(span(X, N, d, ldx, es));
  if (R && (!H || !on_r)) b.read(span(R, N, d, ldr, es));
  b.read(span(w, 1, d, d, es));
  return SN_OK;
}

sn::NormArgs norm_args(const void *X, int64_t N, int64_t d, int64_t ldx, const void *R,
                       int64_t ldr, const void *w, double eps, void *H, int64_t ldh) {
  sn::NormArgs a = {};
  a.X = X;
  a.R = R;
  a.w = w;
  a.N = N;
  a.d = d;
  a.ldx = ldx;
  a.ldr = ldr;
  a.inv_d = static_cast<float>(1.0 / static_cast<double>(d));
  a.eps = static_cast<float>(eps);
  a.H = H;
  a.ldh = ldh;
  return a;
}

// The tensors of a clipping call as the kernels take them, checked: rows without gaps
// as one row, and tensors without elements left out.
int32_t clip_tensors(int32_t count, const sn_tensor *grads, const sn_tensor *out, bool shapes_only,
                     std::vector<sn::ClipTensor> &t) {
  if (count < 0) return fail(SN_ERR_SHAPE, "count must be >= 0");
  if (count > 0 && !grads) return fail(SN_ERR_NULL, "grads is NULL");
  t.reserve(static_cast<size_t>(count));
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) {
    const sn_tensor &g = grads[i];
    if (!dtype_ok(g.dt)) return fail(SN_ERR_DTYPE, "grads[%d]: unknown dtype %d", i, g.dt);
    if (g.rows < 0 || g.rows >= kMaxDim || g.cols < 0 || g.cols >= kMaxElems)
      return fail(SN_ERR_SHAPE, "grads[%d]: %lld x %lld out of range", i, (long long)g.rows,
                  (long long)g.cols);
    if (out && (out[i].rows != g.rows || out[i].cols != g.cols))
      return fail(SN_ERR_SHAPE, "out[%d] has another shape than grads[%d]", i, i);
    if (out && out[i].dt != g.dt)
      return fail(SN_ERR_DTYPE, "out[%d] has another dtype than grads[%d]", i, i);
    if (g.rows == 0 || g.cols == 0) continue;
    // rows < 2^31 and cols < 2^40: compared without their product
    if (g.cols > (kMaxElems - 1) / g.rows || (total += g.rows * g.cols) >= kMaxElems)
      return fail(SN_ERR_SHAPE, "2^40 or more elements");
    const int64_t ldo = out ? out[i].ld : g.ld;
    if (g.rows > 1 && (g.ld < g.cols || g.ld >= kMaxElems || ldo < g.cols || ldo >= kMaxElems))
      return fail(SN_ERR_SHAPE, "tensor %d: the row stride must be >= the columns", i);
    sn::ClipTensor c = {};
    c.g = g.data;
    c.out = out ? out[i].data : g.data;
    if (!shapes_only) {
      if (!c.g || !c.out) return fail(SN_ERR_NULL, "tensor %d is NULL", i);
      if (!elem_aligned(c.g, g.dt) || !elem_aligned(c.out, g.dt))
        return fail(SN_ERR_ALIGN, "tensor %d not aligned to its element size", i);
    }
    const bool gaps = g.rows > 1 && (g.ld != g.cols || ldo != g.cols);
    c.rows = gaps ? g.rows : 1;
    c.cols = gaps ? g.cols : g.rows * g.cols;
    c.ldg = gaps ? g.ld : c.cols;
    c.ldo = gaps ? ldo : c.cols;
    c.f32 = g.dt == SN_F32;
    t.push_back(c);
  }
  return SN_OK;
}

Span clip_span(const sn::ClipTensor &c, bool out) {
  return span(out ? c.out : c.g, c.rows, c.cols, out ? c.ldo : c.ldg, c.f32 ? 4 : 2);
}

// A gradient or output among the others of a clipping call.
struct ClipItem {
  Span s;
  bool out;
  int32_t tensor;
};

// Whether two tensors share an element, a the one that starts first.  Rows of one stride
// (a single row fits any stride that holds it) are compared exactly, so that column
// blocks of one matrix are told apart; of others the extents are.
bool share(const std::vector<sn::ClipTensor> &t, const ClipItem &a, const ClipItem &b) {
  if (!overlap(a.s, b.s)) return false;
  struct Rows {
    uintptr_t n, len, step;  // n rows of len bytes, one each step bytes
  };
  const auto rows = [&](const ClipItem &x) {
    const sn::ClipTensor &c = t[static_cast<size_t>(x.tensor)];
    const int64_t es = c.f32 ? 4 : 2;
    return Rows{static_cast<uintptr_t>(c.rows), static_cast<uintptr_t>(c.cols * es),
                static_cast<uintptr_t>((x.out ? c.ldo : c.ldg) * es)};
  };
  const Rows ra = rows(a), rb = rows(b);
  const uintptr_t step = ra.n > 1 ? ra.step : rb.step;
  if ((ra.n == 1 && rb.n == 1) || (ra.n > 1 && rb.n > 1 && ra.step != rb.step) ||
      ra.len > step || rb.len > step)
    return true;
  // b's first row starts in a's row q at byte r, and ends in row q + 1 where it is longer
  // than what row q has left
  const uintptr_t q = (b.s.lo - a.s.lo) / step, r = (b.s.lo - a.s.lo) % step;
  return (q < ra.n && r < ra.len) || (q + 1 < ra.n && r + rb.len > step);
}

// No output may share an element with another tensor's gradient or output: with the
// extents in order of their starts, each against the extents before it.
int32_t check_clip_alias(const std::vector<sn::ClipTensor> &t) {
  // Lists that are in the order of their addresses, as gradients allocated one after the
  // other are, need no sorting.
  std::vector<ClipItem> gs, os, v;
  gs.reserve(t.size());
  os.reserve(t.size());
  for (const sn::ClipTensor &c : t) {
    const int32_t i = static_cast<int32_t>(&c - t.data());
    os.push_back({clip_span(c, true), true, i});
    if (c.out != c.g || c.ldo != c.ldg) gs.push_back({clip_span(c, false), false, i});
  }
  const auto below = [](const ClipItem &a, const ClipItem &b) { return a.s.lo < b.s.lo; };
  for (std::vector<ClipItem> *l : {&gs, &os})
    if (!std::is_sorted(l->begin(), l->end(), below)) std::sort(l->begin(), l->end(), below);
  v.reserve(gs.size() + os.size());
  std::merge(gs.begin(), gs.end(), os.begin(), os.end(), std::back_inserter(v), below);
  uintptr_t any = 0, outs = 0;  // the furthest end of an extent, of an output's extent
  bool apart = true;
  for (const ClipItem &x : v) {
    apart = apart && x.s.lo >= (x.out ? any : outs);
    any = x.s.hi > any ? x.s.hi : any;
    if (x.out) outs = x.s.hi > outs ? x.s.hi : outs;
  }
  if (apart) return SN_OK;
  // extents that overlap: each pair of them
  std::vector<ClipItem> open;  // those that reach past the present one's start
  for (const ClipItem &x : v) {
    const auto ended = [&](const ClipItem &y) { return y.s.hi <= x.s.lo; };
    open.erase(std::remove_if(open.begin(), open.end(), ended), open.end());
    for (const ClipItem &y : open)
      if ((x.out || y.out) && share(t, y, x))
        return fail(SN_ERR_ALIAS, "an output overlaps another gradient or output");
    open.push_back(x);
  }
  return SN_OK;
}

}  // namespace

extern "C" {

size_t sn_token_logprobs_workspace_bytes(int64_t N, int64_t V, int32_t dt, int32_t n_top) {
  if (!dtype_ok(dt) || N < 1 || N >= kMaxDim || V < 1 || V >= kMaxDim || n_top < 0 || n_top > V ||
      n_top > SN_MAX_TOP)
    return 0;
  return sn::logprobs_workspace_bytes(dt, N, V, n_top);
}

int32_t sn_token_logprobs(const void *Z, int64_t N, int64_t V, int64_t ldz, int32_t dt,
                          double scale, const int32_t *tok, float *logp, float *entropy,
                          float *stats, int32_t n_top, float *top_logp, int32_t *top_id,
                          int32_t *err_flag, void *workspace, size_t workspace_bytes,
                          sn_stream stream) {
  int32_t st = check_logits(Z, N, V, ldz, dt, scale, tok);
  if (st) return st;
  if (n_top < 0 || n_top > V) return fail(SN_ERR_SHAPE, "need 0 <= n_top <= V");
  if (n_top > SN_MAX_TOP) return fail(SN_ERR_UNSUPPORTED, "n_top > SN_MAX_TOP");
  if (N == 0) return ok();
  if (!entropy || !stats || (tok && !logp) || (n_top && (!top_logp || !top_id)))
    return fail(SN_ERR_NULL, "an output is NULL");
  if (!aligned(logp, 4) || !aligned(entropy, 4) || !aligned(stats, 4) || !aligned(top_logp, 4) ||
      !aligned(top_id, 4))
    return fail(SN_ERR_ALIGN, "an output is not 4-byte aligned");
  Buffers b;
  b.read(span(Z, N, V, ldz, elem_size(dt)));
  if (tok) {
    b.read(span(tok, 1, N, N, 4));
    b.write(span(logp, 1, N, N, 4));
  }
  b.write(span(entropy, 1, N, N, 4));
  b.write(span(stats, N, 2, 2, 4));
  if (n_top) {
    b.write(span(top_logp, N, n_top, n_top, 4));
    b.write(span(top_id, N, n_top, n_top, 4));
  }
  const size_t need = sn::logprobs_workspace_bytes(dt, N, V, n_top);
  if (need) {
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    b.write(bytes_span(workspace, need));
  }
  if ((st = b.check("sn_token_logprobs"))) return st;
  const sn::LogprobsArgs a = {Z,       N,     V,     ldz,      static_cast<float>(scale),
                              tok,     tok ? logp : nullptr, entropy, stats,
                              n_top,   top_logp, top_id, err_flag};
  return hip_status(sn::launch_logprobs(dt, a, workspace, static_cast<hipStream_t>(stream)),
                    "sn_token_logprobs launch");
}

int32_t sn_token_logprobs_backward(const void *Z, int64_t N, int64_t V, int64_t ldz, int32_t dt,
                                   double scale, const int32_t *tok, const float *stats,
                                   const float *entropy, const float *g_logp,
                                   const float *g_entropy, void *dZ, int64_t lddz,
                                   int32_t *err_flag, sn_stream stream) {
  Buffers b;
  int32_t st = check_logits(Z, N, V, ldz, dt, scale, tok);
  if (st || (st = check_dlogits(Z, N, V, ldz, dt, dZ, lddz, b))) return st;
  if (N == 0) return ok();
  if (!stats || (g_logp && !tok) || (g_entropy && !entropy))
    return fail(SN_ERR_NULL, "stats, tok with g_logp and entropy with g_entropy are required");
  if (!aligned(stats, 4) || !aligned(entropy, 4) || !aligned(g_logp, 4) || !aligned(g_entropy, 4))
    return fail(SN_ERR_ALIGN, "a float input is not 4-byte aligned");
  b.read(span(stats, N, 2, 2, 4));
  b.read(span(tok, 1, N, N, 4));
  b.read(span(entropy, 1, N, N, 4));
  b.read(span(g_logp, 1, N, N, 4));
  b.read(span(g_entropy, 1, N, N, 4));
  if ((st = b.check("sn_token_logprobs_backward"))) return st;
  const sn::LogprobsGradArgs a = {Z,      N,         V,  ldz,  static_cast<float>(scale), tok, stats,
                                  entropy, g_logp, g_entropy, dZ, lddz, err_flag};
  return hip_status(sn::launch_logprobs_grad(dt, a, static_cast<hipStream_t>(stream)),
                    "sn_token_logprobs_backward launch");
}

int32_t sn_token_loss(const void *Z, int64_t N, int64_t V, int64_t ldz, int32_t dt, double scale,
                      const int32_t *tok, const float *weight, float *logp, void *dZ,
                      int64_t lddz, int32_t *err_flag, sn_stream stream) {
  Buffers b;
  int32_t st = check_logits(Z, N, V, ldz, dt, scale, tok);
  if (st || (st = check_dlogits(Z, N, V, ldz, dt, dZ, lddz, b))) return st;
  if (N == 0) return ok();
  if (!tok || !logp) return fail(SN_ERR_NULL, "tok or logp is NULL");
  if (!aligned(weight, 4) || !aligned(logp, 4))
    return fail(SN_ERR_ALIGN, "weight or logp is not 4-byte aligned");
  // logp is written while rows are still read: not over Z, in place or not
  b.read(span(tok, 1, N, N, 4));
  b.read(span(weight, 1, N, N, 4));
  b.write(span(logp, 1, N, N, 4));
  if ((st = b.check("sn_token_loss"))) return st;
  const sn::LossArgs a = {Z,      N,    V,  ldz,  static_cast<float>(scale), tok,
                          weight, logp, dZ, lddz, err_flag};
  return hip_status(sn::launch_loss(dt, a, static_cast<hipStream_t>(stream)),
                    "sn_token_loss launch");
}

int32_t sn_rmsnorm(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt, const void *R,
                   int64_t ldr, const void *w, double eps, void *H, int64_t ldh, void *Y,
                   int64_t ldy, sn_stream stream) {
  Buffers b;
  int32_t st = check_norm(X, N, d, ldx, dt, R, ldr, w, eps, H, ldh, b);
  if (st || (st = check_rows("Y", N, d, ldy))) return st;
  if (N == 0) return ok();
  if (!Y) return fail(SN_ERR_NULL, "Y is NULL");
  if (!elem_aligned(Y, dt)) return fail(SN_ERR_ALIGN, "Y not aligned to its element size");
  const Span y = span(Y, N, d, ldy, elem_size(dt));
  b.write(y);
  if ((st = b.check("sn_rmsnorm"))) return st;
  sn::NormArgs a = norm_args(X, N, d, ldx, R, ldr, w, eps, H, ldh);
  a.Y = Y;
  a.ldy = ldy;
  return hip_status(sn::launch_rmsnorm(dt, a, static_cast<hipStream_t>(stream)),
                    "sn_rmsnorm launch");
}

int32_t sn_rmsnorm_quant(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt,
                         const void *R, int64_t ldr, const void *w, double eps, void *H,
                         int64_t ldh, int32_t group, void *Q, int64_t ldq, float *S, int64_t lds,
                         sn_stream stream) {
  Buffers b;
  int32_t st = check_norm(X, N, d, ldx, dt, R, ldr, w, eps, H, ldh, b);
  if (st || (st = check_rows("Q", N, d, ldq))) return st;
  if (group < 0) return fail(SN_ERR_SHAPE, "group must be >= 0");
  if (group != 0 && group != 128) return fail(SN_ERR_UNSUPPORTED, "group must be 0 or 128");
  const int64_t scales = group ? sn::ceil_div(d, group) : 1;
  if ((st = check_rows("S", N, scales, lds))) return st;
  if (N == 0) return ok();
  if (!Q || !S) return fail(SN_ERR_NULL, "Q or S is NULL");
  if (!aligned(S, 4)) return fail(SN_ERR_ALIGN, "S is not 4-byte aligned");
  b.write(span(Q, N, d, ldq, 1));
  b.write(span(S, N, scales, lds, 4));
  if ((st = b.check("sn_rmsnorm_quant"))) return st;
  sn::NormArgs a = norm_args(X, N, d, ldx, R, ldr, w, eps, H, ldh);
  a.Y = Q;
  a.ldy = ldq;
  a.S = S;
  a.lds = lds;
  a.group = group;
  return hip_status(sn::launch_rmsnorm(dt, a, static_cast<hipStream_t>(stream)),
                    "sn_rmsnorm_quant launch");
}

size_t sn_rmsnorm_backward_workspace_bytes(int64_t N, int64_t d, int32_t dt) {
  if (!dtype_ok(dt) || N < 1 || N >= kMaxDim || d < 1 || d >= kMaxDim) return 0;
  return sn::rmsnorm_grad_workspace_bytes(dt, N, d);
}

int32_t sn_rmsnorm_backward(const void *H, int64_t N, int64_t d, int64_t ldh, int32_t dt,
                            const void *dY, int64_t lddy, const void *w, double eps,
                            const void *dH, int64_t lddh, void *dX, int64_t lddx, float *gw,
                            void *workspace, size_t workspace_bytes, sn_stream stream) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  int32_t st = check_rows("H", N, d, ldh);
  if (st || (st = check_rows("dY", N, d, lddy)) || (st = check_rows("dX", N, d, lddx)) ||
      (dH && (st = check_rows("dH", N, d, lddh))))
    return st;
  if (!(eps >= 0.0 && eps <= 3.0e38)) return fail(SN_ERR_SHAPE, "eps must be finite and >= 0");
  if (N == 0) return ok();
  if (!H || !dY || !dX) return fail(SN_ERR_NULL, "H, dY or dX is NULL");
  if (!elem_aligned(H, dt) || !elem_aligned(dY, dt) || !elem_aligned(w, dt) ||
      !elem_aligned(dH, dt) || !elem_aligned(dX, dt))
    return fail(SN_ERR_ALIGN, "a matrix or w not aligned to its element size");
  if (!aligned(gw, 4)) return fail(SN_ERR_ALIGN, "gw is not 4-byte aligned");
  const size_t es = elem_size(dt);
  Buffers b;
  b.write(span(dX, N, d, lddx, es));
  b.read(span(H, N, d, ldh, es));
  b.read(span(w, 1, d, d, es));
  if (dX != dY || lddx != lddy) b.read(span(dY, N, d, lddy, es));
  if (dH && (dX != dH || lddx != lddh)) b.read(span(dH, N, d, lddh, es));
  if (gw) {
    const size_t need = sn::rmsnorm_grad_workspace_bytes(dt, N, d);
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    b.write(span(gw, 1, d, d, 4));
    b.write(bytes_span(workspace, need));
  }
  if ((st = b.check("sn_rmsnorm_backward"))) return st;
  sn::NormGradArgs a = {};
  a.H = H;
  a.dY = dY;
  a.w = w;
  a.dH = dH;
  a.N = N;
  a.d = d;
  a.ldh = ldh;
  a.lddy = lddy;
  a.lddh = lddh;
  a.inv_d = static_cast<float>(1.0 / static_cast<double>(d));
  a.eps = static_cast<float>(eps);
  a.dX = dX;
  a.lddx = lddx;
  return hip_status(
      sn::launch_rmsnorm_grad(dt, a, gw, workspace, static_cast<hipStream_t>(stream)),
      "sn_rmsnorm_backward launch");
}

size_t sn_grad_sumsq_workspace_bytes(int32_t count, const sn_tensor *grads) {
  try {
    std::vector<sn::ClipTensor> t;
    if (clip_tensors(count, grads, nullptr, true, t)) return 0;
    const int64_t units = sn::clip_units(t.data(), static_cast<int32_t>(t.size()));
    return sn::align256(static_cast<size_t>(units > 0 ? units : 1) * sizeof(double));
  } catch (const std::exception &) {
    fail(SN_ERR_WORKSPACE, "out of host memory");
    return 0;
  }
}

int32_t sn_grad_sumsq(int32_t count, const sn_tensor *grads, double *sumsq, void *workspace,
                      size_t workspace_bytes, sn_stream stream) {
  try {
    std::vector<sn::ClipTensor> t;
    int32_t st = clip_tensors(count, grads, nullptr, false, t);
    if (st) return st;
    if (!sumsq) return fail(SN_ERR_NULL, "sumsq is NULL");
    if (!aligned(sumsq, 8)) return fail(SN_ERR_ALIGN, "sumsq is not 8-byte aligned");
    const int32_t n = static_cast<int32_t>(t.size());
    const int64_t units = sn::clip_units(t.data(), n);
    const size_t need = sn::align256(static_cast<size_t>(units > 0 ? units : 1) * sizeof(double));
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    const Span ws = bytes_span(workspace, need), to = bytes_span(sumsq, 8);
    if (overlap(ws, to)) return fail(SN_ERR_ALIAS, "sumsq overlaps the workspace");
    for (const sn::ClipTensor &c : t)
      if (overlap(clip_span(c, false), ws) || overlap(clip_span(c, false), to))
        return fail(SN_ERR_ALIAS, "a gradient overlaps the workspace or sumsq");
    return hip_status(
        sn::launch_sumsq(t.data(), n, sumsq, workspace, static_cast<hipStream_t>(stream)),
        "sn_grad_sumsq launch");
  } catch (const std::exception &) {
    return fail(SN_ERR_WORKSPACE, "out of host memory");
  }
}

int32_t sn_grad_clip(int32_t count, const sn_tensor *grads, const sn_tensor *out,
                     const double *sumsq, double max_norm, float *norm, sn_stream stream) {
  try {
    std::vector<sn::ClipTensor> t;
    int32_t st = clip_tensors(count, grads, out, false, t);
    if (st) return st;
    if (!sumsq) return fail(SN_ERR_NULL, "sumsq is NULL");
    if (!aligned(sumsq, 8) || !aligned(norm, 4))
      return fail(SN_ERR_ALIGN, "sumsq or norm is not aligned to its element size");
    if (!(max_norm >= 0.0)) return fail(SN_ERR_SHAPE, "max_norm must be >= 0");
    if ((st = check_clip_alias(t))) return st;
    const Span from = bytes_span(sumsq, 8), to = bytes_span(norm, norm ? 4 : 0);
    if (overlap(from, to)) return fail(SN_ERR_ALIAS, "norm overlaps sumsq");
    bool in_place = true;
    for (const sn::ClipTensor &c : t) {
      const Span g = clip_span(c, false), o = clip_span(c, true);
      if (overlap(o, from) || overlap(g, to) || overlap(o, to))
        return fail(SN_ERR_ALIAS, "a tensor overlaps sumsq or norm");
      in_place = in_place && c.out == c.g && c.ldo == c.ldg;
    }
    return hip_status(sn::launch_clip(t.data(), static_cast<int32_t>(t.size()), in_place, sumsq,
                                      max_norm, norm, static_cast<hipStream_t>(stream)),
                      "sn_grad_clip launch");
  } catch (const std::exception &) {
    return fail(SN_ERR_WORKSPACE, "out of host memory");
  }
}

}  // extern "C"

// ---- a block's end and start, gated feed-forward block, orthogonalised updates ----

namespace {

// What both calls of the block norm share; w_post: NULL without the post norm.
int32_t check_block(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt,
                    const void *w_post, const void *gate, int64_t ldgate, int32_t gate_fn,
                    double alpha, const void *w, double eps) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  int32_t st = check_rows("X", N, d, ldx);
  if (st || (gate && ldgate != 0 && (st = check_rows("gate", N, d, ldgate)))) return st;
  if (gate_fn != SN_GATE_NONE && gate_fn != SN_GATE_SIGMOID)
    return fail(SN_ERR_UNSUPPORTED, "unknown gate function %d", gate_fn);
  if (!(alpha >= -3.0e38 && alpha <= 3.0e38)) return fail(SN_ERR_SHAPE, "alpha must be finite");
  if (!(eps >= 0.0 && eps <= 3.0e38)) return fail(SN_ERR_SHAPE, "eps must be finite and >= 0");
  if (N == 0) return SN_OK;
  if (!X) return fail(SN_ERR_NULL, "X is NULL");
  if (!elem_aligned(X, dt) || !elem_aligned(gate, dt) || !elem_aligned(w, dt) ||
      !elem_aligned(w_post, dt))
    return fail(SN_ERR_ALIGN, "X, the gate or a gain vector is not aligned to its element size");
  return SN_OK;
}

Span gate_span(const void *gate, int64_t N, int64_t d, int64_t ldgate, size_t es) {
  return ldgate ? span(gate, N, d, ldgate, es) : span(gate, 1, d, d, es);
}

int32_t check_ff(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt, const void *Wg,
                 const void *Wu, int64_t ff, int64_t ldw, int32_t act) {
  if (!dtype_ok(dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", dt);
  int32_t st = check_rows("X", N, d, ldx);
  if (st || (st = check_rows("Wg", d, ff, ldw))) return st;
  if (N > (kMaxElems - 1) / (ff > d ? ff : d) || d > (kMaxElems - 1) / ff)
    return fail(SN_ERR_SHAPE, "a matrix of 2^40 or more elements");
  if (act != SN_ACT_SILU && act != SN_ACT_GELU && act != SN_ACT_RELU)
    return fail(SN_ERR_UNSUPPORTED, "unknown activation %d", act);
  return SN_OK;
}

// Two outputs of one row stride, which may be column blocks of one matrix (the gradients of
// [Wg | Wu] in one buffer): compared by their elements, and as one extent with the rest.
int32_t check_pair(const char *na, const char *nb, const void *p, const void *q, int64_t rows,
                   int64_t cols, int64_t ld, size_t es, Buffers &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
  const uintptr_t lo = x < y ? x : y, hi = x < y ? y : x, row = ld * es, len = cols * es;
  const Span s = span(reinterpret_cast<const void *>(lo), rows, cols, ld, es);
  if (hi < s.hi) {
    const uintptr_t r = rows > 1 ? (hi - lo) % row : hi - lo;
    if (r < len || (rows > 1 && r + len > row && (hi - lo) / row + 1 < static_cast<uintptr_t>(rows)))
      return fail(SN_ERR_ALIAS, "%s overlaps %s", na, nb);
    const Span t = span(reinterpret_cast<const void *>(hi), rows, cols, ld, es);
    b.write({s.lo, t.hi > s.hi ? t.hi : s.hi});
    return SN_OK;
  }
  b.write(s);
  b.write(span(reinterpret_cast<const void *>(hi), rows, cols, ld, es));
  return SN_OK;
}

// Matrices of one shape and dtype; those of M are float32.  Appends them to t, as outputs
// (and for `out`, in[i] as the input of out[i]).
int32_t orth_tensors(const char *name, int32_t count, const sn_tensor *a, const sn_tensor *like,
                     int32_t dt, std::vector<sn::ClipTensor> &t, const sn_tensor *out = nullptr) {
  if (!a || (out == nullptr && !like)) return fail(SN_ERR_NULL, "%s is NULL", name);
  for (int32_t i = 0; i < count; ++i) {
    const sn_tensor &m = a[i];
    for (const sn_tensor *q : {&m, out ? &out[i] : &m}) {
      if (q->dt != dt) return fail(SN_ERR_DTYPE, "%s[%d]: dtype %d, not %d", name, i, q->dt, dt);
      if (q->rows != like->rows || q->cols != like->cols)
        return fail(SN_ERR_SHAPE, "%s[%d]: the matrices of a call have one shape", name, i);
      if (q->rows == 0 || q->cols == 0) continue;
      if (q->ld < q->cols || q->ld >= kMaxElems)
        return fail(SN_ERR_SHAPE, "%s[%d]: the row stride must be >= the columns", name, i);
      if (!q->data) return fail(SN_ERR_NULL, "%s[%d] is NULL", name, i);
      if (!elem_aligned(q->data, dt))
        return fail(SN_ERR_ALIGN, "%s[%d] not aligned to its element size", name, i);
    }
    sn::ClipTensor c = {};
    c.g = m.data;
    c.out = out ? out[i].data : m.data;
    const int64_t ldo = out ? out[i].ld : m.ld;
    const bool gaps = m.rows > 1 && (m.ld != m.cols || ldo != m.cols);
    c.rows = gaps ? m.rows : 1;
    c.cols = gaps ? m.cols : m.rows * m.cols;
    c.ldg = gaps ? m.ld : c.cols;
    c.ldo = gaps ? ldo : c.cols;
    c.f32 = dt == SN_F32;
    t.push_back(c);
  }
  return SN_OK;
}

bool orth_shape(int32_t count, int64_t rows, int64_t cols) {
  return count >= 0 && rows >= 0 && rows < kMaxDim && cols >= 0 && cols < kMaxDim &&
         (rows == 0 || cols <= (kMaxElems - 1) / rows);
}

// The checks that both calls on matrices share, and the call, 32 matrices at a time.
int32_t run_orth(const char *call, int32_t count, const sn_tensor *G, const sn_tensor *M,
                 const sn_tensor *W, sn::OrthArgs a, void *workspace, size_t workspace_bytes,
                 sn_stream stream) {
  if (count < 0) return fail(SN_ERR_SHAPE, "count must be >= 0");
  if (a.steps < 1 || a.steps > SN_MAX_ORTH_STEPS)
    return fail(SN_ERR_SHAPE, "steps must lie in [1, %d]", SN_MAX_ORTH_STEPS);
  if (count == 0) return ok();
  if (!G || !W || (a.update && !M)) return fail(SN_ERR_NULL, "an array of matrices is NULL");
  const sn_tensor &like = W[0];
  if (!dtype_ok(like.dt)) return fail(SN_ERR_DTYPE, "unknown dtype %d", like.dt);
  if (!orth_shape(count, like.rows, like.cols))
    return fail(SN_ERR_SHAPE, "%lld x %lld out of range", (long long)like.rows,
                (long long)like.cols);
  std::vector<sn::ClipTensor> t;
  int32_t st;
  if (a.update) {
    if ((st = orth_tensors("W", count, W, &like, like.dt, t)) ||
        (st = orth_tensors("G", count, G, &like, like.dt, t)) ||
        (st = orth_tensors("M", count, M, &like, SN_F32, t)))
      return st;
  } else if ((st = orth_tensors("in", count, G, &like, like.dt, t, W))) {
    return st;
  }
  if (like.rows == 0 || like.cols == 0) return ok();
  const size_t need = sn::orth_workspace_bytes(like.rows, like.cols, count);
  if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
  if ((st = check_clip_alias(t))) return st;
  for (const sn::ClipTensor &c : t)
    if (overlap(clip_span(c, false), bytes_span(workspace, need)) ||
        overlap(clip_span(c, true), bytes_span(workspace, need)))
      return fail(SN_ERR_ALIAS, "%s: a matrix overlaps the workspace", call);
  a.rows = like.rows;
  a.cols = like.cols;
  for (int32_t i = 0; i < count; i += sn::OrthMats::kMost) {
    sn::OrthMats m = {};
    a.count = count - i < sn::OrthMats::kMost ? count - i : sn::OrthMats::kMost;
    for (int32_t j = 0; j < a.count; ++j) {
      m.g[j] = G[i + j].data;
      m.ldg[j] = G[i + j].ld;
      m.w[j] = W[i + j].data;
      m.ldw[j] = W[i + j].ld;
      if (!a.update) continue;
      m.m[j] = static_cast<float *>(M[i + j].data);
      m.ldm[j] = M[i + j].ld;
    }
    if ((st = hip_status(sn::launch_orth(like.dt, m, a, workspace, static_cast<hipStream_t>(stream)),
                         call)))
      return st;
  }
  return ok();
}

}  // namespace

extern "C" {

int32_t sn_block_norm(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt, const void *R,
                      int64_t ldr, int32_t post, const void *w_post, const void *gate,
                      int64_t ldgate, int32_t gate_fn, double alpha, const void *w, double eps,
                      void *H, int64_t ldh, void *Y, int64_t ldy, sn_stream stream) {
  if (!post) w_post = nullptr;
  int32_t st = check_block(X, N, d, ldx, dt, w_post, gate, ldgate, gate_fn, alpha, w, eps);
  if (st || (st = check_rows("R", N, d, ldr)) || (st = check_rows("H", N, d, ldh)) ||
      (Y && (st = check_rows("Y", N, d, ldy))))
    return st;
  if (N == 0) return ok();
  if (!R || !H) return fail(SN_ERR_NULL, "R or H is NULL");
  if (!elem_aligned(R, dt) || !elem_aligned(H, dt) || !elem_aligned(Y, dt))
    return fail(SN_ERR_ALIGN, "R, H or Y not aligned to its element size");
  const size_t es = elem_size(dt);
  Buffers b;
  b.write(span(H, N, d, ldh, es));
  if (H != X || ldh != ldx) b.read(span(X, N, d, ldx, es));
  if (H != R || ldh != ldr) b.read(span(R, N, d, ldr, es));
  b.read(gate_span(gate, N, d, ldgate, es));
  b.read(span(w, 1, d, d, es));
  b.read(span(w_post, 1, d, d, es));
  b.write(span(Y, N, d, ldy, es));
  if ((st = b.check("sn_block_norm"))) return st;
  sn::BlockNormArgs a = {};
  a.X = X;
  a.R = R;
  a.w = w;
  a.w_post = w_post;
  a.gate = gate;
  a.N = N;
  a.d = d;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldgate = ldgate;
  a.inv_d = static_cast<float>(1.0 / static_cast<double>(d));
  a.eps = static_cast<float>(eps);
  a.alpha = static_cast<float>(alpha);
  a.post = post != 0;
  a.sigmoid = gate_fn == SN_GATE_SIGMOID;
  a.H = H;
  a.Y = Y;
  a.ldh = ldh;
  a.ldy = ldy;
  return hip_status(sn::launch_block_norm(dt, a, static_cast<hipStream_t>(stream)),
                    "sn_block_norm launch");
}

size_t sn_block_norm_backward_workspace_bytes(int64_t N, int64_t d, int32_t dt) {
  if (!dtype_ok(dt) || N < 1 || N >= kMaxDim || d < 1 || d >= kMaxDim) return 0;
  return sn::block_norm_grad_workspace_bytes(dt, N, d);
}

int32_t sn_block_norm_backward(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt,
                               const void *H, int64_t ldh, int32_t post, const void *w_post,
                               const void *gate, int64_t ldgate, int32_t gate_fn, double alpha,
                               const void *w, double eps, const void *dY, int64_t lddy,
                               const void *dH, int64_t lddh, void *dX, int64_t lddx, void *dR,
                               int64_t lddr, void *dgate, int64_t lddgate, float *dgate_row,
                               float *gw, float *gw_post, void *workspace, size_t workspace_bytes,
                               sn_stream stream) {
  if (!post) w_post = nullptr;
  int32_t st = check_block(X, N, d, ldx, dt, w_post, gate, ldgate, gate_fn, alpha, w, eps);
  if (st || (st = check_rows("H", N, d, ldh)) || (dY && (st = check_rows("dY", N, d, lddy))) ||
      (dH && (st = check_rows("dH", N, d, lddh))) || (st = check_rows("dX", N, d, lddx)) ||
      (st = check_rows("dR", N, d, lddr)) ||
      (dgate && (st = check_rows("dgate", N, d, lddgate))))
    return st;
  if (N == 0) return ok();
  if (!dX || !dR || (dY && !H)) return fail(SN_ERR_NULL, "dX, dR or H is NULL");
  if ((gw && !dY) || (gw_post && !post))
    return fail(SN_ERR_NULL, "gw needs dY, gw_post the post norm");
  if ((dgate && (!gate || ldgate == 0)) || (dgate_row && (!gate || ldgate != 0)))
    return fail(SN_ERR_SHAPE, "dgate belongs to a gate for each token, dgate_row to one gate row");
  if (!elem_aligned(H, dt) || !elem_aligned(dY, dt) || !elem_aligned(dH, dt) ||
      !elem_aligned(dX, dt) || !elem_aligned(dR, dt) || !elem_aligned(dgate, dt))
    return fail(SN_ERR_ALIGN, "a matrix is not aligned to its element size");
  if (!aligned(gw, 4) || !aligned(gw_post, 4) || !aligned(dgate_row, 4))
    return fail(SN_ERR_ALIGN, "a float32 sum is not 4-byte aligned");
  const size_t es = elem_size(dt);
  const auto same = [](const void *p, int64_t lp, const void *q, int64_t lq) {
    return p == q && lp == lq;
  };
  Buffers b;
  b.write(span(dX, N, d, lddx, es));
  b.write(span(dR, N, d, lddr, es));
  b.write(span(dgate, N, d, lddgate, es));
  if (!same(dX, lddx, X, ldx)) b.read(span(X, N, d, ldx, es));
  if (dY) b.read(span(H, N, d, ldh, es));
  const bool on_y = same(dX, lddx, dY, lddy) || same(dR, lddr, dY, lddy);
  const bool on_h = same(dX, lddx, dH, lddh) || same(dR, lddr, dH, lddh);
  if (dY && !on_y) b.read(span(dY, N, d, lddy, es));
  if (dH && !on_h) b.read(span(dH, N, d, lddh, es));
  if (!dgate || !same(dgate, lddgate, gate, ldgate)) b.read(gate_span(gate, N, d, ldgate, es));
  b.read(span(w, 1, d, d, es));
  b.read(span(w_post, 1, d, d, es));
  b.write(span(gw, 1, d, d, 4));
  b.write(span(gw_post, 1, d, d, 4));
  b.write(span(dgate_row, 1, d, d, 4));
  if (gw || gw_post || dgate_row) {
    const size_t need = sn::block_norm_grad_workspace_bytes(dt, N, d);
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    b.write(bytes_span(workspace, need));
  }
  if ((st = b.check("sn_block_norm_backward"))) return st;
  sn::BlockNormGradArgs a = {};
  a.X = X;
  a.H = H;
  a.w = w;
  a.w_post = w_post;
  a.gate = gate;
  a.dY = dY;
  a.dH = dH;
  a.N = N;
  a.d = d;
  a.ldx = ldx;
  a.ldh = ldh;
  a.ldgate = ldgate;
  a.lddy = lddy;
  a.lddh = lddh;
  a.inv_d = static_cast<float>(1.0 / static_cast<double>(d));
  a.eps = static_cast<float>(eps);
  a.alpha = static_cast<float>(alpha);
  a.post = post != 0;
  a.sigmoid = gate_fn == SN_GATE_SIGMOID;
  a.dX = dX;
  a.dR = dR;
  a.dgate = dgate;
  a.lddx = lddx;
  a.lddr = lddr;
  a.lddg = lddgate;
  a.sums[0] = gw;
  a.sums[1] = gw_post;
  a.sums[2] = dgate_row;
  return hip_status(
      sn::launch_block_norm_grad(dt, a, workspace, static_cast<hipStream_t>(stream)),
      "sn_block_norm_backward launch");
}

size_t sn_gated_ff_workspace_bytes(int64_t N, int64_t d, int64_t ff, int64_t ldx, int64_t ldw,
                                   int32_t dt, int32_t aligned) {
  if (check_ff(nullptr, N, d, ldx, dt, nullptr, nullptr, ff, ldw, SN_ACT_SILU) || N == 0) return 0;
  sn::FfArgs a = {};
  a.N = N;
  a.d = d;
  a.ff = ff;
  a.ldx = ldx;
  a.ldw = ldw;
  return sn::ff_workspace_bytes(dt, a, aligned != 0);
}

size_t sn_gated_ff_backward_workspace_bytes(int64_t N, int64_t d, int64_t ff, int64_t ldx,
                                            int64_t ldw, int64_t ldd, int32_t dt,
                                            int32_t aligned) {
  if (check_ff(nullptr, N, d, ldx, dt, nullptr, nullptr, ff, ldw, SN_ACT_SILU) || N == 0 ||
      ldd < ff || ldd >= kMaxDim)
    return 0;
  sn::FfGradArgs a = {};
  a.N = N;
  a.d = d;
  a.ff = ff;
  a.ldx = ldx;
  a.ldw = ldw;
  a.ldd = ldd;
  return sn::ff_grad_workspace_bytes(dt, a, aligned != 0);
}

int32_t sn_gated_ff(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt, const void *Wg,
                    const void *Wu, int64_t ff, int64_t ldw, int32_t act, void *H, int64_t ldh,
                    void *G, void *U, int64_t ldg, void *workspace, size_t workspace_bytes,
                    sn_stream stream) {
  int32_t st = check_ff(X, N, d, ldx, dt, Wg, Wu, ff, ldw, act);
  if (st || (st = check_rows("H", N, ff, ldh)) ||
      ((G || U) && (st = check_rows("G and U", N, ff, ldg))))
    return st;
  if (N == 0) return ok();
  if (!X || !Wg || !Wu || !H || !G != !U)
    return fail(SN_ERR_NULL, "X, Wg, Wu, H or one of G and U is NULL");
  for (const void *p : {X, Wg, Wu, static_cast<const void *>(H), static_cast<const void *>(G),
                        static_cast<const void *>(U)})
    if (!elem_aligned(p, dt)) return fail(SN_ERR_ALIGN, "a matrix is not aligned to its element size");
  const size_t es = elem_size(dt);
  sn::FfArgs a = {};
  a.X = X;
  a.Wg = Wg;
  a.Wu = Wu;
  a.N = N;
  a.d = d;
  a.ff = ff;
  a.ldx = ldx;
  a.ldw = ldw;
  a.act = act;
  a.H = H;
  a.G = G;
  a.U = U;
  a.ldh = ldh;
  a.ldg = ldg;
  const size_t need = sn::ff_call_bytes(dt, a);
  Buffers b;
  if (need) {
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    b.write(bytes_span(workspace, need));
  }
  b.read(span(X, N, d, ldx, es));
  b.read(span(Wg, d, ff, ldw, es));
  b.read(span(Wu, d, ff, ldw, es));
  b.write(span(H, N, ff, ldh, es));
  if (G && (st = check_pair("G", "U", G, U, N, ff, ldg, es, b))) return st;
  if ((st = b.check("sn_gated_ff"))) return st;
  return hip_status(sn::launch_ff(dt, a, workspace, static_cast<hipStream_t>(stream)),
                    "sn_gated_ff launch");
}

int32_t sn_gated_ff_backward(const void *X, int64_t N, int64_t d, int64_t ldx, int32_t dt,
                             const void *Wg, const void *Wu, int64_t ff, int64_t ldw, int32_t act,
                             const void *G, const void *U, int64_t ldg, const void *dH,
                             int64_t lddh, void *dG, void *dU, int64_t ldd, void *dX, int64_t lddx,
                             void *gWg, void *gWu, int64_t ldgw, int32_t gdt, int32_t accumulate,
                             void *workspace, size_t workspace_bytes, sn_stream stream) {
  int32_t st = check_ff(X, N, d, ldx, dt, Wg, Wu, ff, ldw, act);
  if (st || (st = check_rows("G and U", N, ff, ldg)) || (st = check_rows("dH", N, ff, lddh)) ||
      (st = check_rows("dG and dU", N, ff, ldd)) || (dX && (st = check_rows("dX", N, d, lddx))) ||
      ((gWg || gWu) && (st = check_rows("gWg and gWu", d, ff, ldgw))))
    return st;
  if (!gWg != !gWu) return fail(SN_ERR_NULL, "gWg and gWu: both or neither");
  if (gWg && gdt != dt && gdt != SN_F32) return fail(SN_ERR_DTYPE, "gdt must be dt or SN_F32");
  if (N > 0 && (!X || !Wg || !Wu || !G || !U || !dH || !dG || !dU))
    return fail(SN_ERR_NULL, "an input, dG or dU is NULL");
  for (const void *p : {X, Wg, Wu, G, U, dH, static_cast<const void *>(dG),
                        static_cast<const void *>(dU), static_cast<const void *>(dX)})
    if (!elem_aligned(p, dt)) return fail(SN_ERR_ALIGN, "a matrix is not aligned to its element size");
  if (gWg && (!elem_aligned(gWg, gdt) || !elem_aligned(gWu, gdt)))
    return fail(SN_ERR_ALIGN, "gWg or gWu is not aligned to its element size");
  if (N == 0 && (!gWg || accumulate)) return ok();
  const size_t es = elem_size(dt);
  sn::FfGradArgs a = {};
  a.X = X;
  a.Wg = Wg;
  a.Wu = Wu;
  a.G = G;
  a.U = U;
  a.dH = dH;
  a.N = N;
  a.d = d;
  a.ff = ff;
  a.ldx = ldx;
  a.ldw = ldw;
  a.ldg = ldg;
  a.lddh = lddh;
  a.act = act;
  a.dG = dG;
  a.dU = dU;
  a.ldd = ldd;
  a.dX = dX;
  a.lddx = lddx;
  a.gWg = gWg;
  a.gWu = gWu;
  a.ldgw = ldgw;
  a.gdt = gdt;
  a.add = accumulate != 0;
  const size_t need = N ? sn::ff_grad_call_bytes(dt, a) : 0;
  Buffers b;
  if (need) {
    if ((st = check_workspace(workspace, workspace_bytes, need))) return st;
    b.write(bytes_span(workspace, need));
  }
  if (dX != X || lddx != ldx || gWg) b.read(span(X, N, d, ldx, es));
  b.read(span(Wg, d, ff, ldw, es));
  b.read(span(Wu, d, ff, ldw, es));
  for (const void *p : {G, U})
    if (ldg != ldd || (p != dG && p != dU)) b.read(span(p, N, ff, ldg, es));
  if (lddh != ldd || (dH != dG && dH != dU)) b.read(span(dH, N, ff, lddh, es));
  if (dX) b.write(span(dX, N, d, lddx, es));
  if (N && (st = check_pair("dG", "dU", dG, dU, N, ff, ldd, es, b))) return st;
  if (gWg && (st = check_pair("gWg", "gWu", gWg, gWu, d, ff, ldgw, elem_size(gdt), b))) return st;
  if ((st = b.check("sn_gated_ff_backward"))) return st;
  return hip_status(sn::launch_ff_grad(dt, a, workspace, static_cast<hipStream_t>(stream)),
                    "sn_gated_ff_backward launch");
}

size_t sn_orthogonalize_workspace_bytes(int32_t count, int64_t rows, int64_t cols) {
  if (!orth_shape(count, rows, cols) || count == 0 || rows == 0 || cols == 0) return 0;
  return sn::orth_workspace_bytes(rows, cols, count);
}

int32_t sn_orthogonalize(int32_t count, const sn_tensor *in, const sn_tensor *out, int32_t steps,
                         void *workspace, size_t workspace_bytes, sn_stream stream) {
  try {
    sn::OrthArgs a = {};
    a.steps = steps;
    return run_orth("sn_orthogonalize", count, in, nullptr, out, a, workspace, workspace_bytes,
                    stream);
  } catch (const std::exception &) {
    return fail(SN_ERR_WORKSPACE, "out of host memory");
  }
}

int32_t sn_muon_step(int32_t count, const sn_tensor *W, const sn_tensor *G, const sn_tensor *M,
                     double lr, double momentum, int32_t nesterov, double weight_decay,
                     double scale, int32_t steps, void *workspace, size_t workspace_bytes,
                     sn_stream stream) {
  try {
    const double most = 3.0e38;
    if (!(lr >= 0.0 && lr <= most) || !(weight_decay >= 0.0 && weight_decay <= most) ||
        !(momentum >= 0.0 && momentum < 1.0) || !(scale >= -most && scale <= most) ||
        !(lr * scale >= -most && lr * scale <= most))
      return fail(SN_ERR_SHAPE, "need finite lr, weight_decay >= 0, 0 <= momentum < 1, finite scale");
    sn::OrthArgs a = {};
    a.steps = steps;
    a.update = true;
    a.nesterov = nesterov != 0;
    a.momentum = static_cast<float>(momentum);
    a.rate = static_cast<float>(lr * scale);
    a.decay = static_cast<float>(weight_decay);
    return run_orth("sn_muon_step", count, G, M, W, a, workspace, workspace_bytes, stream);
  } catch (const std::exception &) {
    return fail(SN_ERR_WORKSPACE, "out of host memory");
  }
}

const char *sn_status_string(int32_t status) {
  switch (status) {
    case SN_OK: return "SN_OK";
    case SN_ERR_NULL: return "SN_ERR_NULL";
    case SN_ERR_SHAPE: return "SN_ERR_SHAPE";
    case SN_ERR_DTYPE: return "SN_ERR_DTYPE";
    case SN_ERR_ALIGN: return "SN_ERR_ALIGN";
    case SN_ERR_ALIAS: return "SN_ERR_ALIAS";
    case SN_ERR_INDEX: return "SN_ERR_INDEX";
    case SN_ERR_HIP: return "SN_ERR_HIP";
    case SN_ERR_UNSUPPORTED: return "SN_ERR_UNSUPPORTED";
    case SN_ERR_WORKSPACE: return "SN_ERR_WORKSPACE";
    default: return "SN_ERR_UNKNOWN";
  }
}

const char *sn_last_error(void) { return g_err; }

const char *sn_version(void) { return "0.1.0 gfx950"; }

}  // extern "C"
