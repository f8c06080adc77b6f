// Orthogonalised updates: the singular values of X = B / |B|_F taken towards 1 by the
// odd polynomial of Newton-Schulz steps (K. Jordan et al., the Muon optimiser, 2024),
//   X <- (a I + b A + c A^2) X,  A = X X^T,   a, b, c = 3.4445, -4.7750, 2.0315,
// X Q with A = X^T X where there are more rows than columns.  X keeps its row and
// column space, so the columns of a weight that lie in the codec's subspace stay there.
// As an optimizer step:  M <- mu M + G,  B = G + mu M (or M),  W <- W - rate X - decay W.
//
// Small singular values grow by 3.44 a step, and so do errors in their directions: bf16
// operands would leave an error of some percent.  So X, A and Q = a I + b A + c A^2 are held
// as two fp16 planes, hi + lo (22 bits), and hi lo + lo hi + hi hi are added up in
// float32: a third of the matrix cores' 16-bit rate for results like float32's.  fp16's
// range is no limit: |X| <= 1.21 by the polynomial's maximum on [0, 1.21] and |A|, |Q| by
// 1.45 and 3.45, each is stored times a power of two that keeps it below 65504, and lo
// times 2^11, as large as hi at most, so that what fp16's least normal number, 2^-14, cuts
// off lies below 2^-28 in hi and 2^-39 in all.
// Where the result is rounded to bf16, products are left out whose part of it is small beside
// that rounding (1.7e-3 of the result's norm): A is made of hi hi, A^2 too but in the last
// two steps, and Q X of Q's hi with both planes of X but in the last step: 16 products of
// m x m x n, a symmetric one for half, where 30 make five whole steps.  The error is
// 0.7e-3 to 1.6e-3 of the result's norm (Gaussian matrices, few strong directions, singular
// values over four decades, rank 20 of 384).  What must not go is X's lo: with hi alone
// it is 7e-3 over four decades and 4e-2 in rank 20, where the rounded-off part of X grows
// into directions that X does not have.
// A and Q are symmetric: the tiles on and below the diagonal are computed and mirrored.
// Matrices of one shape share every launch.
#include "sn_internal.h"
#include "sn_mm.h"
#include "sn_rows.h"

namespace sn {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// X and A are stored times 2^15, Q times 2^14.
constexpr float kXScale = 32768.0f, kQScale = 16384.0f, kUp = 2048.0f;

constexpr int kBlockElems = 4096;  // elements of a workgroup's turn in the passes over B
int sum_groups(int64_t rows, int64_t cols) {
  const int64_t n = ceil_div(rows * cols, kBlockElems);
  return static_cast<int>(n < 256 ? n : 256);
}

// Four columns of B: the gradient, or the momentum made from it, which is stored
// where `first`.
template <typename T>
__device__ __forceinline__ f32x4 orth_b(const OrthMats &t, const OrthArgs &a, int z, int64_t r,
                                        int64_t c, bool first) {
  const T *g = static_cast<const T *>(t.g[z]) + r * t.ldg[z] + c;
  float *m = a.update ? t.m[z] + r * t.ldm[z] + c : nullptr;
  f32x4 b = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (c + e >= a.cols) continue;
    const float gv = a.update && !first && !a.nesterov ? 0.0f : to_f32(g[e]);
    if (!a.update) {
      b[e] = gv;
      continue;
    }
    float mv = m[e];
    if (first) {
      mv = fmaf(a.momentum, mv, gv);
      m[e] = mv;
    }
    b[e] = a.nesterov ? fmaf(a.momentum, mv, gv) : mv;
  }
  return b;
}

// The momentum, and the sum of squares of B in float64: one part a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void orth_begin_kernel(OrthMats t, OrthArgs a, int groups,
                                                         double *part) {
  __shared__ double red[4];
  const int z = blockIdx.x / groups, g = blockIdx.x - z * groups;
  const int64_t per = (a.cols + 3) / 4, all = a.rows * per;
  double s = 0.0;
  for (int64_t id = g * 256 + threadIdx.x; id < all; id += static_cast<int64_t>(groups) * 256) {
    const int64_t r = id / per;
    const f32x4 b = orth_b<T>(t, a, z, r, (id - r * per) * 4, true);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fma(static_cast<double>(b[e]), static_cast<double>(b[e]), s);
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = ((red[0] + red[1]) + red[2]) + red[3];
}

__device__ __forceinline__ float f16_value(uint16_t v) {
  return static_cast<float>(__builtin_bit_cast(_Float16, v));
}
__device__ __forceinline__ uint16_t f16_bits(float v) {
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
}
// fp16 planes of four values (low: both of them)
__device__ __forceinline__ void orth_put(uint16_t *to, int64_t plane, f32x4 v, bool low = true) {
  uint16_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = f16_bits(v[e]);
    l[e] = f16_bits((v[e] - f16_value(h[e])) * kUp);
  }
  *reinterpret_cast<u32x2 *>(to) =
      u32x2{h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16};
  if (!low) return;
  *reinterpret_cast<u32x2 *>(to + plane) =
      u32x2{l[0] | static_cast<uint32_t>(l[1]) << 16, l[2] | static_cast<uint32_t>(l[3]) << 16};
}

// X = B / |B|, in planes of rows x ldp (zeros past cols).  A matrix of zeros stays one.
template <typename T>
__global__ __launch_bounds__(256) void orth_split_kernel(OrthMats t, OrthArgs a, int groups,
                                                         int sums, const double *part, uint16_t *X,
                                                         int64_t ldp) {
  __shared__ double red[4];
  const int z = blockIdx.x / groups, g = blockIdx.x - z * groups;
  double s = static_cast<int>(threadIdx.x) < sums ? part[z * sums + threadIdx.x] : 0.0;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = ((red[0] + red[1]) + red[2]) + red[3];
  const double inv = s > 0.0 || s != s ? static_cast<double>(kXScale) / sqrt(s) : 0.0;
  const int64_t per = ldp / 4, all = a.rows * per, plane = a.rows * ldp;
  uint16_t *to = X + z * 2 * plane;
  for (int64_t id = g * 256 + threadIdx.x; id < all; id += static_cast<int64_t>(groups) * 256) {
    const int64_t r = id / per, c = (id - r * per) * 4;
    const f32x4 b = orth_b<T>(t, a, z, r, c, false);
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(static_cast<double>(b[e]) * inv);
    orth_put(to + r * ldp + c, plane, v);
  }
}

// The symmetric products, m x m with stride ldp: A from X, or (POLY) Q from A.
template <class S, bool POLY>
__global__ __launch_bounds__(S::NT, S::NT / 256) void orth_sym_kernel(MmArgs m, int64_t n, int64_t ldp,
                                                                     int64_t side, int64_t from,
                                                                     const uint16_t *A, uint16_t *to,
                                                                     bool low) {
  static_assert(S::BM == S::BN, "a tile on the diagonal is square");
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int64_t tiles = side * (side + 1) / 2;
  const int64_t id = mm_order(blockIdx.x, gridDim.x);
  const int64_t z = id / tiles, k = id - z * tiles;
  int64_t ti = static_cast<int64_t>((sqrtf(8.0f * static_cast<float>(k) + 1.0f) - 1.0f) * 0.5f);
  while (ti * (ti + 1) / 2 > k) --ti;
  while ((ti + 1) * (ti + 2) / 2 <= k) ++ti;
  const int64_t tj = k - ti * (ti + 1) / 2;
  f32x4 acc[S::TM][S::TN];
  mm_tile<S>(m, ti * S::BM, tj * S::BN, 0, mm_steps(m), lds, acc, z * from, z * from);
  const int64_t plane = n * ldp;
  uint16_t *out = to + z * 2 * plane;
  const uint16_t *in = POLY ? A + z * 2 * plane : nullptr;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = ti * S::BM + wave / S::WN * (S::BM / S::WM) + (lane & 15);
  const int64_t col0 = tj * S::BN + wave % S::WN * (S::BN / S::WN) + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int64_t row = row0 + i * 16;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int64_t col = col0 + j * 16;
      if (row >= ldp || col >= ldp) continue;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool inside = row < n && col + e < n;
        if constexpr (POLY) {
          float x = 0.0f;
          if (inside)
            x = fmaf(f16_value(in[plane + row * ldp + col + e]), 1.0f / kUp,
                     f16_value(in[row * ldp + col + e]));
          const float one = row == col + e ? kA * kQScale : 0.0f;
          v[e] = fmaf(kC * kQScale / (kXScale * kXScale), acc[i][j][e],
                      fmaf(kB * kQScale / kXScale, x, one));
        } else {
          v[e] = acc[i][j][e] * (1.0f / kXScale);
        }
        if (!inside) v[e] = 0.0f;
      }
      if (row < n) orth_put(out + row * ldp + col, plane, v, low);
      if (ti == tj) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (col + e >= n) continue;
        uint16_t *p = out + (col + e) * ldp + row;
        p[0] = f16_bits(v[e]);
        if (low) p[plane] = f16_bits((v[e] - f16_value(f16_bits(v[e]))) * kUp);
      }
    }
  }
}

// X' = Q X or X Q, in planes, or in its place in the table.
template <class S, bool LAST, typename T>
__global__ __launch_bounds__(S::NT, S::NT / 256) void orth_apply_kernel(MmArgs m, OrthMats t, OrthArgs a,
                                                                       int64_t gm, int64_t gn,
                                                                       int64_t a_bytes, int64_t b_bytes,
                                                                       uint16_t *to, int64_t ldp) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int64_t tiles = gm * gn, id = mm_order(blockIdx.x, gridDim.x);
  const int64_t z = id / tiles;
  int64_t tm, tn;
  mm_place(id - z * tiles, gm, gn, tm, tn);
  f32x4 acc[S::TM][S::TN];
  mm_tile<S>(m, tm * S::BM, tn * S::BN, 0, mm_steps(m), lds, acc, z * a_bytes, z * b_bytes);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = tm * S::BM + wave / S::WN * (S::BM / S::WM) + (lane & 15);
  const int64_t col0 = tn * S::BN + wave % S::WN * (S::BN / S::WN) + 4 * (lane >> 4);
  const int64_t plane = a.rows * ldp;
  T *W = LAST ? static_cast<T *>(t.w[z]) : nullptr;
  const int64_t ldw = LAST ? t.ldw[z] : 0;
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int64_t row = row0 + i * 16;
    if (row >= a.rows) continue;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int64_t col = col0 + j * 16;
      if (col >= ldp) continue;
      f32x4 v = acc[i][j];
      if constexpr (LAST) {
        T *w = W + row * ldw + col;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (col + e >= a.cols) continue;
          float x = v[e] * (1.0f / (kXScale * kQScale));
          if (a.update) {
            const float old = to_f32(w[e]);
            x = fmaf(-a.rate, x, fmaf(-a.decay, old, old));
          }
          w[e] = from_f32<T>(x);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = col + e < a.cols ? v[e] * (1.0f / kQScale) : 0.0f;
        orth_put(to + z * 2 * plane + row * ldp + col, plane, v);
      }
    }
  }
}

struct OrthPlan {
  int64_t n, ldx, lda;  // the smaller side; the planes' strides
  int sums;
  size_t x[2], a, q, part, total;
};
OrthPlan orth_plan(int64_t rows, int64_t cols, int64_t count) {
  OrthPlan p = {};
  p.n = rows < cols ? rows : cols;
  p.ldx = (cols + 7) / 8 * 8;
  p.lda = (p.n + 7) / 8 * 8;
  p.sums = sum_groups(rows, cols);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  const size_t x = size_t(4) * count * rows * p.ldx, a = size_t(4) * count * p.n * p.lda;
  p.x[0] = take(x);
  p.x[1] = take(x);
  p.a = take(a);
  p.q = take(a);
  p.part = take(sizeof(double) * count * p.sums);
  p.total = at;
  return p;
}

// The products that are added up: hi lo, lo hi and hi hi; hi hi alone; with both planes of
// one operand.
enum Products { kAll, kHigh, kBothOfA, kBothOfB };
void planes(MmArgs &m, const uint16_t *a, int64_t aplane, const uint16_t *b, int64_t bplane,
            Products which) {
  m.segs = 0;
  m.factor = 1.0f / kUp;
  const auto add = [&](int pa, int pb) {
    m.a.p[m.segs] = a + pa * aplane;
    m.b.p[m.segs++] = b + pb * bplane;
  };
  if (which == kAll || which == kBothOfB) add(0, 1);
  if (which == kAll || which == kBothOfA) add(1, 0);
  m.run[0] = m.segs ? m.segs : 1;
  add(0, 0);
  m.run[1] = m.segs;
}

// Largest tile that gives most CUs one.
int orth_tile(int64_t gm, int64_t gn, int64_t count, bool sym) {
  for (int size : {256, 128}) {
    const int64_t r = ceil_div(gm, size), c = ceil_div(gn, size);
    if ((sym ? r * (r + 1) / 2 : r * c) * count >= (size == 256 && sym ? 1024 : 224)) return size;
  }
  return 64;
}

template <bool K, bool POLY>
void run_sym(const MmArgs &m, int64_t n, int64_t ldp, int64_t count, int64_t from, const uint16_t *A,
             uint16_t *to, bool low, hipStream_t s) {
  const int size = orth_tile(n, n, count, true);
  const int64_t side = ceil_div(n, size);
  const unsigned grid = static_cast<unsigned>(side * (side + 1) / 2 * count);
  if (size == 256)
    orth_sym_kernel<MmShape<true, K, K, 256, 256, 2, 4>, POLY><<<grid, 512, 0, s>>>(m, n, ldp, side, from, A, to, low);
  else if (size == 128)
    orth_sym_kernel<MmShape<true, K, K, 128, 128, 2, 2>, POLY><<<grid, 256, 0, s>>>(m, n, ldp, side, from, A, to, low);
  else
    orth_sym_kernel<MmShape<true, K, K, 64, 64, 2, 2>, POLY><<<grid, 256, 0, s>>>(m, n, ldp, side, from, A, to, low);
}

template <bool BK, bool LAST, typename T>
void run_apply(const MmArgs &m, const OrthMats &t, const OrthArgs &a, int64_t a_bytes,
               int64_t b_bytes, uint16_t *to, int64_t ldp, hipStream_t s) {
  const int size = orth_tile(a.rows, a.cols, a.count, false);
  const int64_t gm = ceil_div(a.rows, size), gn = ceil_div(a.cols, size);
  const unsigned grid = static_cast<unsigned>(gm * gn * a.count);
  if (size == 256)
    orth_apply_kernel<MmShape<true, true, BK, 256, 256, 2, 4>, LAST, T>
        <<<grid, 512, 0, s>>>(m, t, a, gm, gn, a_bytes, b_bytes, to, ldp);
  else if (size == 128)
    orth_apply_kernel<MmShape<true, true, BK, 128, 128, 2, 2>, LAST, T>
        <<<grid, 256, 0, s>>>(m, t, a, gm, gn, a_bytes, b_bytes, to, ldp);
  else
    orth_apply_kernel<MmShape<true, true, BK, 64, 64, 2, 2>, LAST, T>
        <<<grid, 256, 0, s>>>(m, t, a, gm, gn, a_bytes, b_bytes, to, ldp);
}

template <typename T>
hipError_t launch_orth_t(const OrthMats &t, const OrthArgs &a, char *ws, hipStream_t s) {
  const OrthPlan p = orth_plan(a.rows, a.cols, a.count);
  uint16_t *X[2] = {reinterpret_cast<uint16_t *>(ws + p.x[0]), reinterpret_cast<uint16_t *>(ws + p.x[1])};
  uint16_t *A = reinterpret_cast<uint16_t *>(ws + p.a), *Q = reinterpret_cast<uint16_t *>(ws + p.q);
  double *part = reinterpret_cast<double *>(ws + p.part);
  const bool tall = a.rows > a.cols;
  orth_begin_kernel<T><<<p.sums * a.count, 256, 0, s>>>(t, a, p.sums, part);
  const int64_t turns = ceil_div(a.rows * p.ldx, kBlockElems);
  const int groups = static_cast<int>(turns < 1024 ? turns : 1024);
  orth_split_kernel<T><<<groups * a.count, 256, 0, s>>>(t, a, groups, p.sums, part, X[0], p.ldx);
  const int64_t xplane = a.rows * p.ldx, aplane = p.n * p.lda;
  for (int i = 0; i < a.steps; ++i) {
    uint16_t *x = X[i & 1], *next = X[~i & 1];
    MmArgs m = {};
    m.k = tall ? a.rows : a.cols;
    m.a.ld = m.b.ld = p.ldx;
    m.a.n = m.b.n = tall ? p.ldx : a.rows;
    const bool whole = sizeof(T) == 4, last = i + 1 == a.steps;
    planes(m, x, xplane, x, xplane, whole ? kAll : kHigh);
    if (tall)
      run_sym<false, false>(m, p.n, p.lda, a.count, 4 * xplane, nullptr, A, true, s);
    else
      run_sym<true, false>(m, p.n, p.lda, a.count, 4 * xplane, nullptr, A, true, s);
    m.k = p.n;
    m.a.ld = m.b.ld = p.lda;
    m.a.n = m.b.n = p.n;
    planes(m, A, aplane, A, aplane, whole || i + 2 >= a.steps ? kAll : kHigh);
    run_sym<true, true>(m, p.n, p.lda, a.count, 4 * aplane, A, Q, whole, s);
    if (tall) {
      m.a.ld = p.ldx;
      m.a.n = a.rows;
      planes(m, x, xplane, Q, aplane, whole ? kAll : last ? kHigh : kBothOfA);
      if (last)
        run_apply<true, true, T>(m, t, a, 4 * xplane, 4 * aplane, next, p.ldx, s);
      else
        run_apply<true, false, T>(m, t, a, 4 * xplane, 4 * aplane, next, p.ldx, s);
    } else {
      m.b.ld = p.ldx;
      m.b.n = p.ldx;
      planes(m, Q, aplane, x, xplane, whole ? kAll : last ? kHigh : kBothOfB);
      if (last)
        run_apply<false, true, T>(m, t, a, 4 * aplane, 4 * xplane, next, p.ldx, s);
      else
        run_apply<false, false, T>(m, t, a, 4 * aplane, 4 * xplane, next, p.ldx, s);
    }
  }
  return hipGetLastError();
}

}  // namespace

size_t orth_workspace_bytes(int64_t rows, int64_t cols, int64_t count) {
  return orth_plan(rows, cols, count < OrthMats::kMost ? count : OrthMats::kMost).total;
}

hipError_t launch_orth(int dt, const OrthMats &t, const OrthArgs &a, void *ws, hipStream_t s) {
  return dt == 0 ? launch_orth_t<float>(t, a, static_cast<char *>(ws), s)
                 : launch_orth_t<bf16_t>(t, a, static_cast<char *>(ws), s);
}

}  // namespace sn
