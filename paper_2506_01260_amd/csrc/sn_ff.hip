// The gated feed-forward block of N tokens:
//   G = X Wg,  U = X Wu,  H = act(G) * U              X: N x d, Wg, Wu: d x ff
// and its backward from the stored G and U,
//   dG = dH U act'(G),  dU = dH act(G),
//   dX = dG Wg^T + dU Wu^T,  gWg = X^T dG,  gWu = X^T dU.
//
// Forward: one kernel takes both products, a wave holding the same columns of G and U,
// and writes H from the 32-bit sums.  Backward: dG and dU are made once, elementwise, and
// rounded to dt, as they are returned: the three products read them so (dX as one product over 2 ff,
// both weights' gradients in one launch).  In bf16 that leaves dX and the weights' gradients off by
// 2.3e-3 of their norm, 1.7e-3 of it their own rounding; dG and dU in two planes would leave 1.7e-3 and
// take twice the products.
// float32 operands are split in three bf16 planes (24 bits together, hi + mid + lo) and the six products
// down to 2^-24 of the largest are added up: at the peak rates 2.6 times what the float32 matrix
// instructions do.  Up to 384 tokens copying the weights' planes would take longer than that gains: the
// forward and dX multiply them as they are.  Matrices that are not 16-byte aligned, or
// whose rows are no multiple of 8 elements, are copied to padded rows first.
//
// Bounds and times: many tokens the matrix cores (32768 x 4096 x 14336 with G and U kept
// 6.4 to 6.8 ms, 1130 to 1200 TFLOP/s; backward of 4999 x 1600 x 4267 400 us, of it 77 to make
// and copy operands of odd sizes; of 2048 x 1024 x 4096 in float32 449), few the weights'
// reading (4096 x 14336: one token 52 us, 4.5 TB/s, the kernel alone 40; 48 tokens 55).
#include <initializer_list>

#include "sn_internal.h"
#include "sn_mm.h"
#include "sn_rows.h"

namespace sn {

namespace {

// ---- activations -------------------------------------------------------------------
__device__ __forceinline__ float ff_act(int act, float g) {
  if (act == kActRelu) return g < 0.0f ? 0.0f : g;
  if (act == kActSilu) return g / (1.0f + expf(-g));
  return 0.5f * g * erfcf(-0.70710678f * g);
}
// act and its derivative
__device__ __forceinline__ void ff_act2(int act, float g, float &a, float &da) {
  if (act == kActRelu) {
    a = g < 0.0f ? 0.0f : g;
    da = g > 0.0f ? 1.0f : 0.0f;
  } else if (act == kActSilu) {
    const float p = 1.0f / (1.0f + expf(-g));
    a = g * p;
    da = p * (1.0f + g * (1.0f - p));
  } else {
    const float p = 0.5f * erfcf(-0.70710678f * g);
    a = g * p;
    da = fmaf(0.39894228f * g, expf(-0.5f * g * g), p);
  }
}

// ---- eight values of a row -----------------------------------------------------------
template <typename T>
__device__ __forceinline__ void get8(const T *row, int64_t c, int64_t n, float (&x)[8]) {
  constexpr int E = Piece<T>::E;
#pragma unroll
  for (int h = 0; h < 8 / E; ++h) {
    float v[E];
    if (c + 8 <= n)
      Piece<T>::unpack(load_piece(row + c + h * E), v);
    else
      load_part(row, c + h * E, n, 0.0f, v);
#pragma unroll
    for (int e = 0; e < E; ++e) x[h * E + e] = v[e];
  }
}
template <typename T>
__device__ __forceinline__ void put8(T *row, int64_t c, int64_t n, const float (&x)[8]) {
  constexpr int E = Piece<T>::E;
#pragma unroll
  for (int h = 0; h < 8 / E; ++h) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = x[h * E + e];
    if (c + 8 <= n)
      store_piece(row + c + h * E, Piece<T>::pack(v));
    else
      store_part(row, c + h * E, n, v);
  }
}
// A value's bf16, as a float; the next one towards 0 where that would be infinite.
__device__ __forceinline__ float bf16_near(float v) {
  const float r = __uint_as_float(pack_bf16x2(0.0f, v) & 0xFFFF0000u);
  return fabsf(r) == INFINITY ? __uint_as_float(__float_as_uint(v) & 0xFFFF0000u) : r;
}
// The planes of eight values: bf16 as it is, float32 as three bf16 that add up to it
// exactly (8 bits each, signed), the second times 2^7 and the third times 2^14: at most a half and
// a quarter of the first, so that their products do not overflow before it does, and no
// smaller than it by more than their leading zeros.  An infinity or a NaN has nothing left
// after the first.
constexpr float kUp = 128.0f;
template <typename T>
__device__ __forceinline__ void put_planes(uint16_t *to, int64_t plane, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4 *>(to) = Piece<bf16_t>::pack(x);
  } else {
    float h[8], m[8], l[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] = bf16_near(x[e]);
      const float r = fabsf(x[e]) <= 3.4028235e38f ? x[e] - h[e] : 0.0f;
      m[e] = bf16_near(r);
      l[e] = (r - m[e]) * (kUp * kUp);
      m[e] *= kUp;
    }
    *reinterpret_cast<u32x4 *>(to) = Piece<bf16_t>::pack(h);
    *reinterpret_cast<u32x4 *>(to + plane) = Piece<bf16_t>::pack(m);
    *reinterpret_cast<u32x4 *>(to + 2 * plane) = Piece<bf16_t>::pack(l);
  }
}

// ---- operands in padded planes -----------------------------------------------------------
// rows x cols (stride ld) to planes of rows x ldp, ldp = cols up to a multiple of 8, 0 in
// the columns past cols.
template <typename T>
__global__ __launch_bounds__(256) void ff_pack_kernel(const T *src, int64_t rows, int64_t cols,
                                                      int64_t ld, uint16_t *dst, int64_t ldp) {
  const int64_t id = group_number() * 256 + threadIdx.x, per = ldp / 8;
  const int64_t r = id / per, c = (id - r * per) * 8;
  if (r >= rows) return;
  float x[8];
  get8(src + r * ld, c, cols, x);
  put_planes<T>(dst + r * ldp + c, rows * ldp, x);
}

// dG and dU, eight columns a thread; with planes, also as operands.
template <typename T>
__global__ __launch_bounds__(256) void ff_dact_kernel(FfGradArgs a, uint16_t *pg, uint16_t *pu,
                                                      int64_t ldp) {
  const int64_t id = group_number() * 256 + threadIdx.x, per = (a.ff + 7) / 8;
  const int64_t r = id / per, c = (id - r * per) * 8;
  if (r >= a.N) return;
  float g[8], u[8], h[8], dg[8], du[8];
  get8(static_cast<const T *>(a.G) + r * a.ldg, c, a.ff, g);
  get8(static_cast<const T *>(a.U) + r * a.ldg, c, a.ff, u);
  get8(static_cast<const T *>(a.dH) + r * a.lddh, c, a.ff, h);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f, df;
    ff_act2(a.act, g[e], f, df);
    dg[e] = h[e] * u[e] * df;
    du[e] = h[e] * f;
  }
  put8(static_cast<T *>(a.dG) + r * a.ldd, c, a.ff, dg);
  put8(static_cast<T *>(a.dU) + r * a.ldd, c, a.ff, du);
  if (pg) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e >= a.ff) dg[e] = du[e] = 0.0f;
    put_planes<T>(pg + r * ldp + c, a.N * ldp, dg);
    put_planes<T>(pu + r * ldp + c, a.N * ldp, du);
  }
}

// ---- forward: both products and the activation ------------------------------------------
template <typename T>
struct FfEpilogue {
  FfArgs a;
  template <class S>
  __device__ __forceinline__ void row(const MmPlace &, int64_t row, int64_t col0,
                                      f32x4 (&acc)[S::TN]) const {
    constexpr int TP = S::TN / 2;
    if (row >= a.N) return;
#pragma unroll
    for (int j = 0; j < TP; ++j) {
      const int64_t col = col0 + j * 16, left = a.ff - col;
      if (left <= 0) continue;
      const f32x4 g = acc[j], u = acc[j + TP];
      f32x4 h;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = ff_act(a.act, g[e]) * u[e];
      put4(static_cast<T *>(a.H) + row * a.ldh + col, left, h);
      if (a.G) {
        put4(static_cast<T *>(a.G) + row * a.ldg + col, left, g);
        put4(static_cast<T *>(a.U) + row * a.ldg + col, left, u);
      }
    }
  }
};

// H (G, U) from the parts of the sums: parts x {G, U} x N x ff, added in order.
template <typename T>
__global__ __launch_bounds__(256) void ff_join_kernel(FfArgs a, int parts) {
  const int64_t id = group_number() * 256 + threadIdx.x, per = (a.ff + 3) / 4;
  const int64_t r = id / per, c = (id - r * per) * 4, left = a.ff - c;
  if (r >= a.N) return;
  f32x4 g = {0, 0, 0, 0}, u = {0, 0, 0, 0};
  const float *p = a.part + r * a.ff + c;
  for (int q = 0; q < parts; ++q, p += 2 * a.N * a.ff) {
    g += get4(p, left);
    u += get4(p + a.N * a.ff, left);
  }
  f32x4 h;
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = ff_act(a.act, g[e]) * u[e];
  put4(static_cast<T *>(a.H) + r * a.ldh + c, left, h);
  if (a.G) {
    put4(static_cast<T *>(a.G) + r * a.ldg + c, left, g);
    put4(static_cast<T *>(a.U) + r * a.ldg + c, left, u);
  }
}

// ---- forward of up to 8 bf16 tokens: the weights stream by ------------------------------
// A workgroup of 16 waves (8 for more than 4 tokens) takes 64 columns of both weights and a
// slice of d (all of it where there are enough columns for the CUs); a lane takes 16 bytes of
// a weight's row, the lanes beside it the rest of the row's 64 columns and further rows.
// Columns past ff: the row's last piece, whose values are stored by two lanes alike.
constexpr int kVecCols = 64;
constexpr int vec_waves(int nb) { return nb <= 4 ? 16 : 8; }
constexpr int vec_slice(int nb) { return nb <= 4 ? 4096 : 2048; }  // longest
template <int NB>
__global__ __launch_bounds__(vec_waves(NB) * 64) void ff_vec_kernel(FfArgs a, int slices) {
  using T = bf16_t;
  constexpr int kVecWaves = vec_waves(NB);
  constexpr int E = Piece<T>::E, LANES = kVecCols / E, ROWS = 64 / LANES, STEP = ROWS * kVecWaves;
  constexpr int UN = NB <= 4 ? 4 : 2, NT = kVecWaves * 64;
  __shared__ __attribute__((aligned(16))) float xs[vec_slice(NB) * NB];
  __shared__ float red[kVecWaves][NB][2][kVecCols];
  const int64_t strips = (a.ff + kVecCols - 1) / kVecCols, id = group_number();
  if (id >= strips * slices) return;
  const int64_t slice = id / strips, strip = id - slice * strips;
  const int64_t k0 = slice * a.d / slices, k1 = (slice + 1) * a.d / slices;
  const int len = static_cast<int>(k1 - k0), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = strip * kVecCols + lane % LANES * E, cb = c < a.ff - E ? c : a.ff - E;
  const int row = wave * ROWS + lane / LANES;
  const T *wg = static_cast<const T *>(a.Wg) + (k0 + row) * a.ldw + cb;
  const int64_t twin = static_cast<const T *>(a.Wu) - static_cast<const T *>(a.Wg);
  float acc[NB][2][E] = {};
  const auto add = [&](int k, u32x4 vg, u32x4 vu) {
    float g[E], u[E];
    Piece<T>::unpack(vg, g);
    Piece<T>::unpack(vu, u);
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      const float x = xs[k * NB + t];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        acc[t][0][e] = fmaf(x, g[e], acc[t][0][e]);
        acc[t][1][e] = fmaf(x, u[e], acc[t][1][e]);
      }
    }
  };
  // the first rows are on their way while the tokens are put into the LDS
  u32x4 vg[UN], vu[UN];
  int k = row;
  const bool any = k + (UN - 1) * STEP < len;
  if (any) {
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      vg[i] = load_piece(wg + i * STEP * a.ldw);
      vu[i] = load_piece(wg + i * STEP * a.ldw + twin);
    }
  }
#pragma unroll 1
  for (int t = 0; t < NB; ++t) {
    const T *x = static_cast<const T *>(a.X) + t * a.ldx + k0;
#pragma unroll 2
    for (int q = threadIdx.x; q < len; q += NT) xs[q * NB + t] = t < a.N ? to_f32(x[q]) : 0.0f;
  }
  __syncthreads();
  if (any) {
#pragma unroll 1
    for (; k + (UN - 1) * STEP < len; k += UN * STEP) {
      // past the last rows these ones again, so that no branch parts the loads
      const T *next = k + (2 * UN - 1) * STEP < len ? wg + UN * STEP * a.ldw : wg;
      wg += UN * STEP * a.ldw;
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        add(k + i * STEP, vg[i], vu[i]);
        vg[i] = load_piece(next + i * STEP * a.ldw);
        vu[i] = load_piece(next + i * STEP * a.ldw + twin);
      }
    }
  }
#pragma unroll 1
  for (; k < len; k += STEP, wg += STEP * a.ldw) add(k, load_piece(wg), load_piece(wg + twin));
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v = acc[t][q][e];
#pragma unroll
        for (int m = LANES; m < 64; m <<= 1) v += __shfl_xor(v, m);
        if (lane < LANES) red[wave][t][q][lane * E + e] = v;
      }
  __syncthreads();
  for (int i = threadIdx.x; i < NB * kVecCols; i += NT) {
    const int t = i / kVecCols, j = i % kVecCols;
    const int64_t c1 = strip * kVecCols + j / E * E;
    const int64_t col = (c1 < a.ff - E ? c1 : a.ff - E) + j % E;
    if (t >= a.N || c1 >= a.ff) continue;
    float s[2] = {0.0f, 0.0f};
#pragma unroll 4
    for (int w = 0; w < kVecWaves; ++w) {
      s[0] += red[w][t][0][j];
      s[1] += red[w][t][1][j];
    }
    if (slices > 1) {
      float *p = a.part + (slice * 2 * a.N + t) * a.ff + col;
      p[0] = s[0];
      p[a.N * a.ff] = s[1];
    } else {
      static_cast<T *>(a.H)[t * a.ldh + col] = from_f32<T>(ff_act(a.act, s[0]) * s[1]);
      if (a.G) {
        static_cast<T *>(a.G)[t * a.ldg + col] = from_f32<T>(s[0]);
        static_cast<T *>(a.U)[t * a.ldg + col] = from_f32<T>(s[1]);
      }
    }
  }
}

// ---- products of up to 384 float32 tokens: the weights as they are -----------------------------------
// Of A (tokens, k contiguous) and a weight: forward X Wg and X Wu (KC false: a weight's rows are k), or
// dX's dG Wg^T and dU Wu^T (KC: its rows are the output's columns).  A workgroup takes 16 TT tokens, a
// slice of k and 64 columns of both weights (KC: 128 of one); every other wave has one half of the
// columns, each pair of waves 16 of the 64 k of a round.  The tokens' part of a round lies in the LDS, in
// two places in turn; weights come straight to registers, D - 1 rounds ahead.  In the float32 matrix
// instruction 16 x 16 x 4 lane l = 16 g + n supplies k = g of row n of either operand; here instruction s
// of 16 k values takes k = 4 g + s, so that a lane's four values of a token are one 16-byte read, and
// of a weight's row (KC) one load.  Where rows are k, a lane's 16 bytes are columns 4 n + e, so the
// products of its value e have rows n for columns 4 n + e, and the sums of all four are 16
// neighbouring columns of the token n.  A sum is four chains of a quarter of the slice's k.
// Piece p of a token's row lies at p ^ (token % 16): the 16 rows of a read are in different banks.
// Bound by the weights' reading up to 32 tokens (4096 x 14336: one token 84 us, 5.6 TB/s, 32 tokens 93), then
// by the instruction (64 tokens 149, 128 253, 256 501: 120 TFLOP/s, 137 on the 224 CUs that have work; the
// same of tiles whose weights go through the LDS too 185, 315, 530).
struct FewArgs {
  const float *A[2], *B[2];  // KC: one for each segment; else A[0], and both weights
  int64_t lda, ldb, N, k, cols;
  int slices;  // of k; KC: those of a segment, behind each other
  float *part;
  FfArgs out;  // not KC, one slice
};
constexpr int kFewK = 64, kFewWaves = 8;
template <bool KC, int TT>
__global__ __launch_bounds__(kFewWaves * 64, 2) void ff_few_kernel(FewArgs a) {
  // (of an odd TT the last load's upper half has no tokens, and lies behind them in the LDS)
  constexpr int NT = kFewWaves * 64, TOK = 16 * TT, L = (TT + 1) / 2, XS = 32 * L * kFewK, D = TT <= 4 ? 4 : 2;
  constexpr int RED = kFewWaves * 16 * 64, BN = KC ? 128 : 64;
  __shared__ __attribute__((aligned(16))) float lds[2 * XS > RED ? 2 * XS : RED];
  const int64_t strips = (a.cols + BN - 1) / BN, blocks = (a.N + TOK - 1) / TOK;
  const int64_t all = strips * blocks * a.slices * (KC ? 2 : 1), id = group_number();
  if (id >= all) return;
  const int64_t number = mm_order(id, all), part = number / blocks;
  const int64_t slice = part / strips, strip = part - slice * strips, first = (number - part * blocks) * TOK;
  const int seg = slice >= a.slices ? 1 : 0;
  const int64_t rounds = (a.k + kFewK - 1) / kFewK, sl = slice - seg * a.slices;
  const int64_t k0 = sl * rounds / a.slices * kFewK, k1 = min((sl + 1) * rounds / a.slices * kFewK, a.k);
  const int64_t full = (k1 - k0) / kFewK, tail = k1 - k0 - full * kFewK;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, n = lane & 15, half = wave & 1, kw = 16 * (wave >> 1) + 4 * g;
  // tokens: piece p of row r, L of them (past the last token that one again: nothing is made of it)
  const int p = threadIdx.x & 15, r0 = threadIdx.x >> 4;
  const float *A = a.A[seg] + k0;
  int64_t at[L];
#pragma unroll
  for (int j = 0; j < L; ++j) at[j] = min(first + r0 + j * (NT / 16), a.N - 1) * a.lda + 4 * p;
  f32x4 xr[L];
  const auto store = [&](float *to) {
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int r = r0 + j * (NT / 16);
      *reinterpret_cast<f32x4 *>(to + r * kFewK + ((p ^ (r & 15)) << 2)) = xr[j];
    }
  };
  const auto fetch = [&](int64_t round) {
#pragma unroll
    for (int j = 0; j < L; ++j) xr[j] = get4(A + round * kFewK + at[j], 4);
  };
  const auto token = [&](const float *from, int i) {
    return *reinterpret_cast<const f32x4 *>(from + (16 * i + n) * kFewK + (((wave >> 1) * 4 + g) ^ n) * 4);
  };
  // weights: KC rows c0 + 16 f + n at k = kw .., else rows kw + s at columns c0 + 4 n ..
  const int64_t c0 = strip * BN + (KC ? 64 * half : 0), cn = c0 + 4 * n;
  const float *B = a.B[KC ? seg : half] + (KC ? k0 : k0 * a.ldb);
  const float *bp[4];
#pragma unroll
  for (int s = 0; s < 4; ++s)
    bp[s] = KC ? B + min(c0 + 16 * s + n, a.cols - 1) * a.ldb + kw : B + (kw + s) * a.ldb + min(cn, a.cols - 4);
  f32x4 w[D][4], acc[TT][4];
  const auto weights = [&](f32x4(&to)[4], int64_t round) {
    const int64_t by = KC ? round * kFewK : round * kFewK * a.ldb;
#pragma unroll
    for (int s = 0; s < 4; ++s) to[s] = get4(bp[s] + by, 4);
  };
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = f32x4{0, 0, 0, 0};
  // value e of the sums: KC fragment e, else columns 4 n + e
  const auto multiply = [&](int i, const f32x4 &x, const f32x4(&v)[4]) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[i][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(KC ? v[e][s] : v[s][e], x[s], acc[i][e], 0, 0, 0);
  };
  if (full > 0) {
    fetch(0);
#pragma unroll
    for (int d = 0; d < D - 1; ++d) weights(w[d], min(static_cast<int64_t>(d), full - 1));
    store(lds);
    fetch(full > 1 ? 1 : 0);
    lds_barrier();
    f32x4 x = token(lds, 0);
    int cur = 0;
#pragma unroll 1
    for (int64_t r = 0; r < full; r += D) {
#pragma unroll
      for (int u = 0; u < D; ++u) {
        if (r + u >= full) break;
        const int64_t now = r + u, last = full - 1;
        store(lds + (XS - cur));
        fetch(now + 2 < last ? now + 2 : last);
        weights(w[(u + D - 1) % D], now + D - 1 < last ? now + D - 1 : last);
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          if (i == TT - 1) {
            lds_barrier();
            cur = XS - cur;
          }
          const f32x4 now_x = x;
          x = token(lds + cur, (i + 1) % TT);  // behind the last round, what nothing uses
          multiply(i, now_x, w[u]);
          // other work between the products, which run for 32 cycles each
#pragma unroll
          for (int m = 0; m < 16; ++m) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
          }
          if (i == TT - 1 || i == TT - 2) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  if (tail > 0) {
    lds_barrier();
    const float *from = A + full * kFewK;
#pragma unroll
    for (int j = 0; j < L; ++j) xr[j] = 4 * p < tail ? get4(from + at[j], tail - 4 * p) : f32x4{0, 0, 0, 0};
    store(lds);
    const int64_t by = KC ? full * kFewK : full * kFewK * a.ldb;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int64_t left = tail - kw - (KC ? 0 : s);
      w[0][s] = left > 0 ? get4(bp[s] + by, KC ? left : 4) : f32x4{0, 0, 0, 0};
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < TT; ++i) multiply(i, token(lds, i), w[0]);
  }
  // the waves' sums are added in order, 16 tokens at a time
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    __syncthreads();
    float *to = lds + (wave * 16 + n) * 64;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4 *>(to + (((KC ? 4 * e + g : 4 * g + e) ^ n) << 2)) =
          KC ? acc[i][e] : f32x4{acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
    __syncthreads();
    // four columns of both halves' sums: of both weights, or neighbours
    if (threadIdx.x >= 256) continue;
    const int t = threadIdx.x >> 4, j = (threadIdx.x & 15) * 4;
    const int64_t row = first + 16 * i + t;
    if (row >= a.N) continue;
    f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) s[v & 1] += *reinterpret_cast<const f32x4 *>(lds + (v * 16 + t) * 64 + (j ^ t << 2));
    if constexpr (KC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t col = strip * BN + 64 * h + j;
        if (col < a.cols) put4(a.part + (slice * a.N + row) * a.cols + col, a.cols - col, s[h]);
      }
    } else {
      if (strip * BN + j >= a.cols) continue;
      const int64_t col = min(strip * BN + j, a.cols - 4);
      if (a.slices > 1) {
        float *q = a.part + (slice * 2 * a.N + row) * a.cols + col;
        put4(q, 4, s[0]);
        put4(q + a.N * a.cols, 4, s[1]);
      } else {
        f32x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = ff_act(a.out.act, s[0][e]) * s[1][e];
        put4(static_cast<float *>(a.out.H) + row * a.out.ldh + col, 4, h);
        if (a.out.G) {
          put4(static_cast<float *>(a.out.G) + row * a.out.ldg + col, 4, s[0]);
          put4(static_cast<float *>(a.out.U) + row * a.out.ldg + col, 4, s[1]);
        }
      }
    }
  }
}

// ---- products of the backward -----------------------------------------------------------
// C (M x N; C2 for the second matrix) = the product, added to what is there with `add`.
template <typename T>
struct FfOut {
  T *C, *C2;
  int64_t M, N, ldc;
  int add;
  template <class S>
  __device__ __forceinline__ void row(const MmPlace &p, int64_t row, int64_t col0,
                                      f32x4 (&acc)[S::TN]) const {
    if (row >= M) return;
    T *to = (p.z ? C2 : C) + row * ldc + col0;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int64_t left = N - col0 - j * 16;
      if (left <= 0) continue;
      f32x4 v = acc[j];
      if (add) v += get4(to + j * 16, left);
      put4(to + j * 16, left, v);
    }
  }
};
template <typename T>
__global__ __launch_bounds__(256) void ff_zero_kernel(FfOut<T> o) {
  const int64_t id = group_number() * 256 + threadIdx.x, per = (o.N + 3) / 4;
  const int64_t r = id / per, c = (id - r * per) * 4;
  if (r >= 2 * o.M) return;
  put4((r < o.M ? o.C + r * o.ldc : o.C2 + (r - o.M) * o.ldc) + c, o.N - c, f32x4{0, 0, 0, 0});
}

// dX: the parts of its sums, in order.
__global__ __launch_bounds__(256) void ff_sum_kernel(const float *part, int parts, FfOut<float> o) {
  const int64_t id = group_number() * 256 + threadIdx.x, per = (o.N + 3) / 4;
  const int64_t r = id / per, c = (id - r * per) * 4, left = o.N - c;
  if (r >= o.M) return;
  f32x4 v = {0, 0, 0, 0};
  const float *p = part + r * o.N + c;
  for (int q = 0; q < parts; ++q, p += o.M * o.N) v += get4(p, left);
  put4(o.C + r * o.ldc + c, left, v);
}

// ---- plans --------------------------------------------------------------------------------
constexpr int kPlanes[2] = {3, 1};  // of float32, bf16
int segs_of(int dt) { return dt == 0 ? 6 : 1; }
int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
bool direct(int dt, const void *p, int64_t cols, int64_t ld) {
  return dt == 1 && cols % 8 == 0 && ld % 8 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

struct Space {  // of a workspace
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  }
};

// Segments of `pairs` products of operands, pair q with an operand's planes from p[q] on
// (`plane` elements each): for float32 the products of planes 2^-14, 2^-7 and 1, of all
// pairs, in this order.
const int kFirst[6] = {1, 0, 2, 0, 1, 0}, kSecond[6] = {1, 2, 0, 1, 0, 0};
void set_segs(MmArgs &m, int dt, int pairs, std::initializer_list<const void *> a, int64_t aplane,
              std::initializer_list<const void *> b, int64_t bplane) {
  const int from[4] = {0, 3, 5, 6};
  m.segs = pairs * segs_of(dt);
  m.run[0] = dt == 0 ? 3 * pairs : m.segs;
  m.run[1] = dt == 0 ? 5 * pairs : m.segs;
  m.factor = 1.0f / kUp;
  int at = 0;
  for (int r = 0; r < 3; ++r)
    for (int q = 0; q < pairs; ++q)
      for (int s = from[r]; s < from[r + 1]; ++s) {
        if (dt != 0 && r < 2) continue;
        m.a.p[at] = static_cast<const uint16_t *>(a.begin()[q]) + (dt == 0 ? kFirst[s] * aplane : 0);
        m.b.p[at++] = static_cast<const uint16_t *>(b.begin()[q]) + (dt == 0 ? kSecond[s] * bplane : 0);
      }
}

dim3 pieces_grid(int64_t rows, int64_t per) { return groups_grid(ceil_div(rows * per, 256)); }

template <typename T>
void pack(const void *src, int64_t rows, int64_t cols, int64_t ld, uint16_t *dst, hipStream_t s) {
  ff_pack_kernel<T><<<pieces_grid(rows, up8(cols) / 8), 256, 0, s>>>(
      static_cast<const T *>(src), rows, cols, ld, dst, up8(cols));
}

// Slices of d: one where the columns alone fill most CUs, else enough for one and a half
// workgroups to each, of 64 rows or more.
int vec_slices(int64_t N, int64_t d, int64_t ff) {
  const int64_t strips = ceil_div(ff, kVecCols), least = ceil_div(d, vec_slice(N <= 4 ? 4 : 8));
  const int64_t want = strips >= 160 ? 1 : ceil_div(384, strips), most = ceil_div(d, 64);
  const int64_t n = want < most ? want : most;
  return static_cast<int>(n > least ? n : least);
}
// bf16 weights of whole pieces are as fast through the matrix cores from two tokens on
// (4096 x 14336: one token 52 us, 16 tokens 54); others would have to be copied first.
bool by_vec(int dt, int64_t N, int64_t ff) { return dt == 1 && N <= (ff % 8 == 0 ? 1 : 8) && ff >= 8; }

// float32 weights as they are, or copied into planes first.  us, so, in planes, and of elementary float32
// products: forward 4096 x 14336 with 160 tokens 337, 557, 345, with 320 681, 768, 747, with 384 759,
// 774, 883, with 512 915, 832, 1020; 1600 x 4267 with 384 106, 115, 130, with 448 158, 127, 144; backward
// (dX so, or all in planes) 4096 x 14336 with 128 484, 768, 597, with 384 1287, 1369, 1532, with 512 1612,
// 1545, 1888.
constexpr int64_t kFewFloats = 384;
bool by_few(int dt, int64_t N) { return dt == 0 && N <= kFewFloats; }
// Tiles of 16 tokens of a workgroup: up to 8 (more would not leave the registers), and as many as the
// fewest blocks of tokens need.
int few_tiles(int64_t N) { return static_cast<int>(ceil_div(N, 16 * ceil_div(N, 128))); }
// Slices of k by the time of as many rounds of workgroups as 256 CUs take, one each: 0.47 us for 64 k of 16
// tokens, 5 for a workgroup's start and end, and where there are parts, writing and adding them.
int few_slices(int64_t N, int64_t strips, int64_t segs, int64_t k, int64_t cols) {
  const int64_t tt = few_tiles(N), groups = strips * ceil_div(N, 16 * tt) * segs, rounds = ceil_div(k, kFewK);
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 16 && (s == 1 || rounds / s >= 2); ++s) {
    double us = static_cast<double>(ceil_div(groups * s, 256)) * (static_cast<double>(ceil_div(rounds, s)) * 0.47 * static_cast<double>(tt < 2 ? 2 : tt) + 5.0);
    if (s * segs > 1) us += 4.0 + 2.0 * sizeof(float) * static_cast<double>(s * segs * N * cols) / 5e6;
    if (s > 1 && us >= least) continue;
    least = us;
    best = s;
  }
  return best;
}

constexpr int64_t kFew = 64;
// Steps of weights on their way to the LDS while few tokens are multiplied: 48 tokens take 55 us
// with 6, 77 with 2.
constexpr int kFewDepth = 6;
// bf16 tokens for one row of tiles of 256 x 128, on half to all of the CUs: long columns of the
// weights come from memory, and two steps of them on their way outdo what smaller tiles share in
// the L2.  us, so and in tiles by mm_plan: 4096 x 14336 with 130 tokens 74 and 91, with 256 86
// and 104; 2048 x 8192 39 and 40, 39 and 45; 8192 x 14336 133 and 167, 155 and 191; of shorter
// columns (1024 x 8192) 25 and 22, of fewer (1024 x 4096) 23 and 14, of more (8192 x 28672) 275
// and 231.
bool in_one(int dt, int64_t N, int64_t d, int64_t ff) {
  const int64_t groups = ceil_div(2 * ff, 128);
  return dt == 1 && N > 128 && N <= 256 && d >= 2048 && groups >= 128 && groups <= 256;
}
constexpr int kOneDepth = 3;
enum { kFewTile = 0, kOneTile = 1 };  // MmPlan's size beside 64, 128 and 256
MmPlan row_plan(int size, int64_t cols) {
  MmPlan p = {};
  p.size = size;
  p.grid.gm = 1;
  p.grid.gn = p.grid.whole = ceil_div(cols, 128);
  p.grid.mats = p.grid.splits = 1;
  return p;
}

struct FfPlan {
  bool vec, few, own_x, own_w;  // own: read in place
  MmPlan t;
  int slices;
  size_t x, w, part, total;
};
FfPlan ff_plan(int dt, int64_t N, int64_t d, int64_t ff, bool own_x, bool own_w) {
  FfPlan p = {};
  Space s;
  if (by_vec(dt, N, ff)) {
    p.vec = true;
    p.slices = vec_slices(N, d, ff);
    if (p.slices > 1) p.part = s.take(sizeof(float) * p.slices * 2 * N * ff);
  } else if (by_few(dt, N) && ff >= 4) {
    p.few = true;
    p.slices = few_slices(N, ceil_div(ff, 64), 1, d, 2 * ff);
    if (p.slices > 1) p.part = s.take(sizeof(float) * p.slices * 2 * N * ff);
  } else {
    p.own_x = own_x;
    p.own_w = own_w;
    // a paired tile has half its columns of either product
    p.t = N <= kFew              ? row_plan(kFewTile, 2 * ff)
          : in_one(dt, N, d, ff) ? row_plan(kOneTile, 2 * ff)
                                 : mm_plan(N, 2 * ff, 1, ceil_div(d, kMmK) * segs_of(dt));
    if (!own_x) p.x = s.take(2 * kPlanes[dt] * N * up8(d));
    if (!own_w) p.w = s.take(2 * 2 * kPlanes[dt] * d * up8(ff));
    p.part = s.take(p.t.part_bytes);
  }
  p.total = s.at;
  return p;
}

void launch_vec(const FfArgs &a, int slices, hipStream_t s) {
  const dim3 grid = groups_grid(ceil_div(a.ff, kVecCols) * slices);
  if (a.N == 1)
    ff_vec_kernel<1><<<grid, 1024, 0, s>>>(a, slices);
  else if (a.N <= 4)  // two tokens alone would take scratch memory
    ff_vec_kernel<4><<<grid, 1024, 0, s>>>(a, slices);
  else
    ff_vec_kernel<8><<<grid, 512, 0, s>>>(a, slices);
  if (slices > 1)
    ff_join_kernel<bf16_t><<<pieces_grid(a.N, ceil_div(a.ff, 4)), 256, 0, s>>>(a, slices);
}
template <bool KC>
void launch_few(const FewArgs &a, hipStream_t s) {
  const int tt = few_tiles(a.N);
  const dim3 grid = groups_grid(ceil_div(a.cols, KC ? 128 : 64) * a.slices * (KC ? 2 : 1) * ceil_div(a.N, 16 * tt));
  const auto run = [&](auto *kernel) { kernel<<<grid, kFewWaves * 64, 0, s>>>(a); };
  switch (tt) {
    case 1: return run(ff_few_kernel<KC, 1>);
    case 2: return run(ff_few_kernel<KC, 2>);
    case 3: return run(ff_few_kernel<KC, 3>);
    case 4: return run(ff_few_kernel<KC, 4>);
    case 5: return run(ff_few_kernel<KC, 5>);
    case 6: return run(ff_few_kernel<KC, 6>);
    case 7: return run(ff_few_kernel<KC, 7>);
    default: return run(ff_few_kernel<KC, 8>);
  }
}
const float *f32(const void *p) { return static_cast<const float *>(p); }

template <typename T>
hipError_t launch_ff_t(int dt, FfArgs a, const FfPlan &p, char *ws, hipStream_t s) {
  a.part = reinterpret_cast<float *>(ws + p.part);
  if (p.vec) {
    launch_vec(a, p.slices, s);
  } else if (p.few) {
    launch_few<false>(FewArgs{{f32(a.X)}, {f32(a.Wg), f32(a.Wu)}, a.ldx, a.ldw, a.N, a.d, a.ff, p.slices, a.part, a}, s);
    if (p.slices > 1)
      ff_join_kernel<float><<<pieces_grid(a.N, ceil_div(a.ff, 4)), 256, 0, s>>>(a, p.slices);
  } else {
    MmArgs m = {};
    m.k = a.d;
    const void *x = a.X, *wg = a.Wg, *wu = a.Wu;
    m.a.ld = a.ldx;
    m.a.n = a.N;
    m.b.ld = a.ldw;
    m.b.n = up8(a.ff);
    if (!p.own_x) {
      uint16_t *to = reinterpret_cast<uint16_t *>(ws + p.x);
      pack<T>(a.X, a.N, a.d, a.ldx, to, s);
      x = to;
      m.a.ld = up8(a.d);
    }
    if (!p.own_w) {
      uint16_t *to = reinterpret_cast<uint16_t *>(ws + p.w);
      uint16_t *to2 = to + kPlanes[dt] * a.d * up8(a.ff);
      pack<T>(a.Wg, a.d, a.ff, a.ldw, to, s);
      pack<T>(a.Wu, a.d, a.ff, a.ldw, to2, s);
      wg = to;
      wu = to2;
      m.b.ld = up8(a.ff);
    }
    m.b.twin = static_cast<const char *>(wu) - static_cast<const char *>(wg);
    set_segs(m, dt, 1, {x}, a.N * up8(a.d), {wg}, a.d * up8(a.ff));
    MmGrid g = p.t.grid;
    g.part = a.part;
    const FfEpilogue<T> e = {a};
    if constexpr (sizeof(T) == 2) {
      if (p.t.size == kOneTile) {
        mm_launch<MmShape<false, true, false, 256, 128, 4, 2, kOneDepth, true>>(m, g, e, s);
        return hipGetLastError();
      }
    }
    if (p.t.size == kFewTile)
      mm_launch<MmShape<false, true, false, 64, 128, 2, 2, kFewDepth, true>>(m, g, e, s);
    else if (p.t.size == 256)
      mm_launch<MmShape<false, true, false, 256, 256, 2, 4, 2, true>>(m, g, e, s);
    else if (p.t.size == 128)
      mm_launch<MmShape<false, true, false, 128, 128, 2, 2, 2, true>>(m, g, e, s);
    else
      mm_launch<MmShape<false, true, false, 64, 64, 2, 2, 4, true>>(m, g, e, s);
  }
  return hipGetLastError();
}

struct FfGradPlan {
  bool few, own_x, own_w, own_g;  // few: dX by it
  int slices;
  MmPlan tx, tw;
  size_t x, w, g, part, total;
};
FfGradPlan ff_grad_plan(int dt, int64_t N, int64_t d, int64_t ff, bool own_x, bool own_w, bool own_g) {
  FfGradPlan p = {};
  Space s;
  p.own_x = own_x;
  p.own_w = own_w;
  p.own_g = own_g;
  p.few = by_few(dt, N);
  p.tw = mm_plan(d, ff, 2, ceil_div(N, kMmK) * segs_of(dt));
  if (!own_x) p.x = s.take(2 * kPlanes[dt] * N * up8(d));
  if (p.few) {
    p.slices = few_slices(N, ceil_div(d, 128), 2, ff, d);
    p.tx.part_bytes = sizeof(float) * 2 * p.slices * N * d;
  } else {
    p.tx = mm_plan(N, d, 1, ceil_div(ff, kMmK) * 2 * segs_of(dt));
    if (!own_w) p.w = s.take(2 * 2 * kPlanes[dt] * d * up8(ff));
  }
  if (!own_g) p.g = s.take(2 * 2 * kPlanes[dt] * N * up8(ff));
  p.part = s.take(p.tx.part_bytes > p.tw.part_bytes ? p.tx.part_bytes : p.tw.part_bytes);
  p.total = s.at;
  return p;
}

template <bool K, typename T>
void run_mm(const MmArgs &m, const FfOut<T> &o, const MmPlan &t, float *part, hipStream_t s) {
  MmGrid g = t.grid;
  g.part = part;
  if (t.size == 256)
    mm_launch<MmShape<false, K, K, 256, 256, 2, 4>>(m, g, o, s);
  else if (t.size == 128)
    mm_launch<MmShape<false, K, K, 128, 128, 2, 2>>(m, g, o, s);
  else
    mm_launch<MmShape<false, K, K, 64, 64, 2, 2, 4>>(m, g, o, s);
}

template <typename T>
FfOut<T> out_of(const FfGradArgs &a) {
  return {static_cast<T *>(a.gWg), static_cast<T *>(a.gWu), a.d, a.ff, a.ldgw, a.add};
}

template <typename T>
hipError_t launch_ff_grad_t(int dt, const FfGradArgs &a, const FfGradPlan &p, char *ws,
                            hipStream_t s) {
  const int64_t ff8 = up8(a.ff), planes = kPlanes[dt];
  const void *x = a.X, *wg = a.Wg, *wu = a.Wu, *dg = a.dG, *du = a.dU;
  int64_t ldx = a.ldx, ldw = a.ldw, ldd = a.ldd;
  uint16_t *pg = nullptr, *pu = nullptr;
  if (!p.own_g) {
    dg = pg = reinterpret_cast<uint16_t *>(ws + p.g);
    du = pu = pg + planes * a.N * ff8;
    ldd = ff8;
  }
  ff_dact_kernel<T><<<pieces_grid(a.N, ff8 / 8), 256, 0, s>>>(a, pg, pu, ldd);
  const bool want_w = a.gWg != nullptr;
  if (!p.own_x && want_w) {
    uint16_t *to = reinterpret_cast<uint16_t *>(ws + p.x);
    pack<T>(a.X, a.N, a.d, a.ldx, to, s);
    x = to;
    ldx = up8(a.d);
  }
  if (!p.own_w && !p.few && a.dX) {
    uint16_t *to = reinterpret_cast<uint16_t *>(ws + p.w), *to2 = to + planes * a.d * ff8;
    pack<T>(a.Wg, a.d, a.ff, a.ldw, to, s);
    pack<T>(a.Wu, a.d, a.ff, a.ldw, to2, s);
    wg = to;
    wu = to2;
    ldw = ff8;
  }
  float *part = reinterpret_cast<float *>(ws + p.part);
  if (a.dX && p.few) {
    if constexpr (sizeof(T) == 4) {
      launch_few<true>(FewArgs{{f32(a.dG), f32(a.dU)}, {f32(a.Wg), f32(a.Wu)}, a.ldd, a.ldw, a.N, a.ff, a.d, p.slices, part, {}}, s);
      ff_sum_kernel<<<pieces_grid(a.N, ceil_div(a.d, 4)), 256, 0, s>>>(
          part, 2 * p.slices, FfOut<float>{static_cast<float *>(a.dX), nullptr, a.N, a.d, a.lddx, 0});
    }
  } else if (a.dX) {
    MmArgs m = {};
    m.k = a.ff;
    m.a.ld = ldd;
    m.a.n = a.N;
    m.b.ld = ldw;
    m.b.n = a.d;
    set_segs(m, dt, 2, {dg, du}, a.N * ff8, {wg, wu}, a.d * ff8);
    run_mm<true, T>(m, {static_cast<T *>(a.dX), nullptr, a.N, a.d, a.lddx, 0}, p.tx, part, s);
  }
  if (want_w) {
    MmArgs m = {};
    m.k = a.N;
    m.a.ld = ldx;
    m.a.n = up8(a.d);
    m.b.ld = ldd;
    m.b.n = ff8;
    m.b.batch = static_cast<const char *>(du) - static_cast<const char *>(dg);
    set_segs(m, dt, 1, {x}, a.N * up8(a.d), {dg}, a.N * ff8);
    if (a.gdt == 0)
      run_mm<false, float>(m, out_of<float>(a), p.tw, part, s);
    else
      run_mm<false, bf16_t>(m, out_of<bf16_t>(a), p.tw, part, s);
  }
  return hipGetLastError();
}

// What may be read in place where every matrix starts on 16 bytes.
struct Places {
  bool x, w, g;
};
Places places_of(int dt, const FfArgs &a, bool pointers) {
  const auto p = [&](const void *q) { return pointers ? q : nullptr; };
  return {direct(dt, p(a.X), a.d, a.ldx),
          direct(dt, p(a.Wg), a.ff, a.ldw) && direct(dt, p(a.Wu), a.ff, a.ldw), false};
}
Places places_of(int dt, const FfGradArgs &a, bool pointers) {
  const auto p = [&](const void *q) { return pointers ? q : nullptr; };
  return {direct(dt, p(a.X), a.d, a.ldx),
          direct(dt, p(a.Wg), a.ff, a.ldw) && direct(dt, p(a.Wu), a.ff, a.ldw),
          direct(dt, p(a.dG), a.ff, a.ldd) && direct(dt, p(a.dU), a.ff, a.ldd)};
}
FfPlan plan_of(int dt, const FfArgs &a, const Places &own) {
  return ff_plan(dt, a.N, a.d, a.ff, own.x, own.w);
}
FfGradPlan plan_of(int dt, const FfGradArgs &a, const Places &own) {
  return ff_grad_plan(dt, a.N, a.d, a.ff, own.x, own.w, own.g);
}
// The bytes of a call whose matrices all start on 16 bytes, or of whichever starts take most.
template <typename A>
size_t most_bytes(int dt, const A &a, bool aligned) {
  const Places best = places_of(dt, a, false);
  size_t most = plan_of(dt, a, best).total;
  for (int m = 0; m < 7 && !aligned; ++m) {
    const size_t n =
        plan_of(dt, a, Places{best.x && (m & 1), best.w && (m & 2), best.g && (m & 4)}).total;
    most = n > most ? n : most;
  }
  return most;
}

}  // namespace

size_t ff_workspace_bytes(int dt, const FfArgs &a, bool aligned) { return most_bytes(dt, a, aligned); }
size_t ff_grad_workspace_bytes(int dt, const FfGradArgs &a, bool aligned) {
  return most_bytes(dt, a, aligned);
}
size_t ff_call_bytes(int dt, const FfArgs &a) { return plan_of(dt, a, places_of(dt, a, true)).total; }
size_t ff_grad_call_bytes(int dt, const FfGradArgs &a) {
  return plan_of(dt, a, places_of(dt, a, true)).total;
}

hipError_t launch_ff(int dt, const FfArgs &a, void *ws, hipStream_t s) {
  const FfPlan p = plan_of(dt, a, places_of(dt, a, true));
  return dt == 0 ? launch_ff_t<float>(dt, a, p, static_cast<char *>(ws), s)
                 : launch_ff_t<bf16_t>(dt, a, p, static_cast<char *>(ws), s);
}
hipError_t launch_ff_grad(int dt, const FfGradArgs &a, void *ws, hipStream_t s) {
  if (a.N == 0) {  // sums of nothing
    const dim3 grid = pieces_grid(2 * a.d, ceil_div(a.ff, 4));
    if (a.gdt == 0)
      ff_zero_kernel<<<grid, 256, 0, s>>>(out_of<float>(a));
    else
      ff_zero_kernel<<<grid, 256, 0, s>>>(out_of<bf16_t>(a));
    return hipGetLastError();
  }
  const FfGradPlan p = plan_of(dt, a, places_of(dt, a, true));
  return dt == 0 ? launch_ff_grad_t<float>(dt, a, p, static_cast<char *>(ws), s)
                 : launch_ff_grad_t<bf16_t>(dt, a, p, static_cast<char *>(ws), s);
}

}  // namespace sn
