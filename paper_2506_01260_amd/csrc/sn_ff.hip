// The gated feed-forward block of N tokens:
//   G = X Wg,  U = X Wu,  H = act(G) * U              X: N x d, Wg, Wu: d x ff
// and its backward from the stored G and U,
//   dG = dH U act'(G),  dU = dH act(G),
//   dX = dG Wg^T + dU Wu^T,  gWg = X^T dG,  gWu = X^T dU.
//
// Forward: one kernel takes both products, a wave holding the same columns of G and U,
// and writes H from the 32-bit sums.  Backward: dG and dU are made once, elementwise, and
// rounded to dt, the operands' type of the three products that read them (dX as one
// product over 2 ff, both weights' gradients in one launch).
// float32 operands (forward: of more than 128 tokens) are split in three bf16 planes (24 bits
// together, hi + mid + lo) and the six products down to 2^-24 of the largest are added up: at the peak rates 2.6 times
// what the float32 matrix instructions do.  Matrices that are not 16-byte aligned, or
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
// exactly (8 bits each, signed), the second times 2^7 and the third times 2^14: at most a
// quarter of the first, so that their products do not overflow before it does, and no
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

// ---- forward of up to 128 float32 tokens: the weights as they are -----------------------------
// A workgroup takes 64 columns of both weights and a slice of d, 128 of its k at a time, whose
// part of the tokens lies in the LDS; a wave takes every eighth four of them.  In the float32 matrix
// instruction 16 x 16 x 4 lane l = 16 g + n supplies k = g of row n of either operand: a lane's 16 bytes
// of a weight's row are columns 4 n + e, so the products of its value e have rows n for columns
// 4 n + e, and the sums of all four are 16 neighbouring columns of the token n.
// Bound by the weights' reading up to 16 tokens (4096 x 14336 85 us, 5.5 TB/s), then by the
// instruction (64 tokens 178 us; its rate alone would take 96).
constexpr int kFourCols = 64, kFourWaves = 8, kFourK = 128;
template <int TT>  // tiles of 16 tokens
__global__ __launch_bounds__(kFourWaves * 64) void ff_four_kernel(FfArgs a, int slices) {
  constexpr int NT = kFourWaves * 64, TOK = 16 * TT, UN = kFourK / 4 / kFourWaves;
  // rows 16 banks apart: the four k that are read together lie in different ones
  constexpr int STRIDE = TT == 1 ? 16 : TOK + 16, XS = kFourK * STRIDE;
  constexpr int RED = 2 * kFourWaves * 16 * kFourCols;
  __shared__ __attribute__((aligned(16))) float lds[2 * XS > RED ? 2 * XS : RED];
  const int64_t strips = (a.ff + kFourCols - 1) / kFourCols, blocks = (a.N + TOK - 1) / TOK;
  const int64_t id = group_number(), part = id / blocks;
  if (part >= strips * slices) return;
  const int64_t slice = part / strips, strip = part - slice * strips, first = (id - part * blocks) * TOK;
  const int64_t k0 = slice * a.d / slices, len = (slice + 1) * a.d / slices - k0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
  const int64_t c = strip * kFourCols + 4 * n, cb = c < a.ff - 4 ? c : a.ff - 4;
  const float *wg = static_cast<const float *>(a.Wg) + k0 * a.ldw + cb;
  const int64_t twin = static_cast<const float *>(a.Wu) - static_cast<const float *>(a.Wg);
  const float *X = static_cast<const float *>(a.X) + first * a.ldx + k0;
  const int64_t tokens = a.N - first;
  // the tokens' share of a thread: four k of token t, TT times
  const int tt = threadIdx.x & 15, tk = threadIdx.x >> 4 << 2;
  f32x4 xr[TT], acc[2][TT][4];
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[q][t][e] = f32x4{0, 0, 0, 0};
  const auto fetch = [&](int64_t at) {
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      xr[t] = f32x4{0, 0, 0, 0};
      if (t * 16 + tt < tokens && at + tk < len) xr[t] = get4(X + (t * 16 + tt) * a.ldx + at + tk, len - at - tk);
    }
  };
  const auto store = [&](float *xs) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) xs[(tk + e) * STRIDE + t * 16 + tt] = xr[t][e];
  };
  u32x4 vg[UN], vu[UN];
  const auto weights = [&](int i, int64_t at) {  // rows past the slice: its last one, as zeros
    const int64_t k = at + (i * kFourWaves + wave) * 4 + g;
    const float *w = wg + (k < len ? k : len - 1) * a.ldw;
    const uint32_t keep = k < len ? ~0u : 0u;
    vg[i] = load_piece(w) & u32x4{keep, keep, keep, keep};
    vu[i] = load_piece(w + twin) & u32x4{keep, keep, keep, keep};
  };
  fetch(0);
#pragma unroll
  for (int i = 0; i < UN; ++i) weights(i, 0);
  store(lds);
  lds_barrier();
  int cur = 0;
#pragma unroll 1
  for (int64_t at = 0; at < len; at += kFourK) {
    const bool more = at + kFourK < len;
    if (more) fetch(at + kFourK);
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      float x[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t)
        x[t] = lds[cur + ((i * kFourWaves + wave) * 4 + g) * STRIDE + t * 16 + n];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          acc[0][t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vg[i][e]), x[t], acc[0][t][e], 0, 0, 0);
          acc[1][t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vu[i][e]), x[t], acc[1][t][e], 0, 0, 0);
        }
      weights(i, more ? at + kFourK : at);  // behind the last ones, these again: no branch parts the loads
    }
    cur ^= XS;
    if (more) store(lds + cur);
    lds_barrier();
  }
  // the waves' sums are added in order, tile by tile
#pragma unroll
  for (int t = 0; t < TT; ++t) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4 *>(lds + ((q * kFourWaves + wave) * 16 + n) * kFourCols + 16 * g + 4 * r) =
            f32x4{acc[q][t][0][r], acc[q][t][1][r], acc[q][t][2][r], acc[q][t][3][r]};
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * kFourCols; i += NT) {
      const int64_t token = first + t * 16 + i / kFourCols;
      const int j = i % kFourCols;
      const int64_t c1 = strip * kFourCols + j / 4 * 4;
      const int64_t col = (c1 < a.ff - 4 ? c1 : a.ff - 4) + j % 4;
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kFourWaves; ++w)
#pragma unroll
        for (int q = 0; q < 2; ++q) s[q] += lds[(q * kFourWaves + w) * 16 * kFourCols + i];
      if (token >= a.N || c1 >= a.ff) continue;
      if (slices > 1) {
        float *p = a.part + (slice * 2 * a.N + token) * a.ff + col;
        p[0] = s[0];
        p[a.N * a.ff] = s[1];
      } else {
        static_cast<float *>(a.H)[token * a.ldh + col] = ff_act(a.act, s[0]) * s[1];
        if (a.G) {
          static_cast<float *>(a.G)[token * a.ldg + col] = s[0];
          static_cast<float *>(a.U)[token * a.ldg + col] = s[1];
        }
      }
    }
    __syncthreads();
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

// float32 weights read as they are, or copied into planes first: 4096 x 14336 with 16 tokens 86
// and 515 us, 48 175 and 519, 100 340 and 515; 1024 x 4096 17, 23, 48 and 64, 66, 52; with more
// tokens the planes' products gain (4096 x 14336, 256 tokens: 672 and 550).
bool by_four(int dt, int64_t N, int64_t ff) { return dt == 0 && N <= 128 && ff >= 4; }
// Tiles of 16 tokens of a workgroup.  Where the columns are half the CUs' or more, so many that
// the weights pass once (2048 x 8192, 64 tokens: 61 us, 86 with a tile each); else one, the
// weights coming from the caches again (1600 x 4267, 48 tokens: 39 us, 69 with four).
int four_tiles(int64_t N, int64_t ff) {
  return N <= 16 || ceil_div(ff, kFourCols) < 128 ? 1 : N <= 32 ? 2 : 4;
}
// Slices of d: as many as give each CU a workgroup at most (4096 x 14336, one token: 85 us; in
// two slices, of which a CU holds two, 95), of a round of k or more, 16 at most.
int four_slices(int64_t N, int64_t d, int64_t ff) {
  const int64_t groups = ceil_div(ff, kFourCols) * ceil_div(N, 16 * four_tiles(N, ff));
  const int64_t fit = 256 / groups, most = ceil_div(d, kFourK);
  const int64_t n = fit < 1 ? 1 : fit < most ? fit : most;
  return static_cast<int>(n < 16 ? n : 16);
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
  bool vec, four, own_x, own_w;  // own: read in place
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
  } else if (by_four(dt, N, ff)) {
    p.four = true;
    p.slices = four_slices(N, d, ff);
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
void launch_four(const FfArgs &a, int slices, hipStream_t s) {
  const int tt = four_tiles(a.N, a.ff);
  const dim3 grid = groups_grid(ceil_div(a.ff, kFourCols) * slices * ceil_div(a.N, 16 * tt));
  if (tt == 1)
    ff_four_kernel<1><<<grid, kFourWaves * 64, 0, s>>>(a, slices);
  else if (tt == 2)
    ff_four_kernel<2><<<grid, kFourWaves * 64, 0, s>>>(a, slices);
  else
    ff_four_kernel<4><<<grid, kFourWaves * 64, 0, s>>>(a, slices);
  if (slices > 1)
    ff_join_kernel<float><<<pieces_grid(a.N, ceil_div(a.ff, 4)), 256, 0, s>>>(a, slices);
}

template <typename T>
hipError_t launch_ff_t(int dt, FfArgs a, const FfPlan &p, char *ws, hipStream_t s) {
  a.part = reinterpret_cast<float *>(ws + p.part);
  if (p.vec) {
    launch_vec(a, p.slices, s);
  } else if (p.four) {
    launch_four(a, p.slices, s);
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
  bool own_x, own_w, own_g;
  MmPlan tx, tw;
  size_t x, w, g, part, total;
};
FfGradPlan ff_grad_plan(int dt, int64_t N, int64_t d, int64_t ff, bool own_x, bool own_w, bool own_g) {
  FfGradPlan p = {};
  Space s;
  p.own_x = own_x;
  p.own_w = own_w;
  p.own_g = own_g;
  p.tx = mm_plan(N, d, 1, ceil_div(ff, kMmK) * 2 * segs_of(dt));
  p.tw = mm_plan(d, ff, 2, ceil_div(N, kMmK) * segs_of(dt));
  if (!own_x) p.x = s.take(2 * kPlanes[dt] * N * up8(d));
  if (!own_w) p.w = s.take(2 * 2 * kPlanes[dt] * d * up8(ff));
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
  if (!p.own_w && a.dX) {
    uint16_t *to = reinterpret_cast<uint16_t *>(ws + p.w), *to2 = to + planes * a.d * ff8;
    pack<T>(a.Wg, a.d, a.ff, a.ldw, to, s);
    pack<T>(a.Wu, a.d, a.ff, a.ldw, to2, s);
    wg = to;
    wu = to2;
    ldw = ff8;
  }
  float *part = reinterpret_cast<float *>(ws + p.part);
  if (a.dX) {
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
