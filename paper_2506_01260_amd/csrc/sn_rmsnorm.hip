// Root-mean-square norm with the residual's addition, N x d:
//   h = x + r,   y = h w / sqrt(mean h^2 + eps)
// h is rounded to dt where it is stored; y is made from the 32-bit sum.  The
// 8-bit form writes q = y / s in e4m3 (largest value 448) with one float32 scale
// s = max |y| / 448 for a row or for each 128 columns of it.  Backward, from the
// stored h, u = dy w and rho = 1 / sqrt(mean h^2 + eps):
//   dx = rho u - h rho^3 mean(u h) + dh,    gw += sum over rows of dy h rho,
// computed as rho (u - n (rho mean(u h))) + dh with n = h rho: rho^3 leaves
// float32's range where rows are of 2^-43 or 2^50.
//
// Memory-bound: each operand passes once, the row staying in registers between
// its sums and its outputs.  R threads hold a row in K pieces each; with R = 64
// a wave has a row of its own and no barrier.
//
// Measured: 32768 x 4096 bf16 with residual 181 us (5.9 TB/s read and written, the
// rate of an addition of two arrays on this card), 8 bits out 158-162 us; one row 2.7 us;
// backward of 16383 x 8192 with the stream's gradient 207 us (5.2 TB/s), 5 of them the
// gain's sum over workgroups.
#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

constexpr float kF8Max = 448.0f;
constexpr uint32_t kTiny = 0x0D800000u;  // 2^-100, the least maximum a scale is made from

// The piece at column c0 of a row of d, 0 past the row's end, in two steps: take()
// loads the piece there, or the one that the row ends with, and fix() moves that
// one's values to their places.  So every load of a row is issued before any is
// waited for, also at widths that are no multiple of the piece (where the last
// piece element by element, or moved as it came, made the backward of 32768 x 1601
// half as long again).  d >= E.  WHOLE: d is a multiple of the piece.
template <typename T>
__device__ __forceinline__ u32x4 take(const T *row, int c0, int d) {
  return load_piece(row + min(c0, d - Piece<T>::E));
}
template <typename T, bool WHOLE>
__device__ __forceinline__ u32x4 fix(u32x4 v, int c0, int d) {
  const int by = c0 - (d - Piece<T>::E);  // values that the piece came early by
  if (by > 0) {
    uint64_t lo = v.x | static_cast<uint64_t>(v.y) << 32, hi = v.z | static_cast<uint64_t>(v.w) << 32;
    const int bits = by * 8 * static_cast<int>(sizeof(T));
    if (WHOLE || bits >= 128) {
      lo = hi = 0;
    } else if (bits >= 64) {
      lo = hi >> (bits - 64);
      hi = 0;
    } else {
      lo = lo >> bits | hi << (64 - bits);
      hi >>= bits;
    }
    v = u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32),
              static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
  }
  return v;
}
// The same in one step, for any d and for rows past the registers.
template <typename T>
__device__ __forceinline__ void get(const T *row, int64_t c0, int64_t d, float (&x)[Piece<T>::E]) {
  if (c0 + Piece<T>::E <= d)
    Piece<T>::unpack(load_piece(row + c0), x);
  else
    load_part(row, c0, d, 0.0f, x);
}
template <typename T, bool WHOLE = false>
__device__ __forceinline__ void put(T *row, int64_t c0, int64_t d, const float (&x)[Piece<T>::E]) {
  if (WHOLE ? c0 < d : c0 + Piece<T>::E <= d)
    store_piece(row + c0, Piece<T>::pack(x));
  else if (!WHOLE)
    store_part(row, c0, d, x);
}

__device__ __forceinline__ uint32_t f8x4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true));
}

// E values of a row in 8 bits
template <int E, bool WHOLE = false>
__device__ __forceinline__ void put8(uint8_t *row, int64_t c0, int64_t d, const float (&q)[E]) {
  uint32_t w[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) w[i] = f8x4(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
  if (WHOLE ? c0 < d : c0 + E <= d) {
    __builtin_memcpy(row + c0, w, E);
  } else if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (c0 + i < d) row[c0 + i] = static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
  }
}

// largest |y| as its bits: as whole numbers they are ordered, a NaN above all
__device__ __forceinline__ uint32_t abs_bits(float y) { return __float_as_uint(y) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int LANES>
__device__ __forceinline__ uint32_t lanes_umax(uint32_t v) {
#pragma unroll
  for (int m = LANES / 2; m; m >>= 1) v = umax(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), m)));
  return v;
}
__device__ __forceinline__ float scale_of(uint32_t bits) {
  return __uint_as_float(umax(bits, kTiny)) / kF8Max;
}
// y / s of one scale, rounded to float32 as a division rounds it, within e4m3's range (a
// NaN stays one).  The product with the rounded reciprocal alone is up to 1.5 units off
// and gives the other code where y / s lies on a boundary between two, as rows of bf16
// put it; the product's remainder corrects it (equal to the division for every
// scale's 2^23 mantissas and the values about every boundary; 4999 x 1600 bf16 13.9 us,
// 13.4 with the product alone, 32768 x 4096 158 with both).  A zero's sign is kept.
struct Quotient {
  float s, inv;
  __device__ __forceinline__ explicit Quotient(float scale) : s(scale), inv(1.0f / scale) {
    // an infinite scale: 0 for what is finite, without inf * 0 in the remainder
    if (s == INFINITY) s = 0.0f;
  }
  __device__ __forceinline__ float operator()(float y) const {
    const float q0 = y * inv, q = fmaf(-fmaf(q0, s, -y), inv, q0);
    return q > kF8Max ? kF8Max : q < -kF8Max ? -kF8Max : q;
  }
};

enum { kOut = 0, kOut8Row = 1, kOut8Group = 2 };
constexpr int kGroup = 128;  // columns of a scale in the grouped form

// R threads per row, NT / R rows in a workgroup at a time.  The row's number is
// the same for a whole wave, so that the rows' addresses are scalars.
template <typename T, int R, int K, int NT, int OUT, bool WHOLE>
__global__ __launch_bounds__(NT) void rmsnorm_kernel(NormArgs a) {
  constexpr int E = Piece<T>::E, W = R / 64, ROWS = NT / R;
  static_assert(ROWS == 1 || W == 1, "a row of several waves has the workgroup to itself");
  __shared__ float red[W];
  __shared__ uint32_t redu[W];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / R);
  const int c = static_cast<int>(threadIdx.x % R) * E, d = static_cast<int>(a.d);
  const T *w = static_cast<const T *>(a.w);
  const int64_t i = group_number() * ROWS + sub;
  if (i >= a.N) return;
  const T *X = static_cast<const T *>(a.X) + i * a.ldx;
  u32x4 in[K], more[K];
#pragma unroll
  for (int k = 0; k < K; ++k) in[k] = take(X, c + k * R * E, d);
  if (a.R) {
    const T *Rs = static_cast<const T *>(a.R) + i * a.ldr;
#pragma unroll
    for (int k = 0; k < K; ++k) more[k] = take(Rs, c + k * R * E, d);
  }
  float h[K][E], ss = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    Piece<T>::unpack(fix<T, WHOLE>(in[k], c + k * R * E, d), h[k]);
    if (a.R) {
      float r[E];
      Piece<T>::unpack(fix<T, WHOLE>(more[k], c + k * R * E, d), r);
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] += r[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(h[k][e], h[k][e], ss);
  }
  ss = group_sum<W>(ss, red);
  if (a.H) {
    T *H = static_cast<T *>(a.H) + i * a.ldh;
#pragma unroll
    for (int k = 0; k < K; ++k) put<T, WHOLE>(H, c + k * R * E, d, h[k]);
  }
  const float rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
  uint32_t big[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c0 = c + k * R * E;
#pragma unroll
    for (int e = 0; e < E; ++e) h[k][e] *= rho;
    if (w) {
      float g[E];
      Piece<T>::unpack(fix<T, WHOLE>(take(w, c0, d), c0, d), g);
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] *= g[e];
    }
    if constexpr (OUT == kOut) {
      put<T, WHOLE>(static_cast<T *>(a.Y) + i * a.ldy, c0, d, h[k]);
    } else {
      big[k] = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) big[k] = umax(big[k], abs_bits(h[k][e]));
    }
  }
  if constexpr (OUT == kOut8Row) {
    uint32_t m = big[0];
#pragma unroll
    for (int k = 1; k < K; ++k) m = umax(m, big[k]);
    m = wave_umax(m);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) redu[threadIdx.x >> 6] = m;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < W; ++j) m = umax(m, redu[j]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) big[k] = m;
    if (c == 0) a.S[i * a.lds] = scale_of(m);
  } else if constexpr (OUT == kOut8Group) {
    constexpr int L = kGroup / E;  // lanes of a scale
#pragma unroll
    for (int k = 0; k < K; ++k) {
      big[k] = lanes_umax<L>(big[k]);
      const int c0 = c + k * R * E;
      if (c0 % kGroup == 0 && c0 < d) a.S[i * a.lds + c0 / kGroup] = scale_of(big[k]);
    }
  }
  if constexpr (OUT != kOut) {
    uint8_t *Q = static_cast<uint8_t *>(a.Y) + i * a.ldy;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Quotient over(scale_of(big[k]));
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] = over(h[k][e]);
      put8<E, WHOLE>(Q, c + k * R * E, d, h[k]);
    }
  }
}

// Rows longer than the registers hold: two or three passes over them.
template <typename T, int OUT>
__global__ __launch_bounds__(1024) void rmsnorm_long_kernel(NormArgs a) {
  constexpr int E = Piece<T>::E, NT = 1024, W = NT / 64;
  __shared__ float red[W];
  __shared__ uint32_t redu[W];
  const T *w = static_cast<const T *>(a.w);
  const int64_t i = group_number();
  if (i >= a.N) return;
  const T *X = static_cast<const T *>(a.X) + i * a.ldx;
  const T *Rs = a.R ? static_cast<const T *>(a.R) + i * a.ldr : nullptr;
  float h[E], r[E], ss = 0.0f;
  auto sum = [&](int64_t c0) {
    get(X, c0, a.d, h);
    if (Rs) {
      get(Rs, c0, a.d, r);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] += r[e];
    }
  };
  for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
    sum(c0);
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(h[e], h[e], ss);
  }
  ss = group_sum<W>(ss, red);
  const float rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
  auto norm = [&](int64_t c0) {
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] *= rho;
    if (w) {
      get(w, c0, a.d, r);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] *= r[e];
    }
  };
  uint32_t m = 0;
  if constexpr (OUT == kOut8Row) {
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      sum(c0);
      norm(c0);
#pragma unroll
      for (int e = 0; e < E; ++e) m = umax(m, abs_bits(h[e]));
    }
    m = wave_umax(m);
    if ((threadIdx.x & 63) == 0) redu[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < W; ++j) m = umax(m, redu[j]);
    if (threadIdx.x == 0) a.S[i * a.lds] = scale_of(m);
  }
  // whole waves stay in the loop, so that the lanes of a scale are all there
  for (int64_t b = 0; b < a.d; b += NT * E) {
    const int64_t c0 = b + threadIdx.x * E;
    sum(c0);
    if (a.H) put(static_cast<T *>(a.H) + i * a.ldh, c0, a.d, h);
    norm(c0);
    if constexpr (OUT == kOut) {
      put(static_cast<T *>(a.Y) + i * a.ldy, c0, a.d, h);
    } else {
      if constexpr (OUT == kOut8Group) {
        constexpr int L = kGroup / E;
        m = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) m = umax(m, abs_bits(h[e]));
        m = lanes_umax<L>(m);
        if (threadIdx.x % L == 0 && c0 < a.d) a.S[i * a.lds + c0 / kGroup] = scale_of(m);
      }
      const Quotient over(scale_of(m));
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = over(h[e]);
      put8<E>(static_cast<uint8_t *>(a.Y) + i * a.ldy, c0, a.d, h);
    }
  }
}

// Backward.  A workgroup takes the rows blockIdx.x, + gridDim.x, ... and keeps its
// part of the gain's gradient in registers; the parts are summed by gain_kernel.
// Everything of a row is loaded before its sums are joined, and stays as loaded
// (16 bytes a piece) until it is used: at d = 8192 bf16 registers for two
// workgroups of 8 waves on a CU instead of one.  Ragged bf16 rows of 12289 to 16383
// columns need more registers than 1024 threads have: 36 bytes of scratch.
template <typename T, int R, int K, int NT, bool WHOLE>
__global__ __launch_bounds__(NT) void rmsnorm_grad_kernel(NormGradArgs a) {
  constexpr int E = Piece<T>::E, W = R / 64, ROWS = NT / R;
  static_assert(ROWS == 1 || W == 1, "a row of several waves has the workgroup to itself");
  __shared__ float red[2][W];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / R);
  const int c = static_cast<int>(threadIdx.x % R) * E, d = static_cast<int>(a.d);
  const T *w = static_cast<const T *>(a.w);
  float gw[K][E] = {};
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * ROWS + sub; i < a.N;
       i += static_cast<int64_t>(gridDim.x) * ROWS) {
    const T *H = static_cast<const T *>(a.H) + i * a.ldh;
    const T *dY = static_cast<const T *>(a.dY) + i * a.lddy;
    u32x4 hp[K], yp[K], dp[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      hp[k] = take(H, c + k * R * E, d);
      yp[k] = take(dY, c + k * R * E, d);
    }
    if (a.dH) {
      const T *dH = static_cast<const T *>(a.dH) + i * a.lddh;
#pragma unroll
      for (int k = 0; k < K; ++k) dp[k] = take(dH, c + k * R * E, d);
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) dp[k] = u32x4{0, 0, 0, 0};
    }
    float h[E], y[E], g[E], ss = 0.0f, uh = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = 1.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = c + k * R * E;
      hp[k] = fix<T, WHOLE>(hp[k], c0, d);
      yp[k] = fix<T, WHOLE>(yp[k], c0, d);
      Piece<T>::unpack(hp[k], h);
      Piece<T>::unpack(yp[k], y);
      if (w) Piece<T>::unpack(fix<T, WHOLE>(take(w, c0, d), c0, d), g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ss = fmaf(h[e], h[e], ss);
        uh = fmaf(y[e] * g[e], h[e], uh);
      }
    }
    ss = group_sum<W>(ss, red[0]);
    uh = group_sum<W>(uh, red[1]);
    const float rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
    const float f = uh * a.inv_d * rho;
    T *dX = static_cast<T *>(a.dX) + i * a.lddx;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = c + k * R * E;
      float o[E];
      Piece<T>::unpack(hp[k], h);
      Piece<T>::unpack(yp[k], y);
      Piece<T>::unpack(fix<T, WHOLE>(dp[k], c0, d), o);
      if (w) Piece<T>::unpack(fix<T, WHOLE>(take(w, c0, d), c0, d), g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float n = h[e] * rho;
        gw[k][e] = fmaf(y[e], n, gw[k][e]);
        o[e] = fmaf(rho, fmaf(-n, f, y[e] * g[e]), o[e]);
      }
      put<T, WHOLE>(dX, c0, d, o);
    }
    if constexpr (W > 1) {
      if (i + gridDim.x < a.N) __syncthreads();  // the LDS is used again
    }
  }
  if (!a.part) return;
  float *part = a.part + static_cast<int64_t>(blockIdx.x) * a.d;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = c + k * R * E;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c0 + e < d) part[c0 + e] = gw[k][e];
    }
  } else {  // the waves' rows are added in order
    __shared__ float sums[ROWS][K * R * E];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) sums[sub][c + k * R * E + e] = gw[k][e];
    __syncthreads();
    for (int j = threadIdx.x; j < d; j += NT) {
      float t = sums[0][j];
#pragma unroll
      for (int q = 1; q < ROWS; ++q) t += sums[q][j];
      part[j] = t;
    }
  }
}

// Rows longer than the registers hold: the part of the gain's gradient is kept
// in the workspace between the workgroup's rows.
template <typename T>
__global__ __launch_bounds__(1024) void rmsnorm_grad_long_kernel(NormGradArgs a) {
  constexpr int E = Piece<T>::E, NT = 1024, W = NT / 64;
  __shared__ float red[2][W];
  const T *w = static_cast<const T *>(a.w);
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const T *H = static_cast<const T *>(a.H) + i * a.ldh;
    const T *dY = static_cast<const T *>(a.dY) + i * a.lddy;
    const T *dH = a.dH ? static_cast<const T *>(a.dH) + i * a.lddh : nullptr;
    float h[E], u[E], g[E], ss = 0.0f, uh = 0.0f;
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      get(H, c0, a.d, h);
      get(dY, c0, a.d, u);
      if (w) get(w, c0, a.d, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        ss = fmaf(h[e], h[e], ss);
        uh = fmaf(w ? u[e] * g[e] : u[e], h[e], uh);
      }
    }
    ss = group_sum<W>(ss, red[0]);
    uh = group_sum<W>(uh, red[1]);
    const float rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
    const float f = uh * a.inv_d * rho;
    float *part = a.part ? a.part + static_cast<int64_t>(blockIdx.x) * a.d : nullptr;
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      float o[E] = {};
      get(H, c0, a.d, h);
      get(dY, c0, a.d, u);
      if (dH) get(dH, c0, a.d, o);
      if (w) get(w, c0, a.d, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float n = h[e] * rho;
        if (part && c0 + e < a.d)
          part[c0 + e] = fmaf(u[e], n, i == blockIdx.x ? 0.0f : part[c0 + e]);
        o[e] = fmaf(rho, fmaf(-n, f, w ? u[e] * g[e] : u[e]), o[e]);
      }
      put(static_cast<T *>(a.dX) + i * a.lddx, c0, a.d, o);
    }
    if (i + gridDim.x < a.N) __syncthreads();  // the LDS is used again
  }
}

// gw[c] += sum over the parts, in float64 and in a fixed order: 32 groups of threads
// take every 32nd part of 32 columns, then the groups in order.
constexpr int kGainCols = 32, kGainGroups = 32;
__global__ __launch_bounds__(kGainCols *kGainGroups) void gain_kernel(
    const float *__restrict__ part, int64_t parts, int64_t d, float *__restrict__ gw) {
  __shared__ double red[kGainGroups][kGainCols];
  const int lane = threadIdx.x % kGainCols, g = threadIdx.x / kGainCols;
  const int64_t c0 = group_number() * kGainCols, c = c0 + lane;
  if (c0 >= d) return;
  double s = 0.0;
  if (c < d) {
#pragma unroll 8
    for (int64_t b = g; b < parts; b += kGainGroups) s += static_cast<double>(part[b * d + c]);
  }
  red[g][lane] = s;
  __syncthreads();
  if (g != 0 || c >= d) return;
#pragma unroll
  for (int i = 1; i < kGainGroups; ++i) s += red[i][lane];
  gw[c] = static_cast<float>(static_cast<double>(gw[c]) + s);
}

// pieces of a row; R * K of them are held by R threads in K pieces each
int64_t pieces_of(int dt, int64_t d) { return ceil_div(d, dt == 0 ? 4 : 8); }

// Threads and pieces of each: three pieces where two or four would leave a third of
// the threads idle (8 bits from 20184 x 5632 float32 151 us with 1024 threads, 129
// with four pieces of 512, 119 with three; backward of 8192 x 12288 bf16 183, 167).
template <typename T, int OUT, bool WHOLE>
hipError_t launch_norm_t(const NormArgs &a, hipStream_t s) {
  const int64_t n = ceil_div(a.d, Piece<T>::E);
  const auto grid = [&](int rows) { return groups_grid(ceil_div(a.N, rows)); };
  if (a.d < Piece<T>::E)  // no whole piece to take
    rmsnorm_long_kernel<T, OUT><<<grid(1), 1024, 0, s>>>(a);
  else if (n <= 64)
    rmsnorm_kernel<T, 64, 1, 256, OUT, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 128)
    rmsnorm_kernel<T, 64, 2, 256, OUT, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 256)
    rmsnorm_kernel<T, 64, 4, 256, OUT, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 512)
    rmsnorm_kernel<T, 256, 2, 256, OUT, WHOLE><<<grid(1), 256, 0, s>>>(a);
  else if (n <= 768)
    rmsnorm_kernel<T, 256, 3, 256, OUT, WHOLE><<<grid(1), 256, 0, s>>>(a);
  else if (n <= 1024)
    rmsnorm_kernel<T, 512, 2, 512, OUT, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else if (n <= 1536)
    rmsnorm_kernel<T, 512, 3, 512, OUT, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else if (n <= 2048)
    rmsnorm_kernel<T, 512, 4, 512, OUT, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else
    rmsnorm_long_kernel<T, OUT><<<grid(1), 1024, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_out(const NormArgs &a, hipStream_t s) {
  if (a.d % Piece<T>::E == 0) {
    if (!a.S) return launch_norm_t<T, kOut, true>(a, s);
    return a.group ? launch_norm_t<T, kOut8Group, true>(a, s)
                   : launch_norm_t<T, kOut8Row, true>(a, s);
  }
  if (!a.S) return launch_norm_t<T, kOut, false>(a, s);
  return a.group ? launch_norm_t<T, kOut8Group, false>(a, s)
                 : launch_norm_t<T, kOut8Row, false>(a, s);
}

// Workgroups of the backward, each with a part of the gain's gradient: what the
// kernels' registers let run at a time, or what the rows fill.  Up to 256 pieces a
// wave has a row of its own and nothing waits at a barrier (32768 x 2048 bf16: 106
// us, 112 with a workgroup to a row; x 1601: 110, 127).  Few rows are not worth more
// parts than two to a CU (1200 x 4096: 18 us with 512, 24 with 1024), many are where
// registers allow them (16384 x 5120: 145 with 768, 153 with 512).
int64_t grad_groups(int dt, int64_t N, int64_t d) {
  const int64_t n = pieces_of(dt, d);
  int64_t most = 512;
  if (n <= 128 && N > 8192) most = 1024;
  if (n > 256 && n <= 512 && N > 4096) most = 1024;
  if (n > 512 && n <= 768 && N > 4096) most = 768;
  const int64_t groups = ceil_div(N, n <= 256 ? 4 : 1);
  return groups < most ? groups : most;
}
// An odd number where every other row starts at an odd bf16 element: those rows take
// longer, and a workgroup should have as many of them as any other (14096 x 3735: 107
// us, 122 with an even number).
int64_t turn_groups(int dt, const NormGradArgs &a) {
  const int64_t g = grad_groups(dt, a.N, a.d);
  const bool odd = dt != 0 && ((a.ldh | a.lddy | (a.dH ? a.lddh : 0) | a.lddx) & 1);
  return odd && pieces_of(dt, a.d) > 256 && a.N >= 8 * g ? g - 1 + g % 2 : g;
}

template <typename T, bool WHOLE>
hipError_t launch_grad_t(int dt, const NormGradArgs &a, hipStream_t s) {
  const int64_t n = ceil_div(a.d, Piece<T>::E);
  const unsigned g = static_cast<unsigned>(turn_groups(dt, a));
  if (a.d < Piece<T>::E)
    rmsnorm_grad_long_kernel<T><<<g, 1024, 0, s>>>(a);
  else if (n <= 64)
    rmsnorm_grad_kernel<T, 64, 1, 256, WHOLE><<<g, 256, 0, s>>>(a);
  else if (n <= 128)
    rmsnorm_grad_kernel<T, 64, 2, 256, WHOLE><<<g, 256, 0, s>>>(a);
  else if (n <= 256)
    rmsnorm_grad_kernel<T, 64, 4, 256, WHOLE><<<g, 256, 0, s>>>(a);
  else if (n <= 512)
    rmsnorm_grad_kernel<T, 256, 2, 256, WHOLE><<<g, 256, 0, s>>>(a);
  else if (n <= 768)
    rmsnorm_grad_kernel<T, 256, 3, 256, WHOLE><<<g, 256, 0, s>>>(a);
  else if (n <= 1024)
    rmsnorm_grad_kernel<T, 512, 2, 512, WHOLE><<<g, 512, 0, s>>>(a);
  else if (n <= 1536)
    rmsnorm_grad_kernel<T, 512, 3, 512, WHOLE><<<g, 512, 0, s>>>(a);
  else if (n <= 2048)
    rmsnorm_grad_kernel<T, 1024, 2, 1024, WHOLE><<<g, 1024, 0, s>>>(a);
  else
    rmsnorm_grad_long_kernel<T><<<g, 1024, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_grad_d(int dt, const NormGradArgs &a, hipStream_t s) {
  return a.d % Piece<T>::E == 0 ? launch_grad_t<T, true>(dt, a, s)
                                : launch_grad_t<T, false>(dt, a, s);
}

}  // namespace

hipError_t launch_rmsnorm(int dt, const NormArgs &a, hipStream_t s) {
  return dt == 0 ? launch_norm_out<float>(a, s) : launch_norm_out<bf16_t>(a, s);
}

size_t rmsnorm_grad_workspace_bytes(int dt, int64_t N, int64_t d) {
  return align256(static_cast<size_t>(grad_groups(dt, N, d)) * d * sizeof(float));
}

hipError_t launch_rmsnorm_grad(int dt, NormGradArgs a, float *gw, void *ws, hipStream_t s) {
  a.part = gw ? static_cast<float *>(ws) : nullptr;
  const hipError_t e = dt == 0 ? launch_grad_d<float>(dt, a, s) : launch_grad_d<bf16_t>(dt, a, s);
  if (e != hipSuccess || !gw) return e;
  gain_kernel<<<groups_grid(ceil_div(a.d, kGainCols)), kGainCols * kGainGroups, 0, s>>>(
      a.part, turn_groups(dt, a), a.d, gw);
  return hipGetLastError();
}

}  // namespace sn
