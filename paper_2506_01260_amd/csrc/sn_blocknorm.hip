// The end of a block and the start of the next, N x d:
//   z = x w1 / sqrt(mean x^2 + eps)  (or z = x),   h = alpha r + g z,
//   y = h w / sqrt(mean h^2 + eps)
// with a gate g (or its sigmoid) of one row or of each token.  h is rounded to dt where it
// is stored; y is made from the 32-bit sum.  Backward, from x and the stored h, with
// n = h rho, u = dy w, q = 1 / sqrt(mean x^2 + eps), m = x q:
//   dh = rho (u - n mean(u n)) + dH,   dR = alpha dh,   dg = dh z g',
//   v = g dh w1,   dX = q (v - m mean(v m))      (dX = g dh without the post norm)
//   gw += sum dy n,   gw_post += sum g dh m,   one gate row's gradient += sum dg.
//
// Memory-bound: each operand passes once, the row staying in registers between its two
// (backward: two joint) sums and its outputs.  R threads hold a row in K pieces each; with
// R = 64 a wave has a row of its own and no barrier.
// bf16 with one gate row: 32768 x 4096 190 us, 5.7 TB/s (add of two arrays: 6.2); backward
// 16383 x 8192 308 us, 5.2 TB/s; with a gate and its gradient for each token 4999 x 1600 37 us,
// of it 4 the second launch that joins the column sums; one token 3.5 us in the kernel.
#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

// A sigmoid and its derivative from t = e^-|g|: 1 / (1 + t), or t / (1 + t) for g < 0, and t / (1 + t)^2,
// so that neither is left over from a difference (g (1 - g) is off by 3e-4 of itself at 9, by all of
// it at 17).  For bf16 t and 1 / (1 + t) are the hardware's, an ulp off; the exponent's rounding, |g| 2^-24
// of t, is made up for.  (Backward of 4999 x 1600 with a gate a token: 36.7 us; with expf and
// a division 49.)
template <typename T>
__device__ __forceinline__ float sigmoid_of(float g, float *slope = nullptr) {
  // past 104 t is 0 in float32; a NaN stays one
  const float a = fabsf(g) > 128.0f ? 128.0f : fabsf(g);
  float t, p;
  if constexpr (sizeof(T) == 2) {
    const float x = -1.4426950f * a, rest = fmaf(-1.925963e-8f, a, fmaf(-1.4426950f, a, -x));
    t = __builtin_amdgcn_exp2f(x);
    t = fmaf(t, 0.69314718f * rest, t);
    p = __builtin_amdgcn_rcpf(1.0f + t);
  } else {
    t = expf(-a);
    p = 1.0f / (1.0f + t);
  }
  if (slope) *slope = t * p * p;
  return g < 0.0f ? t * p : p;
}

// The gate's row of token i.
template <typename T, typename A>
__device__ __forceinline__ const T *gate_row(const A &a, int64_t i) {
  return static_cast<const T *>(a.gate) + i * a.ldgate;
}

// NS sums over a workgroup of W waves in one barrier; red: W * NS floats, free as group_sum's.
// The waves' sums are joined by lanes, not by each thread in turn, which took W * NS registers.
template <int W, int NS>
__device__ __forceinline__ void group_sums(float (&v)[NS], float (*red)[W]) {
#pragma unroll
  for (int s = 0; s < NS; ++s) v[s] = wave_sum(v[s]);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int s = 0; s < NS; ++s) red[s][threadIdx.x >> 6] = v[s];
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int lane = threadIdx.x & 63;
      v[s] = wave_sum(lane < W ? red[s][lane] : 0.0f);
    }
  }
}

// R threads per row, NT / R rows in a workgroup.
template <typename T, int R, int K, int NT, bool WHOLE>
__global__ __launch_bounds__(NT) void block_norm_kernel(BlockNormArgs a) {
  constexpr int E = Piece<T>::E, W = R / 64, ROWS = NT / R;
  static_assert(ROWS == 1 || W == 1, "a row of several waves has the workgroup to itself");
  __shared__ float red[2][W];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / R);
  const int c = static_cast<int>(threadIdx.x % R) * E, d = static_cast<int>(a.d);
  const int64_t i = group_number() * ROWS + sub;
  if (i >= a.N) return;
  const T *X = static_cast<const T *>(a.X) + i * a.ldx;
  const T *Rs = static_cast<const T *>(a.R) + i * a.ldr;
  const T *w = static_cast<const T *>(a.w), *w1 = static_cast<const T *>(a.w_post);
  u32x4 xp[K], rp[K], gp[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    xp[k] = take(X, c + k * R * E, d);
    rp[k] = take(Rs, c + k * R * E, d);
  }
  if (a.gate) {
    const T *G = gate_row<T>(a, i);
#pragma unroll
    for (int k = 0; k < K; ++k) gp[k] = take(G, c + k * R * E, d);
  }
  float h[K][E], sx = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    Piece<T>::unpack(fix<T, WHOLE>(xp[k], c + k * R * E, d), h[k]);
#pragma unroll
    for (int e = 0; e < E; ++e) sx = fmaf(h[k][e], h[k][e], sx);
  }
  float q = 1.0f;
  if (a.post) {
    sx = group_sum<W>(sx, red[0]);
    q = 1.0f / sqrtf(sx * a.inv_d + a.eps);
  }
  float ss = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c0 = c + k * R * E;
    float t[E];
    if (a.post) {
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] *= q;
      if (w1) {
        Piece<T>::unpack(fix<T, WHOLE>(take(w1, c0, d), c0, d), t);
#pragma unroll
        for (int e = 0; e < E; ++e) h[k][e] *= t[e];
      }
    }
    if (a.gate) {
      Piece<T>::unpack(fix<T, WHOLE>(gp[k], c0, d), t);
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] *= a.sigmoid ? sigmoid_of<T>(t[e]) : t[e];
    }
    Piece<T>::unpack(fix<T, WHOLE>(rp[k], c0, d), t);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      h[k][e] = fmaf(a.alpha, t[e], h[k][e]);
      ss = fmaf(h[k][e], h[k][e], ss);
    }
  }
  // H may lie on X or R, whose last piece other threads load too: past a barrier
  ss = group_sum<W>(ss, red[1]);
  T *H = static_cast<T *>(a.H) + i * a.ldh;
#pragma unroll
  for (int k = 0; k < K; ++k) put<T, WHOLE>(H, c + k * R * E, d, h[k]);
  if (!a.Y) return;
  const float rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
  T *Y = static_cast<T *>(a.Y) + i * a.ldy;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c0 = c + k * R * E;
#pragma unroll
    for (int e = 0; e < E; ++e) h[k][e] *= rho;
    if (w) {
      float t[E];
      Piece<T>::unpack(fix<T, WHOLE>(take(w, c0, d), c0, d), t);
#pragma unroll
      for (int e = 0; e < E; ++e) h[k][e] *= t[e];
    }
    put<T, WHOLE>(Y, c0, d, h[k]);
  }
}

// Rows longer than the registers hold, or shorter than a piece: up to three passes.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_long_kernel(BlockNormArgs a) {
  constexpr int E = Piece<T>::E, NT = 1024, W = NT / 64;
  __shared__ float red[2][W];
  const int64_t i = group_number();
  if (i >= a.N) return;
  const T *X = static_cast<const T *>(a.X) + i * a.ldx;
  const T *Rs = static_cast<const T *>(a.R) + i * a.ldr;
  const T *w = static_cast<const T *>(a.w), *w1 = static_cast<const T *>(a.w_post);
  float h[E], t[E], q = 1.0f;
  if (a.post) {
    float sx = 0.0f;
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      get(X, c0, a.d, h);
#pragma unroll
      for (int e = 0; e < E; ++e) sx = fmaf(h[e], h[e], sx);
    }
    sx = group_sum<W>(sx, red[0]);
    q = 1.0f / sqrtf(sx * a.inv_d + a.eps);
  }
  const auto sum = [&](int64_t c0) {
    get(X, c0, a.d, h);
    if (a.post) {
      if (w1) get(w1, c0, a.d, t);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = w1 ? h[e] * q * t[e] : h[e] * q;
    }
    if (a.gate) {
      get(gate_row<T>(a, i), c0, a.d, t);
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] *= a.sigmoid ? sigmoid_of<T>(t[e]) : t[e];
    }
    get(Rs, c0, a.d, t);
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = fmaf(a.alpha, t[e], h[e]);
  };
  float rho = 1.0f;
  if (a.Y) {
    float ss = 0.0f;
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      sum(c0);
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(h[e], h[e], ss);
    }
    ss = group_sum<W>(ss, red[1]);
    rho = 1.0f / sqrtf(ss * a.inv_d + a.eps);
  }
  // H may lie on X or R: each thread has read what it writes over
  for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
    sum(c0);
    put(static_cast<T *>(a.H) + i * a.ldh, c0, a.d, h);
    if (!a.Y) continue;
    if (w) get(w, c0, a.d, t);
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = w ? h[e] * rho * t[e] : h[e] * rho;
    put(static_cast<T *>(a.Y) + i * a.ldy, c0, a.d, h);
  }
}

// Backward.  A workgroup takes the rows blockIdx.x, + gridDim.x, ... and keeps its parts of
// the three column sums in registers; block_sum_kernel adds the parts.
enum { kGw = 0, kGwPost = 1, kGate = 2 };

// Two neighbouring values of a piece, and a piece made of such pairs.
template <typename T>
__device__ __forceinline__ void pair_of(u32x4 v, int q, float &a, float &b) {
  if constexpr (sizeof(T) == 2) {
    a = bf_lo(v[q]);
    b = bf_hi(v[q]);
  } else {
    a = __uint_as_float(v[2 * q]);
    b = __uint_as_float(v[2 * q + 1]);
  }
}
template <typename T>
__device__ __forceinline__ void set_pair(u32x4 &v, int q, float a, float b) {
  if constexpr (sizeof(T) == 2) {
    v[q] = pack_bf16x2(a, b);
  } else {
    v[2 * q] = __float_as_uint(a);
    v[2 * q + 1] = __float_as_uint(b);
  }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void put_piece(T *row, int c0, int d, u32x4 v) {
  if (WHOLE ? c0 < d : c0 + Piece<T>::E <= d) {
    store_piece(row + c0, v);
  } else if (!WHOLE) {
    float x[Piece<T>::E];
    Piece<T>::unpack(v, x);
    store_part(row, c0, d, x);
  }
}

// A row's pieces as they are loaded (a gate of one row is kept with the gains).
template <int K>
struct BlockRow {
  u32x4 x[K], h[K], y[K], d[K], g[K];
};
template <typename T, int R, int K>
__device__ __forceinline__ void fetch_row(const BlockNormGradArgs &a, int64_t i, int c, int d,
                                          BlockRow<K> &r) {
  constexpr int E = Piece<T>::E;
  const auto each = [&](u32x4(&to)[K], const void *p, int64_t ld) {
    const T *row = static_cast<const T *>(p) + i * ld;
#pragma unroll
    for (int k = 0; k < K; ++k) to[k] = take(row, c + k * R * E, d);
  };
  if (a.post || a.gate) each(r.x, a.X, a.ldx);
  if (a.dY) {
    each(r.h, a.H, a.ldh);
    each(r.y, a.dY, a.lddy);
  }
  if (a.dH) each(r.d, a.dH, a.lddh);
  if (a.gate && a.ldgate) each(r.g, a.gate, a.ldgate);
}

// NEXT: a workgroup's next row is sent for before the present one is worked on, so that its
// two waits at barriers leave the memory busy.  Values are taken from their pieces two at a
// time, and u = dy w and dh take the places of dY and dH: with eight at a time 1024 threads
// had 176 bytes of scratch (16383 x 8192 bf16 1260 us).
template <typename T, int R, int K, int NT, bool WHOLE, bool NEXT>
__global__ __launch_bounds__(NT, 2) void block_norm_grad_kernel(BlockNormGradArgs a) {
  constexpr int E = Piece<T>::E, W = R / 64, ROWS = NT / R, P = E / 2;
  static_assert(ROWS == 1 || W == 1, "a row of several waves has the workgroup to itself");
  __shared__ float red[3][W], red2[1][W];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / R);
  const int c = static_cast<int>(threadIdx.x % R) * E, d = static_cast<int>(a.d);
  const bool need_x = a.post || a.gate;
  // The gains and the one gate row of this thread's columns: kept, or (longer rows) loaded
  // again where they are used.
  constexpr bool KEEP = NEXT;
  u32x4 ones;
#pragma unroll
  for (int q = 0; q < P; ++q) set_pair<T>(ones, q, 1.0f, 1.0f);
  const auto gains = [&](const void *p, int k) {
    const int c0 = c + k * R * E;
    return p ? fix<T, WHOLE>(take(static_cast<const T *>(p), c0, d), c0, d) : ones;
  };
  const void *post_gains = a.post ? a.w_post : nullptr, *row_gate = a.ldgate ? nullptr : a.gate;
  u32x4 w_kept[K], w1_kept[K], gate_kept[K];
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      w_kept[k] = gains(a.w, k);
      w1_kept[k] = gains(post_gains, k);
      gate_kept[k] = gains(row_gate, k);
    }
  }
  float sum[3][K][E] = {};
  int64_t i = static_cast<int64_t>(blockIdx.x) * ROWS + sub;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * ROWS;
  BlockRow<K> later;
  if (NEXT && i < a.N) fetch_row<T, R, K>(a, i, c, d, later);
  for (; i < a.N; i += stride) {
    BlockRow<K> r;
    if constexpr (NEXT) {
      r = later;
      if (i + stride < a.N) fetch_row<T, R, K>(a, i + stride, c, d, later);
    } else {
      fetch_row<T, R, K>(a, i, c, d, r);
    }
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = c + k * R * E;
      if (need_x) {
        r.x[k] = fix<T, WHOLE>(r.x[k], c0, d);
#pragma unroll
        for (int q = 0; q < P; ++q) {
          float x0, x1;
          pair_of<T>(r.x[k], q, x0, x1);
          s[0] = fmaf(x1, x1, fmaf(x0, x0, s[0]));
        }
      }
      if (a.dY) {
        r.h[k] = fix<T, WHOLE>(r.h[k], c0, d);
        r.y[k] = fix<T, WHOLE>(r.y[k], c0, d);
        const u32x4 w = KEEP ? w_kept[k] : gains(a.w, k);
#pragma unroll
        for (int q = 0; q < P; ++q) {
          float h0, h1, y0, y1, w0, w1v;
          pair_of<T>(r.h[k], q, h0, h1);
          pair_of<T>(r.y[k], q, y0, y1);
          pair_of<T>(w, q, w0, w1v);
          s[1] = fmaf(h1, h1, fmaf(h0, h0, s[1]));
          s[2] = fmaf(y1 * w1v, h1, fmaf(y0 * w0, h0, s[2]));
        }
      }
      if (a.dH) r.d[k] = fix<T, WHOLE>(r.d[k], c0, d);
      if (a.gate && a.ldgate) r.g[k] = fix<T, WHOLE>(r.g[k], c0, d);
    }
    group_sums<W>(s, red);
    const float q1 = a.post ? 1.0f / sqrtf(s[0] * a.inv_d + a.eps) : 1.0f;
    const float rho = 1.0f / sqrtf(s[1] * a.inv_d + a.eps), f = s[2] * a.inv_d * rho;
    T *dR = static_cast<T *>(a.dR) + i * a.lddr;
    T *dX = static_cast<T *>(a.dX) + i * a.lddx;
    T *dG = a.dgate ? static_cast<T *>(a.dgate) + i * a.lddg : nullptr;
    float v[K][E], sv[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c0 = c + k * R * E;
      const u32x4 w = KEEP ? w_kept[k] : gains(a.w, k), w1 = KEEP ? w1_kept[k] : gains(post_gains, k);
      const u32x4 gate = a.ldgate ? r.g[k] : KEEP ? gate_kept[k] : gains(row_gate, k);
      u32x4 out_r, out_g, out_x;
#pragma unroll
      for (int q = 0; q < P; ++q) {
        float o[2] = {0.0f, 0.0f}, g[2] = {1.0f, 1.0f}, x[2] = {0.0f, 0.0f}, wp[2], t[2];
        if (a.dH) pair_of<T>(r.d[k], q, o[0], o[1]);
        if (a.dY) {
          float h[2], y[2];
          pair_of<T>(r.h[k], q, h[0], h[1]);
          pair_of<T>(r.y[k], q, y[0], y[1]);
          pair_of<T>(w, q, t[0], t[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float n = h[e] * rho;
            sum[kGw][k][2 * q + e] = fmaf(y[e], n, sum[kGw][k][2 * q + e]);
            o[e] = fmaf(rho, fmaf(-n, f, y[e] * t[e]), o[e]);
          }
        }
        set_pair<T>(out_r, q, a.alpha * o[0], a.alpha * o[1]);
        pair_of<T>(w1, q, wp[0], wp[1]);
        if (need_x) {
          pair_of<T>(r.x[k], q, x[0], x[1]);
          x[0] *= q1;
          x[1] *= q1;
        }
        if (a.gate) {
          pair_of<T>(gate, q, g[0], g[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float slope = 1.0f;
            if (a.sigmoid) g[e] = sigmoid_of<T>(g[e], &slope);
            t[e] = o[e] * x[e] * wp[e] * slope;
            if (!dG) sum[kGate][k][2 * q + e] += t[e];
            o[e] *= g[e];
          }
          set_pair<T>(out_g, q, t[0], t[1]);
        }
        if (a.post) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            sum[kGwPost][k][2 * q + e] = fmaf(o[e], x[e], sum[kGwPost][k][2 * q + e]);
            v[k][2 * q + e] = o[e] * wp[e];
            sv[0] = fmaf(v[k][2 * q + e], x[e], sv[0]);
          }
        }
        set_pair<T>(out_x, q, o[0], o[1]);
      }
      put_piece<T, WHOLE>(dR, c0, d, out_r);
      if (dG) put_piece<T, WHOLE>(dG, c0, d, out_g);
      if (!a.post) put_piece<T, WHOLE>(dX, c0, d, out_x);
    }
    if (a.post) {
      group_sums<W>(sv, red2);
      const float f1 = sv[0] * a.inv_d * q1;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        u32x4 out_x;
#pragma unroll
        for (int q = 0; q < P; ++q) {
          float x[2];
          pair_of<T>(r.x[k], q, x[0], x[1]);
          set_pair<T>(out_x, q, q1 * fmaf(-x[0], f1, v[k][2 * q]), q1 * fmaf(-x[1], f1, v[k][2 * q + 1]));
        }
        put_piece<T, WHOLE>(dX, c + k * R * E, d, out_x);
      }
    } else if constexpr (W > 1) {
      __syncthreads();  // red is used again
    }
  }
  if (!a.part) return;
  float *part = a.part + static_cast<int64_t>(blockIdx.x) * a.d;
#pragma unroll
  for (int q = 0; q < 3; ++q, part += static_cast<int64_t>(gridDim.x) * a.d) {
    if (!a.sums[q]) continue;
    if constexpr (ROWS == 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c0 = c + k * R * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c0 + e < d) part[c0 + e] = sum[q][k][e];
      }
    } else {  // the waves' rows are added in order
      __shared__ float rows[ROWS][K * R * E];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) rows[sub][c + k * R * E + e] = sum[q][k][e];
      __syncthreads();
      for (int j = threadIdx.x; j < d; j += NT) {
        float t = rows[0][j];
#pragma unroll
        for (int p = 1; p < ROWS; ++p) t += rows[p][j];
        part[j] = t;
      }
    }
  }
}

// Rows longer than the registers hold, or shorter than a piece: the parts of the sums are
// kept in the workspace between the workgroup's rows.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_grad_long_kernel(BlockNormGradArgs a) {
  constexpr int E = Piece<T>::E, NT = 1024, W = NT / 64;
  __shared__ float red[3][W], red2[1][W];
  const T *w = static_cast<const T *>(a.w), *w1 = static_cast<const T *>(a.w_post);
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const T *X = static_cast<const T *>(a.X) + i * a.ldx;
    const T *H = static_cast<const T *>(a.H) + i * a.ldh;
    const T *dY = a.dY ? static_cast<const T *>(a.dY) + i * a.lddy : nullptr;
    const T *dH = a.dH ? static_cast<const T *>(a.dH) + i * a.lddh : nullptr;
    float x[E], h[E], y[E], t[E], s[3] = {0.0f, 0.0f, 0.0f};
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      if (a.post) {
        get(X, c0, a.d, x);
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      }
      if (dY) {
        get(H, c0, a.d, h);
        get(dY, c0, a.d, y);
        if (w) get(w, c0, a.d, t);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          s[1] = fmaf(h[e], h[e], s[1]);
          s[2] = fmaf(w ? y[e] * t[e] : y[e], h[e], s[2]);
        }
      }
    }
    group_sums<W>(s, red);
    const float q = a.post ? 1.0f / sqrtf(s[0] * a.inv_d + a.eps) : 1.0f;
    const float rho = 1.0f / sqrtf(s[1] * a.inv_d + a.eps), f = s[2] * a.inv_d * rho;
    // o: dh, x: m (or x), t: the post norm's gains, g: the gate, all of this column
    float o[E], g[E], slope[E], n[E];
    const auto column = [&](int64_t c0) {
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = n[e] = y[e] = 0.0f;
      if (dH) get(dH, c0, a.d, o);
      if (dY) {
        get(H, c0, a.d, h);
        get(dY, c0, a.d, y);
        if (w) get(w, c0, a.d, t);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          n[e] = h[e] * rho;
          o[e] = fmaf(rho, fmaf(-n[e], f, w ? y[e] * t[e] : y[e]), o[e]);
        }
      }
      get(X, c0, a.d, x);
      if (w1) get(w1, c0, a.d, t);
      if (a.gate) get(gate_row<T>(a, i), c0, a.d, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] *= q;
        if (!a.post || !w1) t[e] = 1.0f;
        slope[e] = 1.0f;
        if (!a.gate) g[e] = 1.0f;
        if (a.gate && a.sigmoid) g[e] = sigmoid_of<T>(g[e], &slope[e]);
      }
    };
    float f1 = 0.0f;
    if (a.post) {
      float sv[1] = {0.0f};
      for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
        column(c0);
#pragma unroll
        for (int e = 0; e < E; ++e) sv[0] = fmaf(o[e] * g[e] * t[e], x[e], sv[0]);
      }
      group_sums<W>(sv, red2);
      f1 = sv[0] * a.inv_d;
    } else {
      __syncthreads();  // red is used again
    }
    const bool first = i == blockIdx.x;
    float *part = a.part ? a.part + static_cast<int64_t>(blockIdx.x) * a.d : nullptr;
    const auto add = [&](int which, int64_t col, float v) {
      if (!part || !a.sums[which] || col >= a.d) return;
      float *p = part + which * static_cast<int64_t>(gridDim.x) * a.d + col;
      *p = (first ? 0.0f : *p) + v;
    };
    for (int64_t c0 = threadIdx.x * E; c0 < a.d; c0 += NT * E) {
      column(c0);
      float r[E], dg[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        r[e] = a.alpha * o[e];
        dg[e] = o[e] * x[e] * t[e] * slope[e];
        const float dz = o[e] * g[e];
        add(kGw, c0 + e, y[e] * n[e]);
        add(kGwPost, c0 + e, dz * x[e]);
        add(kGate, c0 + e, dg[e]);
        o[e] = a.post ? q * fmaf(-x[e], f1, dz * t[e]) : dz;
      }
      put(static_cast<T *>(a.dR) + i * a.lddr, c0, a.d, r);
      if (a.dgate) put(static_cast<T *>(a.dgate) + i * a.lddg, c0, a.d, dg);
      put(static_cast<T *>(a.dX) + i * a.lddx, c0, a.d, o);
    }
  }
}

// sums[q][c] += sum over the parts, in float64 and in a fixed order: 32 groups of threads
// take every 32nd part of 32 columns, then the groups in order.
constexpr int kSumCols = 32, kSumGroups = 32;
__global__ __launch_bounds__(kSumCols *kSumGroups) void block_sum_kernel(const float *__restrict__ part,
                                                                         int64_t parts, int64_t d,
                                                                         BlockNormGradArgs a) {
  __shared__ double red[kSumGroups][kSumCols];
  const int64_t blocks = (d + kSumCols - 1) / kSumCols, id = group_number();
  if (id >= 3 * blocks) return;
  const int which = static_cast<int>(id / blocks);
  float *to = which == 0 ? a.sums[0] : which == 1 ? a.sums[1] : a.sums[2];
  if (!to) return;
  part += which * parts * d;
  const int lane = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
  const int64_t c = (id - which * blocks) * kSumCols + lane;
  double s = 0.0;
  if (c < d) {
#pragma unroll 8
    for (int64_t b = g; b < parts; b += kSumGroups) s += static_cast<double>(part[b * d + c]);
  }
  red[g][lane] = s;
  __syncthreads();
  if (g != 0 || c >= d) return;
#pragma unroll
  for (int i = 1; i < kSumGroups; ++i) s += red[i][lane];
  to[c] = static_cast<float>(static_cast<double>(to[c]) + s);
}

template <typename T, bool WHOLE>
hipError_t launch_norm_t(const BlockNormArgs &a, hipStream_t s) {
  const int64_t n = ceil_div(a.d, Piece<T>::E);
  const auto grid = [&](int rows) { return groups_grid(ceil_div(a.N, rows)); };
  if (a.d < Piece<T>::E)  // no whole piece to take
    block_norm_long_kernel<T><<<grid(1), 1024, 0, s>>>(a);
  else if (n <= 64)
    block_norm_kernel<T, 64, 1, 256, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 128)
    block_norm_kernel<T, 64, 2, 256, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 256)
    block_norm_kernel<T, 64, 4, 256, WHOLE><<<grid(4), 256, 0, s>>>(a);
  else if (n <= 512)
    block_norm_kernel<T, 256, 2, 256, WHOLE><<<grid(1), 256, 0, s>>>(a);
  else if (n <= 768)
    block_norm_kernel<T, 256, 3, 256, WHOLE><<<grid(1), 256, 0, s>>>(a);
  else if (n <= 1024)
    block_norm_kernel<T, 512, 2, 512, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else if (n <= 1536)
    block_norm_kernel<T, 512, 3, 512, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else if (n <= 2048)
    block_norm_kernel<T, 512, 4, 512, WHOLE><<<grid(1), 512, 0, s>>>(a);
  else
    block_norm_long_kernel<T><<<grid(1), 1024, 0, s>>>(a);
  return hipGetLastError();
}

int64_t pieces_of(int dt, int64_t d) { return ceil_div(d, dt == 0 ? 4 : 8); }
// Workgroups of the backward, each with a part of the column sums: as many as run at a time,
// but some 5 rows for each, so that the parts stay small beside the rows.
int64_t grad_groups(int dt, int64_t N, int64_t d) {
  const int64_t n = pieces_of(dt, d);
  const int64_t rows = n <= 64 ? 4 : 1;  // of a workgroup at a time
  const int64_t most = n <= 64 ? 768 : n <= 128 ? 1536 : n <= 256 ? 768 : n <= 512 ? 512 : 256;
  const int64_t few = ceil_div(N, 5 * rows), all = ceil_div(N, rows);
  int64_t g = few < 256 ? (all < 256 ? all : 256) : few;
  return g < most ? g : most;
}

template <typename T, bool WHOLE>
hipError_t launch_grad_t(int dt, const BlockNormGradArgs &a, hipStream_t s) {
  const int64_t n = ceil_div(a.d, Piece<T>::E);
  const unsigned g = static_cast<unsigned>(grad_groups(dt, a.N, a.d));
  if (a.d < Piece<T>::E)
    block_norm_grad_long_kernel<T><<<g, 1024, 0, s>>>(a);
  else if (n <= 64)
    block_norm_grad_kernel<T, 64, 1, 256, WHOLE, true><<<g, 256, 0, s>>>(a);
  else if (n <= 128)
    block_norm_grad_kernel<T, 128, 1, 128, WHOLE, true><<<g, 128, 0, s>>>(a);
  else if (n <= 256)
    block_norm_grad_kernel<T, 256, 1, 256, WHOLE, true><<<g, 256, 0, s>>>(a);
  else if (n <= 512)
    block_norm_grad_kernel<T, 256, 2, 256, WHOLE, true><<<g, 256, 0, s>>>(a);
  else if (n <= 1024)
    block_norm_grad_kernel<T, 512, 2, 512, WHOLE, true><<<g, 512, 0, s>>>(a);
  else if (n <= 1536)  // (ragged bf16 rows: 12 registers in scratch memory)
    block_norm_grad_kernel<T, 512, 3, 512, WHOLE, false><<<g, 512, 0, s>>>(a);
  else if (n <= 2048) {
    // Such rows and their three column sums do not fit the registers: of float32 2 go to scratch memory
    // (ragged rows 8), of bf16 60 (119; of 1024 x 2, whose threads have half as many, 80 and 103).
    // bf16 4096 x 16000 takes 390 us, 2.0 TB/s, 4096 x 13001 515.
    if constexpr (sizeof(T) == 4)
      block_norm_grad_kernel<T, 1024, 2, 1024, WHOLE, false><<<g, 1024, 0, s>>>(a);
    else
      block_norm_grad_kernel<T, 512, 4, 512, WHOLE, false><<<g, 512, 0, s>>>(a);
  } else {
    block_norm_grad_long_kernel<T><<<g, 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(int dt, const BlockNormArgs &a, hipStream_t s) {
  if (dt == 0)
    return a.d % 4 == 0 ? launch_norm_t<float, true>(a, s) : launch_norm_t<float, false>(a, s);
  return a.d % 8 == 0 ? launch_norm_t<bf16_t, true>(a, s) : launch_norm_t<bf16_t, false>(a, s);
}

size_t block_norm_grad_workspace_bytes(int dt, int64_t N, int64_t d) {
  return align256(static_cast<size_t>(grad_groups(dt, N, d)) * d * sizeof(float) * 3);
}

hipError_t launch_block_norm_grad(int dt, BlockNormGradArgs a, void *ws, hipStream_t s) {
  const bool sums = a.sums[0] || a.sums[1] || a.sums[2];
  a.part = sums ? static_cast<float *>(ws) : nullptr;
  hipError_t e;
  if (dt == 0)
    e = a.d % 4 == 0 ? launch_grad_t<float, true>(dt, a, s) : launch_grad_t<float, false>(dt, a, s);
  else
    e = a.d % 8 == 0 ? launch_grad_t<bf16_t, true>(dt, a, s) : launch_grad_t<bf16_t, false>(dt, a, s);
  if (e != hipSuccess || !sums) return e;
  block_sum_kernel<<<groups_grid(3 * ceil_div(a.d, kSumCols)), kSumCols * kSumGroups, 0, s>>>(
      a.part, grad_groups(dt, a.N, a.d), a.d, a);
  return hipGetLastError();
}

}  // namespace sn
