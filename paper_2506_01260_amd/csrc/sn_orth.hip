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
// A result of bf16 needs the same: roundings to 11 bits average out in random matrices (1e-3 of the
// result's norm with hi hi alone for A and A^2), but are all alike in matrices of equal or few
// distinct values, where they add up: 5e-3 to 8e-3 for constant matrices, one-hot rows and
// diagonal blocks, whose rounding to bf16 is 1.6e-3 to 3.1e-3.
// What 2^-22 leaves in directions that X does not have grows by 3.4445 a step, to some
// 2^-24.5 3.4445^steps of the norm (rank 4 of 1024 x 1024: 2e-5 after 5 steps, 7e-4 after 8, 0.1
// after 12): the steps are limited to 8.
// A and Q are symmetric: the tiles on and below the diagonal are computed and mirrored.
// Matrices of one shape share every launch.
//
// Bounds and times of a whole update: the matrix cores in large matrices (four of 4096 x 4096
// bf16 15.6 ms, 1060 TFLOP/s, of it 0.27 the two passes over gradient and momentum at 5 TB/s), how
// whole tiles fit the matrix in middling ones (two of 1600 x 4267 float32 1.6 ms, one of
// 1024 x 4096 0.51), the launches of three products a step in small ones (six of 256 x 256 102 us).
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
  const int64_t left = a.cols - c;
  f32x4 g = {0, 0, 0, 0};
  if (!a.update || first || a.nesterov)
    g = get4(static_cast<const T *>(t.g[z]) + r * t.ldg[z] + c, left);
  if (!a.update) return g;
  float *at = t.m[z] + r * t.ldm[z] + c;
  f32x4 m = get4(at, left);
  if (first) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = fmaf(a.momentum, m[e], g[e]);
    put4(at, left, m);
  }
  if (a.nesterov) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = fmaf(a.momentum, m[e], g[e]);
  }
  return m;
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
// fp16 planes of four values
__device__ __forceinline__ void orth_put(uint16_t *to, int64_t plane, f32x4 v) {
  uint16_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = f16_bits(v[e]);
    l[e] = f16_bits((v[e] - f16_value(h[e])) * kUp);
  }
  *reinterpret_cast<u32x2 *>(to) =
      u32x2{h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16};
  *reinterpret_cast<u32x2 *>(to + plane) =
      u32x2{l[0] | static_cast<uint32_t>(l[1]) << 16, l[2] | static_cast<uint32_t>(l[3]) << 16};
}

__device__ __forceinline__ f32x4 orth_get(const uint16_t *from, int64_t plane) {
  const u32x2 h = *reinterpret_cast<const u32x2 *>(from), l = *reinterpret_cast<const u32x2 *>(from + plane);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int bits = 16 * (e & 1);
    v[e] = fmaf(f16_value(static_cast<uint16_t>((e < 2 ? l.x : l.y) >> bits)), 1.0f / kUp,
                f16_value(static_cast<uint16_t>((e < 2 ? h.x : h.y) >> bits)));
  }
  return v;
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

// The symmetric products, n x n with stride ldp: A from X, or (POLY) Q from A.
template <bool POLY>
struct OrthSym {
  int64_t n, ldp;
  const uint16_t *A;
  uint16_t *to;
  template <class S>
  __device__ __forceinline__ void row(const MmPlace &p, int64_t row, int64_t col0,
                                      f32x4 (&acc)[S::TN]) const {
    const int64_t plane = n * ldp;
    uint16_t *out = to + p.z * 2 * plane;
    const uint16_t *in = POLY ? A + p.z * 2 * plane : nullptr;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int64_t col = col0 + j * 16;
      if (row >= ldp || col >= ldp) continue;
      f32x4 v, at = {0, 0, 0, 0};
      if (POLY && row < n) at = orth_get(in + row * ldp + col, plane);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool inside = row < n && col + e < n;
        if constexpr (POLY) {
          const float one = row == col + e ? kA * kQScale : 0.0f;
          v[e] = fmaf(kC * kQScale / (kXScale * kXScale), acc[j][e],
                      fmaf(kB * kQScale / kXScale, at[e], one));
        } else {
          v[e] = acc[j][e] * (1.0f / kXScale);
        }
        if (!inside) v[e] = 0.0f;
      }
      if (row < n) orth_put(out + row * ldp + col, plane, v);
      if (p.tm == p.tn) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (col + e >= n) continue;
        uint16_t *q = out + (col + e) * ldp + row;
        q[0] = f16_bits(v[e]);
        q[plane] = f16_bits((v[e] - f16_value(f16_bits(v[e]))) * kUp);
      }
    }
  }
};

// X' = Q X or X Q, in planes, or in its place in the table.
template <bool LAST, typename T>
struct OrthApply {
  OrthMats t;
  OrthArgs a;
  uint16_t *to;
  int64_t ldp;
  template <class S>
  __device__ __forceinline__ void row(const MmPlace &p, int64_t row, int64_t col0,
                                      f32x4 (&acc)[S::TN]) const {
    if (row >= a.rows) return;
    const int64_t plane = a.rows * ldp;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int64_t col = col0 + j * 16;
      if (col >= ldp) continue;
      f32x4 v = acc[j];
      if constexpr (LAST) {
        T *w = static_cast<T *>(t.w[p.z]) + row * t.ldw[p.z] + col;
        const int64_t left = a.cols - col;
        if (left <= 0) continue;
        v *= 1.0f / (kXScale * kQScale);
        if (a.update) {
          const f32x4 old = get4(w, left);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(-a.rate, v[e], fmaf(-a.decay, old[e], old[e]));
        }
        put4(w, left, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = col + e < a.cols ? v[e] * (1.0f / kQScale) : 0.0f;
        orth_put(to + p.z * 2 * plane + row * ldp + col, plane, v);
      }
    }
  }
};

// ---- products of small matrices ---------------------------------------------------------
// Where a product has few tiles its time is that of its steps, one after the other.  Here a
// workgroup holds 32 x 32 sums, a wave 16 x 16 of them, and has 256 k values of both planes of both
// operands in the LDS: one wait for K <= 256 instead of twelve.  Five steps over six 256 x 256
// float32 matrices take 108 us, 149 with tiles of 64 x 64; each of the 17 launches is
// then bound by its own latency.  Layout: KC, piece p of a row's 32 lies at p ^ (row % 16); else
// 64 bytes a k, the second of its two chunks first where k / 8 is odd.
struct SmallShape {
  static constexpr int BM = 32, BN = 32, WM = 2, WN = 2, TN = 1, PAIR = 0;
};
constexpr int kSmallK = 256, kSmallPlane = 32 * kSmallK * 2, kSmallBytes = 4 * kSmallPlane;

// This lane's part of an operand's planes from k0 on, 16 loads of 1 KB a plane.
template <bool KC>
__device__ __forceinline__ void small_load(const uint16_t *p, int64_t ld, int64_t n, int64_t r0, int64_t k0,
                                           int64_t K, uint32_t lds, int wave, int lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int idx = (j * 4 + wave) * 64 + lane;
    const uint16_t *src;
    bool there;
    if constexpr (KC) {
      const int r = idx >> 5, k = ((idx & 31) ^ (r & 15)) * 8;
      src = p + min(r0 + r, n - 1) * ld + k0 + k;
      there = k0 + k < K;
    } else {
      const int k = idx >> 2, slot = idx & 3;
      const int c = (((slot >> 1) ^ (k >> 3 & 1)) << 4) | ((slot & 1) << 3);
      src = p + (k0 + k) * ld + min(r0 + c, n - 8);
      there = k0 + k < K;
    }
    lds_load_16(there ? static_cast<const void *>(src) : &mm_zeros, lds + (j * 4 + wave) * 1024);
  }
}
// The fragment of 16 rows from `half` of the tile, k values 32 ks ..
template <bool KC>
__device__ __forceinline__ u32x4 small_read(const char *lds, int half, int ks, int lane) {
  const int g = lane >> 4, n = lane & 15;
  if constexpr (KC) {
    return *reinterpret_cast<const u32x4 *>(lds + (half * 16 + n) * 512 + (((ks * 4 + g) ^ n) << 4));
  } else {
    u32x2 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *q = lds + (ks * 32 + 8 * g + 4 * h + (n >> 2)) * 64 + ((half ^ (g & 1)) << 5) + (n & 3) * 8;
      v[h] = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                     (__attribute__((address_space(3))) s16x4 *)(const_cast<char *>(q))));
    }
    return u32x4{v[0].x, v[0].y, v[1].x, v[1].y};
  }
}

// low_a, low_b: elements to the operands' low planes.  STAGES: 1 where K <= 256.
template <bool AK, bool BK, int STAGES, class Epi>
__global__ __launch_bounds__(256, 3 - STAGES) void orth_small_kernel(MmArgs m, int64_t low_a, int64_t low_b, MmGrid g,
                                                            Epi e) {
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * kSmallBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const MmPlace p = mm_where(g, blockIdx.x);
  const uint16_t *a = m.a.p[0] + p.z * (m.a.batch / 2), *b = m.b.p[0] + p.z * (m.b.batch / 2);
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(lds));
  const auto load = [&](int64_t k0, uint32_t to) {
    small_load<AK>(a, m.a.ld, m.a.n, p.tm * 32, k0, m.k, to, wave, lane);
    small_load<BK>(b, m.b.ld, m.b.n, p.tn * 32, k0, m.k, to + 2 * kSmallPlane, wave, lane);
    small_load<AK>(a + low_a, m.a.ld, m.a.n, p.tm * 32, k0, m.k, to + kSmallPlane, wave, lane);
    small_load<BK>(b + low_b, m.b.ld, m.b.n, p.tn * 32, k0, m.k, to + 3 * kSmallPlane, wave, lane);
  };
  f32x4 high = {0, 0, 0, 0}, low = {0, 0, 0, 0};
  uint32_t cur = 0;
  load(0, base);
  for (int64_t k0 = 0; k0 < m.k; k0 += kSmallK) {
    wait_vmcnt<0>();
    lds_barrier();
    if (STAGES > 1 && k0 + kSmallK < m.k) load(k0 + kSmallK, base + (cur ^ kSmallBytes));
    const char *at = lds + cur;
    const int64_t left = m.k - k0;
    const int steps = left < kSmallK ? static_cast<int>((left + 31) / 32) : kSmallK / 32;
    for (int ks = 0; ks < steps; ++ks) {
      const u32x4 ah = small_read<AK>(at, wave >> 1, ks, lane);
      const u32x4 bh = small_read<BK>(at + 2 * kSmallPlane, wave & 1, ks, lane);
      high = mm_mfma<true>(bh, ah, high);
      low = mm_mfma<true>(small_read<BK>(at + 3 * kSmallPlane, wave & 1, ks, lane), ah, low);
      low = mm_mfma<true>(bh, small_read<AK>(at + kSmallPlane, wave >> 1, ks, lane), low);
    }
    if constexpr (STAGES > 1) cur ^= kSmallBytes;
  }
  f32x4 acc[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[0][i] = fmaf(low[i], 1.0f / kUp, high[i]);
  mm_row<SmallShape>(e, p, 0, acc);
}

// Whether a product of M x N is one of small matrices: no more workgroups of 32 x 32 than run at a
// time, and k values for a few stages.  Whole calls, float32, all products in this way and all in
// the other, us: 128 x 128 40 times 228 and 254, 256 x 256 6 times 108 and 149, 12 times 143 and
// 157, 24 times 226 and 183; 512 x 512 once 121 and 203, 3 times 229 and 231; 729 x 729 266 and
// 265; 256 x 1024 112 and 165; 64 x 4096 191 and 147.
bool small_product(int64_t M, int64_t N, int64_t count, int64_t k, bool sym) {
  const int64_t r = ceil_div(M, 32), c = ceil_div(N, 32);
  return k <= 4 * kSmallK && (sym ? r * (r + 1) / 2 : r * c) * count <= (k <= kSmallK ? 512 : 256);
}

constexpr int kSegs = 3;  // hi lo, lo hi and hi hi
MmPlan cut(int64_t M, int64_t N, int64_t count, int64_t k, bool sym) {
  return mm_plan(M, N, count, ceil_div(k, kMmK) * kSegs, sym);
}
struct OrthPlan {
  int64_t n, ldx, lda;  // the smaller side; the planes' strides
  int sums;
  size_t x[2], a, q, part, sums_at, total;
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
  p.sums_at = take(sizeof(double) * count * p.sums);
  size_t part = 0;
  for (const MmPlan &m : {cut(p.n, p.n, count, rows < cols ? cols : rows, true),
                          cut(p.n, p.n, count, p.n, true), cut(rows, cols, count, p.n, false)})
    part = m.part_bytes > part ? m.part_bytes : part;
  p.part = take(part);
  p.total = at;
  return p;
}

void planes(MmArgs &m, const uint16_t *a, int64_t aplane, const uint16_t *b, int64_t bplane) {
  m.segs = kSegs;
  m.factor = 1.0f / kUp;
  m.run[0] = 2;
  m.run[1] = 3;
  m.a.p[0] = m.a.p[2] = a;
  m.a.p[1] = a + aplane;
  m.b.p[0] = b + bplane;
  m.b.p[1] = m.b.p[2] = b;
}

template <bool AK, bool BK, class Epi>
void run(const MmArgs &m, int64_t M, int64_t N, int64_t count, bool sym, float *part, const Epi &e,
         hipStream_t s) {
  if (small_product(M, N, count, m.k, sym)) {
    MmArgs h = m;
    h.b.p[0] = m.b.p[2];
    const int64_t low_a = m.a.p[1] - m.a.p[0], low_b = m.b.p[0] - m.b.p[2];
    MmGrid g = {};
    g.gm = ceil_div(M, 32);
    g.gn = ceil_div(N, 32);
    g.mats = count;
    g.sym = sym;
    const unsigned grid = static_cast<unsigned>((sym ? g.gm * (g.gm + 1) / 2 : g.gm * g.gn) * count);
    if (m.k <= kSmallK)
      orth_small_kernel<AK, BK, 1, Epi><<<grid, 256, 0, s>>>(h, low_a, low_b, g, e);
    else
      orth_small_kernel<AK, BK, 2, Epi><<<grid, 256, 0, s>>>(h, low_a, low_b, g, e);
    return;
  }
  const MmPlan p = cut(M, N, count, m.k, sym);
  MmGrid g = p.grid;
  g.part = part;
  if (p.size == 256)
    mm_launch<MmShape<true, AK, BK, 256, 256, 2, 4>>(m, g, e, s);
  else if (p.size == 128)
    mm_launch<MmShape<true, AK, BK, 128, 128, 2, 2>>(m, g, e, s);
  else
    mm_launch<MmShape<true, AK, BK, 64, 64, 2, 2, 4>>(m, g, e, s);
}

template <typename T>
hipError_t launch_orth_t(const OrthMats &t, const OrthArgs &a, char *ws, hipStream_t s) {
  const OrthPlan p = orth_plan(a.rows, a.cols, a.count);
  uint16_t *X[2] = {reinterpret_cast<uint16_t *>(ws + p.x[0]), reinterpret_cast<uint16_t *>(ws + p.x[1])};
  uint16_t *A = reinterpret_cast<uint16_t *>(ws + p.a), *Q = reinterpret_cast<uint16_t *>(ws + p.q);
  double *sums = reinterpret_cast<double *>(ws + p.sums_at);
  float *part = reinterpret_cast<float *>(ws + p.part);
  const bool tall = a.rows > a.cols;
  orth_begin_kernel<T><<<p.sums * a.count, 256, 0, s>>>(t, a, p.sums, sums);
  const int64_t turns = ceil_div(a.rows * p.ldx, kBlockElems);
  const int groups = static_cast<int>(turns < 1024 ? turns : 1024);
  orth_split_kernel<T><<<groups * a.count, 256, 0, s>>>(t, a, groups, p.sums, sums, X[0], p.ldx);
  const int64_t xplane = a.rows * p.ldx, aplane = p.n * p.lda;
  for (int i = 0; i < a.steps; ++i) {
    uint16_t *x = X[i & 1], *next = X[~i & 1];
    MmArgs m = {};
    m.k = tall ? a.rows : a.cols;
    m.a.ld = m.b.ld = p.ldx;
    m.a.n = m.b.n = tall ? p.ldx : a.rows;
    m.a.batch = m.b.batch = 4 * xplane;
    planes(m, x, xplane, x, xplane);
    const OrthSym<false> gram = {p.n, p.lda, nullptr, A};
    if (tall)
      run<false, false>(m, p.n, p.n, a.count, true, part, gram, s);
    else
      run<true, true>(m, p.n, p.n, a.count, true, part, gram, s);
    m.k = p.n;
    m.a.ld = m.b.ld = p.lda;
    m.a.n = m.b.n = p.n;
    m.a.batch = m.b.batch = 4 * aplane;
    planes(m, A, aplane, A, aplane);
    run<true, true>(m, p.n, p.n, a.count, true, part, OrthSym<true>{p.n, p.lda, A, Q}, s);
    MmOperand &o = tall ? m.a : m.b;  // X's
    o.ld = p.ldx;
    o.n = tall ? a.rows : p.ldx;
    o.batch = 4 * xplane;
    if (tall)
      planes(m, x, xplane, Q, aplane);
    else
      planes(m, Q, aplane, x, xplane);
    const auto apply = [&](const auto &e) {
      if (tall)
        run<true, true>(m, a.rows, a.cols, a.count, false, part, e, s);
      else
        run<true, false>(m, a.rows, a.cols, a.count, false, part, e, s);
    };
    if (i + 1 == a.steps)
      apply(OrthApply<true, T>{t, a, next, p.ldx});
    else
      apply(OrthApply<false, T>{t, a, next, p.ldx});
  }
  return hipGetLastError();
}

}  // namespace

// Of the launches' groups of matrices: the whole ones', or the last one's, whose few matrices may
// be cut into more parts.
size_t orth_workspace_bytes(int64_t rows, int64_t cols, int64_t count) {
  const int64_t last = count % OrthMats::kMost;
  const size_t whole = count < OrthMats::kMost ? 0 : orth_plan(rows, cols, OrthMats::kMost).total;
  const size_t rest = last ? orth_plan(rows, cols, last).total : 0;
  return whole > rest ? whole : rest;
}

hipError_t launch_orth(int dt, const OrthMats &t, const OrthArgs &a, void *ws, hipStream_t s) {
  return dt == 0 ? launch_orth_t<float>(t, a, static_cast<char *>(ws), s)
                 : launch_orth_t<bf16_t>(t, a, static_cast<char *>(ws), s);
}

}  // namespace sn
