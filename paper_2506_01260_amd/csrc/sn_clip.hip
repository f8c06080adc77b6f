// Global gradient norm over many tensors, and clipping:
//   sumsq = sum of g^2 over all tensors,  norm = sqrt(sumsq),
//   g <- g * (norm <= max_norm ? 1 : max_norm / norm).
// Two calls, so that the sum can be reduced over ranks between them.
//
// Memory-bound: the first reads every gradient, the second reads and writes it.
// The tensors' places travel in the kernel's arguments, kClipTensors per launch,
// and are cut into units of about the same size, one workgroup each: many small
// tensors cost one launch.  Squares are summed in float64 (no square of a float
// overflows it), a unit's threads in a tree, then the units in a fixed order.
#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

constexpr int kNT = 256;

// Elements of a unit: 16384, or 2048 (a piece or two for each thread) where that
// leaves fewer than two workgroups for each CU.
int64_t unit_elems(int64_t total) { return total >= (int64_t(1) << 23) ? 16384 : 2048; }

// Units of a tensor: pieces of `u` columns of a row, or u / cols rows together.
int64_t units_of(const ClipTensor &t, int64_t u) {
  if (t.rows == 0 || t.cols == 0) return 0;
  return t.cols >= u ? t.rows * ceil_div(t.cols, u) : ceil_div(t.rows, u / t.cols);
}

// rows [r0, r1) x columns [c0, c1) of tensor t
struct Unit {
  int t;
  int64_t r0, r1, c0, c1;
};

__device__ __forceinline__ Unit unit_at(const ClipTable &tab, uint32_t unit, int64_t u) {
  int lo = 0, hi = tab.n;  // the last tensor whose first unit is <= unit
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tab.unit0[mid] <= unit) lo = mid;
    else hi = mid;
  }
  const ClipTensor &t = tab.t[lo];
  const uint32_t k = unit - tab.unit0[lo];
  Unit x;
  x.t = lo;
  if (t.cols >= u) {
    const int64_t parts = (t.cols + u - 1) / u;
    x.r0 = k / parts;
    x.r1 = x.r0 + 1;
    x.c0 = (k - x.r0 * parts) * u;
    x.c1 = x.c0 + u < t.cols ? x.c0 + u : t.cols;
  } else {
    const int64_t per = u / t.cols;
    x.r0 = k * per;
    x.r1 = x.r0 + per < t.rows ? x.r0 + per : t.rows;
    x.c0 = 0;
    x.c1 = t.cols;
  }
  return x;
}

// The unit's elements, piece by piece: f(row, column, columns in the piece).
template <int E, typename F>
__device__ __forceinline__ void each_piece(const Unit &x, F &&f) {
  const uint32_t n = static_cast<uint32_t>(x.c1 - x.c0), per = (n + E - 1) / E;
  const uint32_t all = per * static_cast<uint32_t>(x.r1 - x.r0);
  if (x.r1 - x.r0 == 1) {
#pragma unroll 4
    for (uint32_t q = threadIdx.x; q < all; q += kNT) f(x.r0, x.c0 + q * E);
  } else {
    for (uint32_t q = threadIdx.x; q < all; q += kNT) {
      const uint32_t r = q / per;
      f(x.r0 + r, x.c0 + static_cast<int64_t>(q - r * per) * E);
    }
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

template <typename T>
__device__ __forceinline__ double unit_sumsq(const ClipTensor &t, const Unit &x) {
  constexpr int E = Piece<T>::E;
  const T *g = static_cast<const T *>(t.g);
  double s = 0.0;
  each_piece<E>(x, [&](int64_t r, int64_t c) {
    float v[E];
    const T *row = g + r * t.ldg;
    if (c + E <= x.c1)
      Piece<T>::unpack(load_piece(row + c), v);
    else
      load_part(row, c, x.c1, 0.0f, v);
#pragma unroll
    for (int e = 0; e < E; ++e) s = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), s);
  });
  return s;
}

__global__ __launch_bounds__(kNT) void sumsq_kernel(ClipTable tab, int64_t u,
                                                    double *__restrict__ part) {
  __shared__ double red[kNT / 64];
  const Unit x = unit_at(tab, blockIdx.x, u);
  const ClipTensor &t = tab.t[x.t];
  double s = t.f32 ? unit_sumsq<float>(t, x) : unit_sumsq<bf16_t>(t, x);
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kNT / 64; ++i) s += red[i];
    part[blockIdx.x] = s;
  }
}

// the units' sums; one workgroup
__global__ __launch_bounds__(1024) void sumsq_total_kernel(const double *__restrict__ part,
                                                           int64_t n, double *__restrict__ out) {
  __shared__ double red[16];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i];
    *out = s;
  }
}

template <typename T>
__device__ __forceinline__ void unit_scale(const ClipTensor &t, const Unit &x, float f) {
  constexpr int E = Piece<T>::E;
  const T *g = static_cast<const T *>(t.g);
  T *o = static_cast<T *>(t.out);
  each_piece<E>(x, [&](int64_t r, int64_t c) {
    float v[E];
    const T *src = g + r * t.ldg;
    T *dst = o + r * t.ldo;
    if (c + E <= x.c1) {
      Piece<T>::unpack(load_piece(src + c), v);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= f;
      store_piece(dst + c, Piece<T>::pack(v));
    } else {
      load_part(src, c, x.c1, 0.0f, v);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] *= f;
      store_part(dst, c, x.c1, v);
    }
  });
}

__global__ __launch_bounds__(kNT) void clip_kernel(ClipTable tab, int64_t u, int in_place,
                                                   const double *__restrict__ sumsq,
                                                   double max_norm, float *__restrict__ norm_out) {
  const double norm = sqrt(*sumsq);
  // a NaN norm fails the comparison and makes the factor a NaN
  const float f = norm <= max_norm ? 1.0f : static_cast<float>(max_norm / norm);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = static_cast<float>(norm);
  if (tab.n == 0 || (in_place && f == 1.0f)) return;  // every value is its own product
  const Unit x = unit_at(tab, blockIdx.x, u);
  const ClipTensor &t = tab.t[x.t];
  if (t.f32)
    unit_scale<float>(t, x, f);
  else
    unit_scale<bf16_t>(t, x, f);
}

// Tables of up to kClipTensors tensors that have elements: launch(table, units).
template <typename F>
hipError_t each_table(const ClipTensor *t, int32_t count, int64_t u, F &&launch) {
  ClipTable tab;
  int64_t units = 0;
  for (int32_t i = 0; i <= count; ++i) {
    const int64_t more = i < count ? units_of(t[i], u) : 0;
    // a grid holds fewer than 2^32 threads
    if (tab.n && (i == count || tab.n == kClipTensors || units + more > (1 << 23))) {
      launch(tab, static_cast<unsigned>(units));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      tab.n = 0;
      units = 0;
    }
    if (more == 0) continue;
    tab.t[tab.n] = t[i];
    tab.unit0[tab.n++] = static_cast<uint32_t>(units);
    units += more;
  }
  return hipSuccess;
}

int64_t total_elems(const ClipTensor *t, int32_t count) {
  int64_t n = 0;
  for (int32_t i = 0; i < count; ++i) n += t[i].rows * t[i].cols;
  return n;
}

}  // namespace

int64_t clip_units(const ClipTensor *t, int32_t count) {
  const int64_t u = unit_elems(total_elems(t, count));
  int64_t n = 0;
  for (int32_t i = 0; i < count; ++i) n += units_of(t[i], u);
  return n;
}

hipError_t launch_sumsq(const ClipTensor *t, int32_t count, double *sumsq, void *ws,
                        hipStream_t s) {
  const int64_t u = unit_elems(total_elems(t, count));
  double *part = static_cast<double *>(ws);
  int64_t n = 0;
  const hipError_t e = each_table(t, count, u, [&](const ClipTable &tab, unsigned units) {
    sumsq_kernel<<<units, kNT, 0, s>>>(tab, u, part + n);
    n += units;
  });
  if (e != hipSuccess) return e;
  sumsq_total_kernel<<<1, 1024, 0, s>>>(part, n, sumsq);
  return hipGetLastError();
}

hipError_t launch_clip(const ClipTensor *t, int32_t count, bool in_place, const double *sumsq,
                       double max_norm, float *norm, hipStream_t s) {
  const int64_t u = unit_elems(total_elems(t, count));
  bool told = norm == nullptr;
  const hipError_t e = each_table(t, count, u, [&](const ClipTable &tab, unsigned units) {
    clip_kernel<<<units, kNT, 0, s>>>(tab, u, in_place, sumsq, max_norm, told ? nullptr : norm);
    told = true;
  });
  if (e != hipSuccess || told) return e;
  clip_kernel<<<1, kNT, 0, s>>>(ClipTable(), u, in_place, sumsq, max_norm, norm);  // nothing to scale
  return hipGetLastError();
}

}  // namespace sn
