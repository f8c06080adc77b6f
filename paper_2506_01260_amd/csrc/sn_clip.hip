// Global gradient norm over many tensors, and clipping:
//   sumsq = sum of g^2 over all tensors,  norm = sqrt(sumsq),
//   g <- g * (norm <= max_norm ? 1 : max_norm / norm).
// Two calls, so that the sum can be reduced over ranks between them.
//
// Memory-bound: the first reads every gradient, the second reads and writes it.
// The tensors' places travel in the kernel's arguments, 128 per launch (64 where some
// have gaps), and are cut into units of about the same size, one workgroup each: many
// small tensors cost one launch.  Squares are summed in float64 (no square of a float
// overflows it), a unit's threads in a tree, then the units in a fixed order.
//
// Measured: 1.1e9 bf16 gradients, norm 360 us (6.1 TB/s read) and scaling into other
// tensors 770 us (5.7 TB/s read and written), both calls 1129-1139 us, 1117 in place and
// 398 in place with the factor 1; 38 tensors of 4.5e6 floats in all, both calls
// 16.5-19.6 us, three launches (6.5, 2.3, 8.4); 155 of 6.9e6 bf16 29 us, 36 with 64 tensors
// to a launch.
#include <algorithm>
#include <cstring>

#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

constexpr int kNT = 256;
// Pieces of a thread in flight: read and summed, and read, scaled and written.
constexpr int kSumBatch = 8, kClipBatch = 4;

// Elements of a unit: 2048 (a piece or two for each thread) below 2^23 elements, to
// fill the chip.  Above, the norm's units are few enough for one workgroup to add up
// quickly (5 us for the 16900 of 1.1e9 gradients), and a clipping unit is one batch:
// 774 us there, 792 with twice as many elements and 810 with eight times.  A tensor is
// of fewer than 2^40 elements and its units of more than half as many as these, so that
// a launch has fewer than 2^29: more than one grid dimension's 2^32 threads.
int64_t sum_unit(int64_t total) {
  return total < (int64_t(1) << 23) ? 2048 : total < (int64_t(1) << 27) ? 16384 : 65536;
}
int64_t clip_unit(int64_t total) { return total < (int64_t(1) << 23) ? 2048 : 8192; }

// Units of a tensor: pieces of `u` columns of a row, or u / cols rows together.
int64_t units_of(const ClipTensor &t, int64_t u) {
  if (t.rows == 0 || t.cols == 0) return 0;
  return t.cols >= u ? t.rows * ceil_div(t.cols, u) : ceil_div(t.rows, u / t.cols);
}

// rows [r0, r1) x columns [c0, c1) of a tensor
struct Unit {
  int64_t r0, r1, c0, c1;
};

// Each lane looks at one tensor's first unit of each 64: a load and a ballot where
// halving the table takes six loads one after the other.
template <typename TAB>
__device__ __forceinline__ int tensor_at(const TAB &tab, uint32_t unit) {
  int t = -1;
#pragma unroll
  for (int i = 0; i < TAB::kTensors; i += 64)
    t += __popcll(__ballot(tab.unit0[i + (threadIdx.x & 63)] <= unit));
  return t;
}
// The unit's tensor and place.
__device__ __forceinline__ Unit unit_at(const ClipTable &tab, uint32_t unit, int64_t u,
                                        ClipTensor &t) {
  const int i = tensor_at(tab, unit);
  t = tab.t[i];
  const uint32_t k = unit - tab.unit0[i];
  const uint32_t r = t.per_row == 1 ? k : k / t.per_row;
  Unit x;
  x.r0 = static_cast<int64_t>(r) * t.rows_each;
  x.r1 = x.r0 + t.rows_each < t.rows ? x.r0 + t.rows_each : t.rows;
  x.c0 = (k - r * t.per_row) * u;
  x.c1 = x.c0 + u < t.cols ? x.c0 + u : t.cols;
  return x;
}
__device__ __forceinline__ Unit unit_at(const FlatTable &tab, uint32_t unit, int64_t u,
                                        ClipTensor &t) {
  const int i = tensor_at(tab, unit);
  const FlatTable::Tensor &f = tab.t[i];
  t.g = f.g;
  t.out = f.out;
  t.ldg = t.ldo = 0;  // one row
  t.f32 = f.size2 & 1;
  const int64_t cols = f.size2 >> 1;
  Unit x;
  x.r0 = 0;
  x.r1 = 1;
  x.c0 = (unit - tab.unit0[i]) * u;
  x.c1 = x.c0 + u < cols ? x.c0 + u : cols;
  return x;
}

// The unit's whole pieces, B of each thread at a time: load(row, column) of all of
// them, then use(row, column, piece); then the rows' ends, element by element:
// last(row, column).
template <int E, int B, typename L, typename U, typename R>
__device__ __forceinline__ void each_piece(const Unit &x, L &&load, U &&use, R &&last) {
  const uint32_t n = static_cast<uint32_t>(x.c1 - x.c0), per = n / E, rest = n % E;
  const uint32_t rows = static_cast<uint32_t>(x.r1 - x.r0), all = per * rows;
  for (uint32_t q0 = threadIdx.x; q0 < all; q0 += B * kNT) {
    u32x4 v[B];
    uint32_t r[B], c[B];
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const uint32_t q = q0 + k * kNT;
      r[k] = rows == 1 ? 0 : q / per;
      c[k] = (q - r[k] * per) * E;
      v[k] = u32x4{0, 0, 0, 0};
      if (q < all) v[k] = load(x.r0 + r[k], x.c0 + c[k]);
    }
#pragma unroll
    for (int k = 0; k < B; ++k)
      if (q0 + k * kNT < all) use(x.r0 + r[k], x.c0 + c[k], v[k]);
  }
  for (uint32_t q = threadIdx.x; q < rest * rows; q += kNT) {
    const uint32_t k = q / rest;
    last(x.r0 + k, x.c0 + per * E + (q - k * rest));
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
  const auto add = [&](float v) { s = fma(static_cast<double>(v), static_cast<double>(v), s); };
  each_piece<E, kSumBatch>(
      x, [&](int64_t r, int64_t c) { return load_piece(g + r * t.ldg + c); },
      [&](int64_t, int64_t, u32x4 p) {
        float v[E];
        Piece<T>::unpack(p, v);
#pragma unroll
        for (int e = 0; e < E; ++e) add(v[e]);
      },
      [&](int64_t r, int64_t c) { add(to_f32(g[r * t.ldg + c])); });
  return s;
}

template <typename TAB>
__global__ __launch_bounds__(kNT) void sumsq_kernel(TAB tab, uint32_t units, int64_t u,
                                                    double *__restrict__ part) {
  __shared__ double red[kNT / 64];
  const uint32_t unit = static_cast<uint32_t>(group_number());
  if (unit >= units) return;
  ClipTensor t;
  const Unit x = unit_at(tab, unit, u, t);
  double s = t.f32 ? unit_sumsq<float>(t, x) : unit_sumsq<bf16_t>(t, x);
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kNT / 64; ++i) s += red[i];
    part[unit] = s;
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
  each_piece<E, kClipBatch>(
      x, [&](int64_t r, int64_t c) { return load_piece<T, true>(g + r * t.ldg + c); },
      [&](int64_t r, int64_t c, u32x4 p) {
        float v[E];
        Piece<T>::unpack(p, v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= f;
        store_piece<T, true>(o + r * t.ldo + c, Piece<T>::pack(v));
      },
      [&](int64_t r, int64_t c) { o[r * t.ldo + c] = from_f32<T>(to_f32(g[r * t.ldg + c]) * f); });
}

// The units in the opposite order of the norm's: of the gradients the last ones that
// it read are still in the Infinity Cache, and the products are stored past it.
template <typename TAB>
__global__ __launch_bounds__(kNT) void clip_kernel(TAB tab, uint32_t units, int64_t u, int in_place,
                                                   const double *__restrict__ sumsq,
                                                   double max_norm, float *__restrict__ norm_out) {
  const uint32_t group = static_cast<uint32_t>(group_number());
  if (group >= units) return;
  const double norm = sqrt(*sumsq);
  // a NaN norm fails the comparison and makes the factor a NaN
  const float f = norm <= max_norm ? 1.0f : static_cast<float>(max_norm / norm);
  if (norm_out && group == 0 && threadIdx.x == 0) *norm_out = static_cast<float>(norm);
  if (tab.n == 0 || (in_place && f == 1.0f)) return;  // every value is its own product
  ClipTensor t;
  const Unit x = unit_at(tab, units - 1 - group, u, t);
  if (t.f32)
    unit_scale<float>(t, x, f);
  else
    unit_scale<bf16_t>(t, x, f);
}

void enter(ClipTable &tab, const ClipTensor &t, int64_t u) {
  ClipTensor &e = tab.t[tab.n];
  e = t;
  e.per_row = static_cast<uint32_t>(ceil_div(t.cols, u));
  e.rows_each = static_cast<uint32_t>(t.cols < u ? u / t.cols : 1);
}
void enter(FlatTable &tab, const ClipTensor &t, int64_t) {
  tab.t[tab.n] = {t.g, t.out, 2 * t.cols + t.f32};
}

// Tables of the tensors: launch(table, units), the last tables first with `back` (the
// tables are the same).
template <typename TAB, typename F>
hipError_t each_table(const ClipTensor *t, int32_t count, int64_t u, bool back, F &&launch) {
  const int32_t tables = static_cast<int32_t>(ceil_div(count, TAB::kTensors));
  for (int32_t b = 0; b < tables; ++b) {
    const int32_t i0 = (back ? tables - 1 - b : b) * TAB::kTensors;
    TAB tab;
    std::memset(tab.unit0, 0xFF, sizeof(tab.unit0));
    int64_t units = 0;
    for (int32_t i = i0; i < count && tab.n < TAB::kTensors; ++i) {
      enter(tab, t[i], u);
      tab.unit0[tab.n++] = static_cast<uint32_t>(units);
      units += units_of(t[i], u);
    }
    launch(tab, static_cast<uint32_t>(units));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename F>
hipError_t each_table(const ClipTensor *t, int32_t count, int64_t u, bool back, F &&launch) {
  const bool flat = std::all_of(t, t + count, [](const ClipTensor &x) { return x.rows == 1; });
  return flat ? each_table<FlatTable>(t, count, u, back, launch)
              : each_table<ClipTable>(t, count, u, back, launch);
}

int64_t total_elems(const ClipTensor *t, int32_t count) {
  int64_t n = 0;
  for (int32_t i = 0; i < count; ++i) n += t[i].rows * t[i].cols;
  return n;
}

}  // namespace

int64_t clip_units(const ClipTensor *t, int32_t count) {
  const int64_t u = sum_unit(total_elems(t, count));
  int64_t n = 0;
  for (int32_t i = 0; i < count; ++i) n += units_of(t[i], u);
  return n;
}

hipError_t launch_sumsq(const ClipTensor *t, int32_t count, double *sumsq, void *ws,
                        hipStream_t s) {
  const int64_t u = sum_unit(total_elems(t, count));
  double *part = static_cast<double *>(ws);
  int64_t n = 0;
  const hipError_t e = each_table(t, count, u, false, [&](const auto &tab, uint32_t units) {
    sumsq_kernel<<<groups_grid(units), kNT, 0, s>>>(tab, units, u, part + n);
    n += units;
  });
  if (e != hipSuccess) return e;
  sumsq_total_kernel<<<1, 1024, 0, s>>>(part, n, sumsq);
  return hipGetLastError();
}

hipError_t launch_clip(const ClipTensor *t, int32_t count, bool in_place, const double *sumsq,
                       double max_norm, float *norm, hipStream_t s) {
  const int64_t u = clip_unit(total_elems(t, count));
  bool told = norm == nullptr;
  const hipError_t e = each_table(t, count, u, true, [&](const auto &tab, uint32_t units) {
    clip_kernel<<<groups_grid(units), kNT, 0, s>>>(tab, units, u, in_place, sumsq, max_norm,
                                                   told ? nullptr : norm);
    told = true;
  });
  if (e != hipSuccess || told) return e;
  clip_kernel<<<1, kNT, 0, s>>>(FlatTable(), 1, u, in_place, sumsq, max_norm, norm);  // nothing to scale
  return hipGetLastError();
}

}  // namespace sn
