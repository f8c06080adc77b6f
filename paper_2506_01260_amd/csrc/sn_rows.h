// Row pieces and reductions shared by the kernels that work along rows of any
// length and alignment (gfx950 only).
#pragma once

#include "sn_device.h"

namespace sn {

// A piece: 16 bytes of a row, 8 bf16 or 4 floats, one load or store of a lane.
// Rows may start at any element (odd strides): the pointer types below promise
// the element's alignment only, and gfx950 loads and stores 16 bytes at any
// such address in one instruction.
typedef uint32_t piece_b16 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t piece_b32 __attribute__((ext_vector_type(4), aligned(4)));

template <typename T> struct Piece;

template <> struct Piece<bf16_t> {
  static constexpr int E = 8;
  typedef piece_b16 mem;
  static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[E]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf_lo(w[i]);
      x[2 * i + 1] = bf_hi(w[i]);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[E]) {
    return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                 pack_bf16x2(x[6], x[7])};
  }
};

template <> struct Piece<float> {
  static constexpr int E = 4;
  typedef piece_b32 mem;
  static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[E]) {
    const f32x4 f = __builtin_bit_cast(f32x4, v);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
  }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[E]) {
    return __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
  }
};

// NT: non-temporal, for data that nothing reads again soon.
template <typename T, bool NT = false>
__device__ __forceinline__ u32x4 load_piece(const T *p) {
  auto q = reinterpret_cast<const typename Piece<T>::mem *>(p);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  return *q;
}
template <typename T, bool NT = false>
__device__ __forceinline__ void store_piece(T *p, u32x4 v) {
  auto q = reinterpret_cast<typename Piece<T>::mem *>(p);
  if constexpr (NT)
    __builtin_nontemporal_store(static_cast<typename Piece<T>::mem>(v), q);
  else
    *q = v;
}

// The same for piece `base` + threadIdx.x of a row, base the same in all threads.
template <typename T, bool NT = false>
__device__ __forceinline__ u32x4 load_own(const T *row, int base) {
  const auto b = reinterpret_cast<const char *>(row + static_cast<int64_t>(base) * Piece<T>::E);
  return load_piece<T, NT>(reinterpret_cast<const T *>(b + 16u * threadIdx.x));
}

// Loads of rows that start at an odd element of 2 bytes.  Off a multiple of 4 bytes
// the memory pipe takes a third longer (reads of such rows were held to 4.8 TB/s,
// those at any multiple of 4 reach 5.9), so a piece is loaded from one element before
// its start, and its last element comes from the next lane's, which loaded it: in
// two steps, so that all loads are under way before the first is waited for.  The
// values and their order are those of a plain load.
struct OddPiece {
  u32x4 v;
  uint32_t last;  // the piece's last element, where no lane has it
};
template <typename T>
__device__ __forceinline__ bool is_odd(const T *row) {
  return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(row) & 2) != 0;
}
// Piece base + threadIdx.x < full of a row of at least `full` whole pieces.
template <typename T, bool NT = false>
__device__ __forceinline__ OddPiece fetch_own(const T *row, int base, int full, bool odd) {
  OddPiece r;
  r.last = 0;
  if constexpr (sizeof(T) == 2) {
    const T *at = row + static_cast<int64_t>(base) * Piece<T>::E;
    const int p = base + static_cast<int>(threadIdx.x);
    const bool early = odd && p > 0;  // never before the row
    r.v = load_piece<T, NT>(at + (static_cast<int>(threadIdx.x) * Piece<T>::E - (early ? 1 : 0)));
    if (odd && ((threadIdx.x & 63) == 63 || p + 1 >= full))
      r.last = at[threadIdx.x * Piece<T>::E + (Piece<T>::E - 1)];
  } else {
    r.v = load_own<T, NT>(row, base);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ u32x4 settle_own(const OddPiece &r, int base, int full, bool odd) {
  u32x4 v = r.v;
  if constexpr (sizeof(T) == 2) {
    if (odd) {
      // wave_shl:1, lane i from lane i + 1; a lane without a source keeps `last`
      const uint32_t next = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
          static_cast<int>(r.last), static_cast<int>(v.x), 0x130, 0xF, 0xF, false));
      const int p = base + static_cast<int>(threadIdx.x);
      const uint32_t end = (threadIdx.x & 63) == 63 || p + 1 >= full ? r.last : next;
      if (p > 0)
        v = u32x4{__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16),
                  __builtin_amdgcn_alignbit(v.w, v.z, 16), __builtin_amdgcn_alignbit(end, v.w, 16)};
    }
  }
  return v;
}
template <typename T, bool NT = false>
__device__ __forceinline__ void store_own(T *row, int base, u32x4 v) {
  const auto b = reinterpret_cast<char *>(row + static_cast<int64_t>(base) * Piece<T>::E);
  store_piece<T, NT>(reinterpret_cast<T *>(b + 16u * threadIdx.x), v);
}

// Workgroups numbered over two grid dimensions, one of which holds fewer than 2^32
// threads: one row (or part of one) each.  A loop over rows inside the kernel made
// the compiler keep the addresses and comparisons of the whole unrolled body in
// registers across it, up to 190 of them for 60.
constexpr int64_t kGridX = 1 << 20;
__device__ __forceinline__ int64_t group_number() {
  return static_cast<int64_t>(blockIdx.y) * kGridX + blockIdx.x;
}
inline dim3 groups_grid(int64_t n) {
  return dim3(static_cast<unsigned>(n < kGridX ? n : kGridX),
              static_cast<unsigned>((n + kGridX - 1) / kGridX));
}

// The elements c0 .. c0 + E - 1 of a row of n: those at or past n read as `fill`
// and are not written.
template <typename T>
__device__ __forceinline__ void load_part(const T *row, int64_t c0, int64_t n, float fill,
                                          float (&x)[Piece<T>::E]) {
#pragma unroll
  for (int i = 0; i < Piece<T>::E; ++i) x[i] = c0 + i < n ? to_f32(row[c0 + i]) : fill;
}
template <typename T>
__device__ __forceinline__ void store_part(T *row, int64_t c0, int64_t n,
                                           const float (&x)[Piece<T>::E]) {
#pragma unroll
  for (int i = 0; i < Piece<T>::E; ++i)
    if (c0 + i < n) row[c0 + i] = from_f32<T>(x[i]);
}

// ---- reductions: every lane / thread gets the result ------------------------
// Over the wave by data-parallel-primitive moves, which cost a vector instruction
// each where a shuffle is a trip to the LDS: within rows of 16 lanes, then row 0
// to 1 and 2 to 3, then the lower half to the upper; lane 63 has the total.  A
// lane without a source keeps `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t v, uint32_t none) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
      static_cast<int>(none), static_cast<int>(v), CTRL, ROWS, 0xF, false));
}
template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t none, F &&f) {
  v = f(v, dpp<0x111, 0xF>(v, none));  // row_shr:1, 2, 4, 8
  v = f(v, dpp<0x112, 0xF>(v, none));
  v = f(v, dpp<0x114, 0xF>(v, none));
  v = f(v, dpp<0x118, 0xF>(v, none));
  v = f(v, dpp<0x142, 0xA>(v, none));  // row_bcast:15 into rows 1 and 3
  v = f(v, dpp<0x143, 0xC>(v, none));  // row_bcast:31 into rows 2 and 3
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ float wave_max(float v) {
  return __uint_as_float(
      wave_reduce(__float_as_uint(v), __float_as_uint(-INFINITY), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
      }));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Sums over a workgroup of W waves; red: W floats of LDS that no thread uses
// between the caller's last barrier and the call, nor after it before the next
// barrier.  One barrier.  The waves are added in order.
template <int W>
__device__ __forceinline__ float group_sum(float v, float *red) {
  v = wave_sum(v);
  if constexpr (W == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) v += red[i];
  return v;
}

}  // namespace sn
