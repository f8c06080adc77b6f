// Matrix products on the matrix cores with 16-bit operands (gfx950): the tile
// loop shared by the gated feed-forward block and the orthogonalised updates.
//
//   acc[i, j] = sum over segments s, sum_k  A_s[i, k] B_s[j, k]
//
// Segments are products added up: several pairs of operands (dG Wg^T + dU Wu^T), or
// the planes that a float32 operand is held in (hi + lo, 16 bits each: hi lo + lo hi +
// hi hi).  Each operand lies with its k values contiguous (KC: rows of k, as X in X W^T)
// or with its rows contiguous (rows of the other index, one for each k, as W in X W).
//
// A workgroup holds BM x BN sums in registers and takes 64 k values a step: both
// tiles come straight to the LDS (16 bytes a lane, no registers), two steps of them,
// the next one on its way while this one is multiplied.  A tile's 16-byte pieces are
// permuted so that the reads of an operand touch every LDS bank:
//   KC    64 k values are 8 pieces of a row; piece p of row r lies at p ^ (r / 2 % 8)
//   else  a k's row is R / 16 chunks of 16 values; chunk c of row k lies at c ^ (k % 8),
//         and ds_read_b64_tr_b16 turns 4 k x 16 values into 4 k values of a lane
// MFMA 16x16x32: lane l = 16 g + n supplies k = 8 g .. 8 g + 7 of row n of either
// operand.  B is passed first, so that a lane's 4 results are 4 consecutive columns
// j = 4 g + e of the row i = n.
#pragma once

#include "sn_device.h"
#include "sn_internal.h"
#include "sn_mfma_common.h"

namespace sn {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t f16_t;  // fp16 bit pattern in memory

constexpr int kMmK = 64;  // k values of a step
constexpr int kMmSegs = 12;

// An operand: 16-byte aligned, ld a multiple of 8.  KC rows hold zeros from k up to the
// next multiple of 8.
struct MmOperand {
  const uint16_t *p[kMmSegs];  // one for each segment
  int64_t ld;                  // elements between rows (KC), or between k (else)
  int64_t n;                   // rows (KC) or values for each k (else; a multiple of 8)
  int64_t twin;                // bytes from a segment to its twin's (paired columns)
};

// Segments of split operands go from the smallest products to the largest in up to three
// runs, segments [0, run[0]), [run[0], run[1]), [run[1], segs): before each run but the
// first the sums are multiplied by `factor`, since the lower planes are stored larger by
// its inverse, as large as the first (the matrix cores take bf16 below 2^-126 as 0).
struct MmArgs {
  MmOperand a, b;
  int64_t k;  // of each segment
  int segs;
  int run[2];    // segs where there are fewer runs
  float factor;
};

// Source of the pieces past k: 16 bytes of zeros that every lane may load.
__device__ const u32x4 mm_zeros = {0, 0, 0, 0};

__device__ __forceinline__ void lds_load_16(const void *src, void *dst) {
  __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void *)(dst), 16, 0, 0);
}

// This thread's share of an operand's tile: L loads of 16 bytes a step.
// PAIR: of every PAIR tile columns the first half come from the operand and the second
// half, the same columns, from its twin: column v of the tile is column
// v / PAIR * (PAIR / 2) + v % (PAIR / 2) of one or the other.
template <bool KC, int R, int WAVES, int PAIR = 0>
struct MmLoader {
  static constexpr int L = R / 8 / WAVES;
  static_assert(L >= 1 && R % (8 * WAVES) == 0, "a step is whole loads of every wave");
  const char *p[L];
  int64_t step;  // bytes
  int klane;     // the lane's first k of a step for load 0; KROW more for each further load
  static constexpr int KROW = KC ? 0 : WAVES * 64 / (R / 8);

  // Column v of the tile (row v where KC): its place in the operand.
  __device__ __forceinline__ void init(const MmOperand &o, int64_t r0, int wave, int lane) {
    step = KC ? kMmK * 2 : kMmK * 2 * o.ld;
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int idx = (j * WAVES + wave) * 64 + lane;
      if constexpr (KC) {
        const int r = idx >> 3, kp = (idx & 7) ^ ((r >> 1) & 7);
        const int64_t row = min(r0 + r, o.n - 1);
        p[j] = reinterpret_cast<const char *>(o.p[0] + row * o.ld + kp * 8);
        klane = kp * 8;
      } else {
        constexpr int S = R / 8, MASK = R >= 128 ? 7 : R / 16 - 1;
        const int kr = idx / S, slot = idx % S;
        int v = (((slot >> 1) ^ (kr & MASK)) << 4) | ((slot & 1) << 3);
        int64_t twin = 0;
        if constexpr (PAIR > 0) {
          twin = v % PAIR >= PAIR / 2 ? o.twin : 0;
          v = v / PAIR * (PAIR / 2) + v % (PAIR / 2);
        }
        const int64_t col = min(r0 + v, o.n - 8);
        p[j] = reinterpret_cast<const char *>(o.p[0] + kr * o.ld + col) + twin;
        if (j == 0) klane = kr;
      }
    }
  }
  // Loads the step at k0 of a segment of k values into lds (this operand's tile) and
  // moves on.
  __device__ __forceinline__ void load(char *lds, int64_t left, int wave) {
    if (left >= kMmK) {
#pragma unroll
      for (int j = 0; j < L; ++j) lds_load_16(p[j], lds + (j * WAVES + wave) * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < L; ++j)
        lds_load_16(klane + j * KROW < left ? static_cast<const void *>(p[j]) : &mm_zeros,
                    lds + (j * WAVES + wave) * 1024);
    }
#pragma unroll
    for (int j = 0; j < L; ++j) p[j] += step;
  }
  __device__ __forceinline__ void move(int64_t bytes) {
#pragma unroll
    for (int j = 0; j < L; ++j) p[j] += bytes;
  }
};

// The operand's fragment of 16 rows from a tile in the LDS.
template <bool KC, int R>
struct MmReader {
  int off[2];  // KC: of the two halves of a step; else: of k % 8 < 4 and >= 4
  __device__ __forceinline__ void init(int first, int lane) {
    const int g = lane >> 4, n = lane & 15;
    if constexpr (KC) {
      const int s = (n >> 1) & 7;
      off[0] = (first + n) * 128 + ((g ^ s) << 4);
      off[1] = off[0] ^ 64;
    } else {
      constexpr int MASK = R >= 128 ? 7 : R / 16 - 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kr = 8 * g + 4 * h + (n >> 2);
        off[h] = kr * R * 2 + ((((first >> 4) ^ (kr & MASK))) << 5) + (n & 3) * 8;
      }
    }
  }
  // fragment `tile` (16 rows each), half ks of the step
  __device__ __forceinline__ u32x4 read(const char *lds, int tile, int ks) const {
    if constexpr (KC) {
      return *reinterpret_cast<const u32x4 *>(lds + off[ks] + tile * 2048);
    } else {
      u32x2 v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char *q = lds + ((off[h] ^ (tile << 5)) + ks * 32 * R * 2);
        v[h] = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4 *)(const_cast<char *>(q))));
      }
      return u32x4{v[0].x, v[0].y, v[1].x, v[1].y};
    }
  }
};

template <bool F16>
__device__ __forceinline__ f32x4 mm_mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Sizes of a kernel: BM x BN sums, WM x WN waves, the operands' layouts.
// PAIRED: every wave has columns of the operand B and the same ones of its twin.
template <bool F16_, bool AK_, bool BK_, int BM_, int BN_, int WM_, int WN_, bool PAIRED_ = false>
struct MmShape {
  static constexpr bool F16 = F16_, AK = AK_, BK = BK_;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int WAVES = WM * WN, NT = WAVES * 64;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // fragments of a wave
  static constexpr int PAIR = PAIRED_ ? BN / WN : 0;
  static constexpr int kTileBytes = (BM + BN) * kMmK * 2, kLds = 2 * kTileBytes;
};

// Steps of 64 k values over all segments.
__host__ __device__ __forceinline__ int64_t mm_steps(const MmArgs &m) {
  return (m.k + kMmK - 1) / kMmK * m.segs;
}

// The sums of the tile at row r0, column c0, over the steps t0 .. t1 - 1 (t0 < t1).
// lds: S::kLds bytes.  a_off, b_off: bytes that the operands lie behind
// their segments' addresses.
template <class S>
__device__ __forceinline__ void mm_tile(const MmArgs &m, int64_t r0, int64_t c0, int64_t t0,
                                        int64_t t1, char *lds, f32x4 (&acc)[S::TM][S::TN],
                                        int64_t a_off = 0, int64_t b_off = 0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  MmLoader<S::AK, S::BM, S::WAVES> la;
  MmLoader<S::BK, S::BN, S::WAVES, S::PAIR> lb;
  la.init(m.a, r0, wave, lane);
  lb.init(m.b, c0, wave, lane);
  MmReader<S::AK, S::BM> ra;
  MmReader<S::BK, S::BN> rb;
  ra.init(wave / S::WN * (S::BM / S::WM), lane);
  rb.init(wave % S::WN * (S::BN / S::WN), lane);
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  const int64_t steps = (m.k + kMmK - 1) / kMmK;  // of a segment
  int seg = static_cast<int>(t0 / steps);
  const int64_t done = t0 - seg * steps;
  int64_t left = m.k - done * kMmK;
  la.move((m.a.p[seg] - m.a.p[0]) * 2 + done * la.step + a_off);
  lb.move((m.b.p[seg] - m.b.p[0]) * 2 + done * lb.step + b_off);
  const auto load = [&](char *buf) {
    la.load(buf, left, wave);
    lb.load(buf + S::BM * kMmK * 2, left, wave);
    left -= kMmK;
    if (left <= 0 && seg + 1 < m.segs) {
      la.move((m.a.p[seg + 1] - m.a.p[seg]) * 2 - steps * la.step);
      lb.move((m.b.p[seg + 1] - m.b.p[seg]) * 2 - steps * lb.step);
      ++seg;
      left = m.k;
    }
  };
  load(lds);
  int cur = 0;
  int64_t t = t0;
#pragma unroll 1
  for (int r = 0; r < 3; ++r) {
    const int64_t end = r < 2 ? m.run[r] * steps : t1;
    if (r && m.run[r - 1] < m.segs) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] *= m.factor;
    }
#pragma unroll 1
    for (; t < end && t < t1; ++t, cur ^= 1) {
      const char *buf = lds + cur * S::kTileBytes;
      wait_vmcnt<0>();
      lds_barrier();
      if (t + 1 < t1) load(lds + (cur ^ 1) * S::kTileBytes);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        u32x4 fa[S::TM], fb[S::TN];
#pragma unroll
        for (int j = 0; j < S::TN; ++j) fb[j] = rb.read(buf + S::BM * kMmK * 2, j, ks);
#pragma unroll
        for (int i = 0; i < S::TM; ++i) fa[i] = ra.read(buf, i, ks);
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int j = 0; j < S::TN; ++j) acc[i][j] = mm_mfma<S::F16>(fb[j], fa[i], acc[i][j]);
      }
    }
  }
}

// Workgroup `id` of n, one for each tile: the tile's number.  Workgroups go to the eight
// XCDs in turn; each XCD gets a run of neighbouring tiles, which share operands in its L2.
__device__ __forceinline__ int64_t mm_order(int64_t id, int64_t n) {
  const int64_t q = n / 8, r = n % 8, x = id % 8;
  return x * q + (x < r ? x : r) + id / 8;
}
// Tile `t` of gm x gn: down columns of kMmGroup rows of tiles.
constexpr int kMmGroup = 4;
__device__ __forceinline__ void mm_place(int64_t t, int64_t gm, int64_t gn, int64_t &tm, int64_t &tn) {
  const int64_t per = kMmGroup * gn, g = t / per, in = t - g * per;
  const int64_t rows = gm - g * kMmGroup < kMmGroup ? gm - g * kMmGroup : kMmGroup;
  tm = g * kMmGroup + in % rows;
  tn = in / rows;
}

}  // namespace sn
