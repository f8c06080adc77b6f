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
// tiles come straight to the LDS (16 bytes a lane, no registers), into DEPTH places in turn.
// A step is two halves of 32 k values.  While a half is multiplied, the next one's
// operands are read, each register as its last product has been started; between the
// halves the step that follows has landed, the present one's place is read out, and a
// later step (with two places, the one after the next) is sent for into it.  One barrier a
// step.  A tile's 16-byte pieces are permuted so that the reads of an operand touch every
// LDS bank:
//   KC    64 k values are 8 pieces of a row; piece p of row r lies at p ^ (r / 2 % 8)
//   else  a k's row is R / 16 chunks of 16 values; chunk c of row k lies at c ^ mm_key(k),
//         and ds_read_b64_tr_b16 turns 4 k x 16 values into 4 k values of a lane
// (ds_read_b128 serves lanes 0-3, 12-15 and 20-27 of a wave's half at a time, b64 32 lanes.
// KC rows of 32 k values, 64 bytes, took a third longer: half lines from the L2.)
// What it reaches: 8192 x 8192 x 8192 in bf16 1110 TFLOP/s in all layouts with tiles of
// 256 x 256 and 1015 with 128 x 128, where the library has 1285 on the same card.  The loads to
// the LDS and the card's power bound it: 1461 with operands of zeros, 1992 with those and no
// loads.  Tried and slower: 32 k values a step in four places, products of 32 x 32, waves of
// other priority, rows of 2, 8 or 16 tiles, four waves to 256 x 256.
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
  int64_t batch;               // bytes from a matrix's segment to the next matrix's
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

// The 16 bytes at src (per lane) to LDS address dst + 16 * lane, dst the same in the wave.  In
// assembly, as the compiler would wait for every such load before the first transposed
// read after it (22 percent of the time of an 8192 x 8192 x 8192 product); it has no output
// register, and the tile loop waits for it.
// (The compiler keeps m0 for itself and warns of its name among the clobbered: it must not place this
// between its own write of m0 and what that is for.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_load_16(const void *src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(src)
               : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char *)(p)));
}

// Where the chunks of k's row lie in a tile of R values a row: rows k, k + 1, .. k + 3 and
// k + 8, .. k + 11 are read together.
template <int R>
__device__ __forceinline__ int mm_key(int k) {
  return R >= 128 ? (k & 3) | (k >> 1 & 4) : R == 64 ? (k >> 1 & 1) | (k >> 2 & 2) : 0;
}

// This thread's share of an operand's tile: L loads of 16 bytes a step.
// PAIR: of every PAIR tile columns the first half come from the operand and the second
// half, the same columns, from its twin: column v of the tile is column
// v / PAIR * (PAIR / 2) + v % (PAIR / 2) of one or the other.
template <bool KC, int R, int WAVES, int PAIR = 0>
struct MmLoader {
  static constexpr int L = R / 8 / WAVES;
  static_assert(L >= 1 && R % (8 * WAVES) == 0 && WAVES >= 4, "a step is whole loads of every wave");
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
        constexpr int S = R / 8;
        const int kr = idx / S, slot = idx % S;
        int v = (((slot >> 1) ^ mm_key<R>(kr)) << 4) | ((slot & 1) << 3);
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
  // Loads a step of which `left` k values are there into lds (this operand's tile) and
  // moves on.
  template <bool WHOLE>
  __device__ __forceinline__ void load(uint32_t lds, int64_t left, int wave) {
#pragma unroll
    for (int j = 0; j < L; ++j)
      lds_load_16(WHOLE || klane + j * KROW < left ? static_cast<const void *>(p[j]) : &mm_zeros,
                  lds + (j * WAVES + wave) * 1024);
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
  int off[2];  // KC: of a step's halves; else: of k % 8 < 4 and >= 4
  __device__ __forceinline__ void init(int first, int lane) {
    const int g = lane >> 4, n = lane & 15;
    if constexpr (KC) {
      off[0] = (first + n) * 128 + ((g ^ ((n >> 1) & 7)) << 4);
      off[1] = off[0] ^ 64;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kr = 8 * g + 4 * h + (n >> 2);
        off[h] = kr * R * 2 + (((first >> 4) ^ mm_key<R>(kr)) << 5) + (n & 3) * 8;
      }
    }
  }
  // fragment `tile` (16 rows each) of half h of the step in lds
  __device__ __forceinline__ u32x4 read(const char *lds, int tile, int h) const {
    if constexpr (KC) {
      return *reinterpret_cast<const u32x4 *>(lds + off[h] + tile * 2048);
    } else {
      u32x2 v[2];
#pragma unroll
      for (int q4 = 0; q4 < 2; ++q4) {
        const char *q = lds + (off[q4] ^ (tile << 5)) + h * 32 * R * 2;
        v[q4] = __builtin_bit_cast(
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
// DEPTH: steps in the LDS.
template <bool F16_, bool AK_, bool BK_, int BM_, int BN_, int WM_, int WN_, int DEPTH_ = 2,
          bool PAIRED_ = false>
struct MmShape {
  static constexpr bool F16 = F16_, AK = AK_, BK = BK_;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, DEPTH = DEPTH_;
  static constexpr int WAVES = WM * WN, NT = WAVES * 64;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // fragments of a wave
  static constexpr int PAIR = PAIRED_ ? BN / WN : 0;
  static constexpr int kTileBytes = (BM + BN) * kMmK * 2, kLds = DEPTH * kTileBytes;
  static constexpr int kLoads = (BM + BN) / 8 / WAVES;  // of a lane and step
};

// Steps over all segments.
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
  constexpr int kB = S::BM * kMmK * 2;  // B's tile of a step lies behind A's
  const uint32_t place = __builtin_amdgcn_readfirstlane(lds_address(lds));
  const auto load = [&](uint32_t to) {
    if (left >= kMmK) {
      la.template load<true>(to, left, wave);
      lb.template load<true>(to + kB, left, wave);
    } else {
      la.template load<false>(to, left, wave);
      lb.template load<false>(to + kB, left, wave);
    }
    left -= kMmK;
    if (left <= 0 && seg + 1 < m.segs) {
      la.move((m.a.p[seg + 1] - m.a.p[seg]) * 2 - steps * la.step);
      lb.move((m.b.p[seg + 1] - m.b.p[seg]) * 2 - steps * lb.step);
      ++seg;
      left = m.k;
    }
  };
  u32x4 fa[S::TM], fb[2][S::TN];
  // With more than two places, steps past the last are loaded as zeros, so that as many loads
  // are on their way as ever.
  constexpr bool kAlways = S::DEPTH > 2;
  load(place);
#pragma unroll
  for (int d = 1; d < S::DEPTH; ++d)
    if (kAlways || t0 + d < t1) load(place + d * S::kTileBytes);
  if (kAlways || t0 + 1 < t1)
    wait_vmcnt<(S::DEPTH - 1) * S::kLoads>();
  else
    wait_vmcnt<0>();
  lds_barrier();
#pragma unroll
  for (int j = 0; j < S::TN; ++j) fb[0][j] = rb.read(lds + kB, j, 0);
#pragma unroll
  for (int i = 0; i < S::TM; ++i) fa[i] = ra.read(lds, i, 0);
  // the products of half h; meanwhile the operands of half `to` from buf
  const auto half = [&](const char *buf, int h, int to) {
#pragma unroll
    for (int j = 0; j < S::TN; ++j) fb[to][j] = rb.read(buf + kB, j, to);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
#pragma unroll
      for (int j = 0; j < S::TN; ++j) acc[i][j] = mm_mfma<S::F16>(fb[h][j], fa[i], acc[i][j]);
      fa[i] = ra.read(buf, i, to);
    }
    // A's reads each behind the products that it is free after, B's behind the first
    constexpr int RA = S::AK ? 1 : 2, RB = S::BK ? 1 : 2;
    __builtin_amdgcn_sched_group_barrier(0x008, S::TN, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, RA + S::TN * RB, 0);
#pragma unroll
    for (int i = 1; i < S::TM; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, S::TN, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, RA, 0);
    }
  };
  int64_t t = t0;
  uint32_t cur = 0;  // where the present step lies
#pragma unroll 1
  for (int r = 0; r < 3; ++r) {
    const int64_t end = r < 2 && m.run[r] * steps < t1 ? m.run[r] * steps : t1;
    if (r && m.run[r - 1] < m.segs) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] *= m.factor;
    }
#pragma unroll 1
    for (; t < end; ++t) {
      half(lds + cur, 0, 1);
      wait_vmcnt<(S::DEPTH - 2) * S::kLoads>();  // the next step's loads
      lds_barrier();
      if (kAlways || t + S::DEPTH < t1) load(place + cur);
      cur = cur + S::kTileBytes == S::kLds ? 0 : cur + S::kTileBytes;
      half(lds + cur, 1, 0);  // behind the last step, operands that nothing uses
    }
  }
  if (kAlways) wait_vmcnt<0>();  // the LDS is another workgroup's when this one ends
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

// Four values of a row from p on, of which `left` lie in it; at any alignment.
typedef uint32_t quad_b16 __attribute__((ext_vector_type(2), aligned(2)));
typedef float quad_b32 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
__device__ __forceinline__ void put4(T *p, int64_t left, f32x4 v) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<quad_b16 *>(p) = quad_b16{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
    else
      *reinterpret_cast<quad_b32 *>(p) = quad_b32{v.x, v.y, v.z, v.w};
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) p[e] = from_f32<T>(v[e]);
  }
}
template <typename T>
__device__ __forceinline__ f32x4 get4(const T *p, int64_t left) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 2) {
      const quad_b16 w = *reinterpret_cast<const quad_b16 *>(p);
      return f32x4{bf_lo(w.x), bf_hi(w.x), bf_lo(w.y), bf_hi(w.y)};
    } else {
      const quad_b32 w = *reinterpret_cast<const quad_b32 *>(p);
      return f32x4{w.x, w.y, w.z, w.w};
    }
  }
  f32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < left) v[e] = to_f32(p[e]);
  return v;
}

// The workgroups of a product: `mats` matrices of gm x gn tiles, or the tiles on and below
// the diagonal of gm x gm.  The first `whole` tiles have a workgroup each; the `rest`, too few
// to keep every CU busy, are cut into `splits` runs of steps, whose sums go to `part` as the
// threads hold them and are added, in order, by mm_finish_kernel.  All tiles are cut alike: with
// the steps shared out evenly, across tiles, neighbours were at different k and shared nothing
// (two 1600 x 4267 float32 updates 1929 us, 1701 so).
struct MmGrid {
  int64_t gm, gn, mats;
  bool sym;
  int64_t whole, rest;
  int splits;
  float *part;
};
struct MmPlace {
  int64_t z, tm, tn;
};
__device__ __forceinline__ MmPlace mm_where(const MmGrid &g, int64_t tile) {
  MmPlace p;
  if (g.sym) {
    const int64_t each = g.gm * (g.gm + 1) / 2;
    p.z = tile / each;
    const int64_t k = tile - p.z * each;
    p.tm = static_cast<int64_t>((sqrtf(8.0f * static_cast<float>(k) + 1.0f) - 1.0f) * 0.5f);
    while (p.tm * (p.tm + 1) / 2 > k) --p.tm;
    while ((p.tm + 1) * (p.tm + 2) / 2 <= k) ++p.tm;
    p.tn = k - p.tm * (p.tm + 1) / 2;
  } else {
    const int64_t each = g.gm * g.gn;
    p.z = tile / each;
    mm_place(tile - p.z * each, g.gm, g.gn, p.tm, p.tn);
  }
  return p;
}
// A row of fragments to the epilogue: e.row<S>(place, row, column of this lane's first sum of
// the first fragment, sums); fragment j lies 16 j columns on (paired: the twin's sums in the
// second half of the fragments).
template <class S, class Epi>
__device__ __forceinline__ void mm_row(const Epi &e, const MmPlace &p, int i, f32x4 (&acc)[S::TN]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int C = S::PAIR ? 2 : 1;
  const int64_t row = p.tm * S::BM + wave / S::WN * (S::BM / S::WM) + i * 16 + (lane & 15);
  const int64_t col = p.tn * (S::BN / C) + wave % S::WN * (S::BN / S::WN / C) + 4 * (lane >> 4);
  e.template row<S>(p, row, col, acc);
}

template <class S, class Epi>
__global__ __launch_bounds__(S::NT, S::NT / 256) void mm_kernel(MmArgs m, MmGrid g, Epi e) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int64_t id = static_cast<int64_t>(blockIdx.y) * (1 << 20) + blockIdx.x;
  if (id >= g.whole + g.rest * g.splits) return;
  const int64_t steps = mm_steps(m);
  int64_t tile, t0 = 0, t1 = steps, split = 0;
  if (id < g.whole) {
    tile = mm_order(id, g.whole);
  } else {
    const int64_t o = mm_order(id - g.whole, g.rest * g.splits);
    split = o / g.rest;
    tile = g.whole + o - split * g.rest;
    t0 = split * steps / g.splits;
    t1 = (split + 1) * steps / g.splits;
  }
  const MmPlace p = mm_where(g, tile);
  f32x4 acc[S::TM][S::TN];
  mm_tile<S>(m, p.tm * S::BM, p.tn * (S::PAIR ? S::BN / 2 : S::BN), t0, t1, lds, acc,
             p.z * m.a.batch, p.z * m.b.batch);
  if (id < g.whole || g.splits == 1) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i) mm_row<S>(e, p, i, acc[i]);
  } else {
    f32x4 *to = reinterpret_cast<f32x4 *>(g.part) +
                ((tile - g.whole) * g.splits + split) * (S::TM * S::TN * S::NT) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j) to[(i * S::TN + j) * S::NT] = acc[i][j];
  }
}
// A workgroup for each row of fragments of the cut tiles.
template <class S, class Epi>
__global__ __launch_bounds__(S::NT) void mm_finish_kernel(MmGrid g, Epi e) {
  const int64_t id = static_cast<int64_t>(blockIdx.y) * (1 << 20) + blockIdx.x;
  if (id >= g.rest * S::TM) return;
  const int64_t tile = id / S::TM;
  const int i = static_cast<int>(id - tile * S::TM);
  const f32x4 *from = reinterpret_cast<const f32x4 *>(g.part) +
                      (tile * g.splits * S::TM + i) * (S::TN * S::NT) + threadIdx.x;
  f32x4 acc[S::TN];
#pragma unroll
  for (int j = 0; j < S::TN; ++j) acc[j] = f32x4{0, 0, 0, 0};
  for (int s = 0; s < g.splits; ++s, from += S::TM * S::TN * S::NT)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[j] += from[j * S::NT];
  const MmPlace p = mm_where(g, g.whole + tile);
  mm_row<S>(e, p, i, acc);
}

inline dim3 mm_groups(int64_t n) {
  return dim3(static_cast<unsigned>(n < (1 << 20) ? n : 1 << 20),
              static_cast<unsigned>(ceil_div(n, 1 << 20)));
}
template <class S, class Epi>
void mm_launch(const MmArgs &m, const MmGrid &g, const Epi &e, hipStream_t s) {
  mm_kernel<S, Epi><<<mm_groups(g.whole + g.rest * g.splits), S::NT, 0, s>>>(m, g, e);
  if (g.splits > 1) mm_finish_kernel<S, Epi><<<mm_groups(g.rest * S::TM), S::NT, 0, s>>>(g, e);
}

// How a product of M x N sums over `steps` steps is cut (N: both twins' columns where they are
// paired): the tile and the splits of the shortest time by this model, in us.  A step of a tile
// takes what the kernels measured on full CUs; a CU holds one workgroup of 256 x 256, two of
// 128 x 128 or 64 x 64; the parts are written and read at 6 TB/s, and adding them takes a launch.
struct MmPlan {
  int size;
  MmGrid grid;
  size_t part_bytes;
};
inline MmPlan mm_plan(int64_t M, int64_t N, int64_t mats, int64_t steps, bool sym = false) {
  struct Kind {
    int size, per_cu;
    double step;
  };
  const Kind kinds[3] = {{256, 1, 1.93}, {128, 2, 1.06}, {64, 2, 0.45}};
  MmPlan best = {};
  double least = 0.0;
  for (const Kind &k : kinds) {
    MmGrid g = {};
    g.gm = ceil_div(M, k.size);
    g.gn = ceil_div(N, k.size);
    g.mats = mats;
    g.sym = sym;
    const int64_t tiles = (sym ? g.gm * (g.gm + 1) / 2 : g.gm * g.gn) * mats, slots = 256 * k.per_cu;
    for (int s = 1; s <= 16; ++s) {
      g.splits = s;
      if (s > 1 && steps / s < 4) break;
      const int64_t rounds = tiles / slots;
      g.whole = s == 1 ? tiles : rounds * slots;
      g.rest = tiles - g.whole;
      if (s > 1 && (g.rest == 0 || g.rest * s > 2 * slots)) break;
      const double tile = k.step * static_cast<double>(steps) + 3.0;
      double us = static_cast<double>(s == 1 ? ceil_div(tiles, slots) : rounds) * tile;
      const double bytes = static_cast<double>(g.rest) * s * k.size * k.size * sizeof(float);
      if (s > 1)
        us += static_cast<double>(ceil_div(g.rest * s, slots)) *
                  (k.step * static_cast<double>(ceil_div(steps, s)) + 3.0) + 4.0 + 2.0 * bytes / 6e6;
      if (least > 0.0 && us >= least) continue;
      least = us;
      best.size = k.size;
      best.grid = g;
      best.part_bytes = s > 1 ? static_cast<size_t>(bytes) : 0;
    }
  }
  return best;
}

}  // namespace sn
