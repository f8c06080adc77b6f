// Token log probabilities: rows of logits z (N x V), scale c, with
//   m = max z,  x = c (z - m),  S = sum e^x,  L = log S
//   log p = x - L,  H = -sum p log p = L - (sum e^x x) / S
// for the given token's log p, the entropy H and the largest logits; the
// gradient of sum_i (gl_i log p_i[t_i] + gh_i H_i),
//   dz_j = c (gl (d_jt - p_j) - gh p_j (log p_j + H)),
// and, for a weighted loss whose weights are known beforehand, both in one call.
//
// Memory-bound, with the vector ALU close behind: a logit costs 8 instructions and an
// exponential in the forward call, 18 with two exponentials in the loss.  One
// workgroup per row, each thread with a running maximum and sums of its own that are
// rescaled where the maximum grows: one pass over the row, joined over the threads at
// its end.  All sums are float32 over at most V / 64 terms each, then in a tree.
//
// Measured: 8192 x 128256 bf16 334 us (6.3 TB/s, what reads alone reach on this
// card); 4999 x 50257 with eight alternatives 96 us (5.2); one row of 128256 11 us.
// Backward of 8192 x 32000 float32 354-367 us (5.7-5.9 TB/s read and written), loss of
// 32768 x 32000 bf16 710-750 us (5.6-5.9), 788 over its own logits.
#include <cfloat>

#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

// e^(c d) is 2^(c2 d) with c2 = c log2 e rounded to float32, one multiplication of the
// difference d: |c d| 2^-24 of the exponential more than with exp(c d), so that float32
// outputs lie up to twice as far from 64 bits (5e-8 to 9e-8 of the outputs' norm for 3e-8
// to 6e-8), below one unit of theirs.
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxTop = 64;    // SN_MAX_TOP
constexpr int kMaxParts = 16;  // of a row

// Few long rows in parts: columns of a part, and what the parts leave.
struct LogprobsParts {
  int parts;
  int64_t cols;
  float *stat;     // (m, s, t) of each part of each row
  uint64_t *keys;  // n_top of each
};
// Below any difference whose exponential is not 0, and far from overflow: a
// forbidden logit's difference (-inf) is taken as this where it is multiplied by
// its exponential 0.
constexpr float kFar = -1e30f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The running statistics of one thread.  m never falls below -FLT_MAX, so that
// z - m is no difference of infinities where every logit is -inf.
struct Running {
  float best = -INFINITY;  // largest logit seen
  float m = -FLT_MAX, s = 0.0f, t = 0.0f;  // sum e^x, sum e^x (z - m)

  template <int E, bool ENT>
  __device__ __forceinline__ void add(const float (&z)[E], float c2) {
    float top = z[0];
#pragma unroll
    for (int i = 1; i < E; ++i) top = fmaxf(top, z[i]);
    if (top > best) {
      best = top;
      const float mn = fmaxf(top, -FLT_MAX), d = fmaxf(m - mn, kFar), cr = exp2_fast(d * c2);
      if constexpr (ENT) t = cr * fmaf(s, d, t);
      s *= cr;
      m = mn;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float x = z[i] - m, e = exp2_fast(x * c2);
      s += e;  // a NaN logit, and +inf (inf - inf), leave a NaN here
      if constexpr (ENT) t = fmaf(e, fmaxf(x, kFar), t);
    }
  }
};

// One pass over a row by NT threads: thread i takes the pieces i, i + NT, ...
template <typename T, int NT, bool ENT>
__device__ __forceinline__ Running scan_row(const T *row, int64_t V, float c2) {
  constexpr int E = Piece<T>::E, U = 4;
  const int full = static_cast<int>(V / E), tid = threadIdx.x;
  const bool odd = is_odd(row);
  Running r;
  float z[E];
  int b = 0;
  for (; b + U * NT <= full; b += U * NT) {
    OddPiece v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = fetch_own(row, b + u * NT, full, odd);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Piece<T>::unpack(settle_own<T>(v[u], b + u * NT, full, odd), z);
      r.add<E, ENT>(z, c2);
    }
  }
  for (; b + tid < full; b += NT) {
    Piece<T>::unpack(settle_own<T>(fetch_own(row, b, full, odd), b, full, odd), z);
    r.add<E, ENT>(z, c2);
  }
  if (b + tid == full && V % E != 0) {  // the row's last, short piece
    load_part(row, static_cast<int64_t>(full) * E, V, -INFINITY, z);
    r.add<E, ENT>(z, c2);
  }
  return r;
}

// The threads' statistics joined over a workgroup of W waves (m and s in every
// thread, t too with ENT): over each wave, then over the waves in order.  red: 3 W
// floats of LDS.  One barrier.
template <int W, bool ENT>
__device__ __forceinline__ Running join(Running r, float *red, float c2) {
  const auto rescale = [&](float m, float &s, float &t, float to) {
    const float d = fmaxf(m - to, kFar), cr = exp2_fast(d * c2);
    if constexpr (ENT) t = cr * fmaf(s, d, t);
    s *= cr;
  };
  const float m = wave_max(r.m);
  rescale(r.m, r.s, r.t, m);
  r.m = m;
  r.s = wave_sum(r.s);
  if constexpr (ENT) r.t = wave_sum(r.t);
  if constexpr (W == 1) return r;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) {
    red[wave] = r.m;
    red[W + wave] = r.s;
    if constexpr (ENT) red[2 * W + wave] = r.t;
  }
  __syncthreads();
  // lane i of each wave takes wave i's: again a reduction over a wave
  const bool has = lane < W;
  Running g;
  if (has) {
    g.m = red[lane];
    g.s = red[W + lane];
    if constexpr (ENT) g.t = red[2 * W + lane];
  }
  return join<1, ENT>(g, red, c2);
}

// ---- the largest logits --------------------------------------------------------
// A float's bits made ascending as a whole number (-0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
// A 64-bit key orders logits by value, the lower index first among equals.
__device__ __forceinline__ uint64_t order_key(float v, uint32_t index) {
  return (static_cast<uint64_t>(ordered(v)) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) {
  return 0xFFFFFFFFu - static_cast<uint32_t>(k);
}

// Candidates a workgroup keeps for a row: little more than n of them reach the
// bound (8 n where a row is sorted), but for rows of many equal logits, which look
// twice or, where many lie above the bound too, take a pass for each value.
constexpr int kCandidates = 512;

template <int NT>
struct TopLds {
  uint32_t best[NT];  // the threads' largest logits, ordered()
  uint16_t sel[NT];   // threads that may hold one of the n largest
  uint64_t cand[kCandidates];
  uint32_t sels, cands;
};

// The largest bound that n of 64 P groups' largest logits reach (0 if fewer have
// any), built from its highest bit down to bit LOW: the same in each wave.
template <int NT, int P, int LOW>
__device__ __forceinline__ uint32_t nth_best(const uint32_t (&best)[NT], int n) {
  const int lane = threadIdx.x & 63;
  uint32_t v[P], bound = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    v[i] = best[64 * i + lane];
#pragma unroll
    for (int j = i + P; j < NT / 64; j += P) v[i] = max(v[i], best[64 * j + lane]);
  }
  for (uint32_t bit = 0x80000000u; bit >= 1u << LOW; bit >>= 1) {
    int count = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) count += __popcll(__ballot(v[i] >= (bound | bit)));
    if (count >= n) bound |= bit;
    if (count == n) break;  // exactly n reach it: no higher bound is needed
  }
  return bound;
}

__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
#pragma unroll
  for (int m = 32; m; m >>= 1) {
    const uint64_t o = __shfl_xor(static_cast<unsigned long long>(k), m);
    k = o > k ? o : k;
  }
  return k;
}

// What top_row starts from; a barrier has to follow (join has one, but for a wave).
template <typename T, int NT>
__device__ __forceinline__ void init_top(TopLds<NT> &lds, const Running &r, int64_t V) {
  // 0, below every logit's, for a thread without a piece
  lds.best[threadIdx.x] = static_cast<int64_t>(threadIdx.x) * Piece<T>::E < V ? ordered(r.best) : 0;
  if (threadIdx.x == 0) lds.sels = lds.cands = 0;
  if constexpr (NT == 64) __syncthreads();
}

// The n largest logits of a row, by the threads that scanned it: put(rank, key)
// is called once for each rank below n.  A logit below the n-th largest of the
// threads' maxima has n others above it, so only the pieces of threads whose
// maximum reaches that bound are read again, and only logits that reach it are
// candidates; each one's rank is the number of candidates above it.
template <typename T, int NT, typename F>
__device__ __forceinline__ void top_row(const T *row, int64_t V, int n, TopLds<NT> &lds, F &&put) {
  constexpr int E = Piece<T>::E;
  const uint32_t pieces = static_cast<uint32_t>((V + E - 1) / E), each = (pieces + NT - 1) / NT;
  // Groups of threads, at least four to a logit asked for: nearly as good a bound as
  // the threads' own.  A bf16 logit's order lies in the upper 16 bits.
  constexpr int LOW = sizeof(T) == 2 ? 16 : 0;
  const uint32_t bound = NT == 64 || n <= 16 ? nth_best<NT, 1, LOW>(lds.best, n)
                                             : nth_best<NT, NT == 64 ? 1 : 4, LOW>(lds.best, n);
  const uint32_t mine = lds.best[threadIdx.x];
  if (mine != 0 && mine >= bound) lds.sel[atomicAdd(&lds.sels, 1u)] = threadIdx.x;
  __syncthreads();
  const uint32_t all = lds.sels * each;
  // the candidates from `least` on, and their number: in all threads
  const auto look = [&](uint32_t least) {
    for (uint32_t q = threadIdx.x; q < all; q += NT) {
      const uint32_t k = q / each, p = lds.sel[k] + (q - k * each) * NT;
      if (p >= pieces) continue;
      const int64_t c0 = static_cast<int64_t>(p) * E;
      float z[E];
      if (c0 + E <= V)
        Piece<T>::unpack(load_piece(row + c0), z);
      else
        load_part(row, c0, V, -INFINITY, z);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c0 + e < V && ordered(z[e]) >= least) {
          const uint32_t at = atomicAdd(&lds.cands, 1u);
          if (at < kCandidates) lds.cand[at] = order_key(z[e], static_cast<uint32_t>(c0 + e));
        }
    }
    __syncthreads();
    return lds.cands;
  };
  const auto rank_all = [&](uint32_t count) {
    for (uint32_t i = threadIdx.x; i < count; i += NT) {
      const uint64_t k = lds.cand[i];
      int rank = 0;
      for (uint32_t j = 0; j < count; ++j) rank += lds.cand[j] > k;
      if (rank < n) put(rank, k);
    }
  };
  uint32_t count = look(bound);
  if (count <= kCandidates) return rank_all(count);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // the logits of one value (ordered() >> low) from index `from` on, in order of their
  // index, until there are n
  int r = 0;
  const auto fill = [&](uint32_t value, int low, int64_t from) {
    for (int64_t c = from / NT * NT + threadIdx.x; r < n && c - threadIdx.x < V; c += NT) {
      const float z = c < V ? to_f32(row[c]) : 0.0f;
      const bool hit = c < V && ordered(z) >> low == value;
      const uint64_t hits = __ballot(hit);
      __syncthreads();  // the LDS has been read
      if (lane == 0) lds.best[wave] = __popcll(hits);
      __syncthreads();
      int rank = r + __popcll(hits & ((1ull << lane) - 1));
#pragma unroll
      for (int i = 0; i < NT / 64; ++i) {
        rank += i < wave ? lds.best[i] : 0;
        r += lds.best[i];
      }
      if (hit && rank < n) put(rank, order_key(z, static_cast<uint32_t>(c)));
    }
  };
  // Many logits equal to the bound, which is -inf where few tokens are allowed: those
  // above it, then those equal to it.
  __syncthreads();
  if (threadIdx.x == 0) lds.cands = 0;
  __syncthreads();
  count = look(((bound >> LOW) + 1) << LOW);
  if (count <= kCandidates) {
    rank_all(count);
    r = static_cast<int>(count);
    return fill(bound >> LOW, LOW, 0);
  }
  // many above it too: a pass over the row for the next value, then its logits
  uint64_t last = ~0ull;
  while (r < n) {
    uint64_t k = 0;
    for (int64_t c = threadIdx.x; c < V; c += NT) {
      const uint64_t o = order_key(to_f32(row[c]), static_cast<uint32_t>(c));
      k = o < last && o > k ? o : k;
    }
    k = wave_max(k);
    __syncthreads();  // the LDS has been read
    if (lane == 0) lds.cand[wave] = k;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) k = lds.cand[i] > k ? lds.cand[i] : k;
    fill(static_cast<uint32_t>(k >> 32), 0, key_index(k));
    last = k >> 32 << 32;
  }
}

// ---- kernels ---------------------------------------------------------------------

// A row's outputs from its joined statistics: L = -inf where nothing is allowed, NaN
// where a logit is NaN or +inf.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int64_t i, const T *row,
                                          const Running &r) {
  if (threadIdx.x != 0) return;
  const float L = logf(r.s);
  if (a.logp) {
    const int32_t tok = a.tok[i];
    float lp = 0.0f;
    if (tok != -1) {
      const float z = to_f32(row[clamp_id(tok, a.V, a.err_flag, 1)]);
      lp = r.s > 0.0f ? fmaf(z - r.m, a.scale, -L) : L;
    }
    a.logp[i] = lp;
  }
  a.entropy[i] = r.s == 0.0f ? 0.0f : L - a.scale * r.t / r.s;
  a.stats[2 * i] = r.s > 0.0f ? r.m : L;
  a.stats[2 * i + 1] = L;
}
__device__ __forceinline__ void write_top(const LogprobsArgs &a, int64_t i, const Running &r,
                                          int rank, uint64_t k) {
  const float L = logf(r.s);
  const int64_t o = i * a.n_top + rank;
  a.top_logp[o] = r.s > 0.0f ? fmaf(key_value(k) - r.m, a.scale, -L) : L;
  a.top_id[o] = r.s == r.s ? static_cast<int32_t>(key_index(k)) : -1;
}

template <typename T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void logprobs_kernel(LogprobsArgs a) {
  constexpr int W = NT / 64;
  __shared__ float red[3 * W];
  __shared__ TopLds<TOP ? NT : 64> lds;
  const float c2 = a.scale * kLog2e;
  const int64_t i = group_number();
  if (i >= a.N) return;
  const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
  Running r = scan_row<T, NT, true>(row, a.V, c2);
  if constexpr (TOP) init_top<T, NT>(lds, r, a.V);
  r = join<W, true>(r, red, c2);
  write_row(a, i, row, r);
  if constexpr (TOP) {
    if (r.s == r.s)
      top_row<T, NT>(row, a.V, a.n_top, lds, [&](int rank, uint64_t k) { write_top(a, i, r, rank, k); });
    else if (threadIdx.x < a.n_top)
      write_top(a, i, r, threadIdx.x, 0);
  }
}

// Few long rows, in parts: a workgroup for each of `parts` pieces of a row leaves its
// statistics (3 floats) and its n_top largest keys, in order, in the workspace.
template <typename T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void logprobs_part_kernel(LogprobsArgs a, LogprobsParts w) {
  constexpr int W = NT / 64;
  __shared__ float red[3 * W];
  __shared__ TopLds<TOP ? NT : 64> lds;
  const float c2 = a.scale * kLog2e;
  const int64_t i = blockIdx.x / w.parts, part = blockIdx.x, c0 = (blockIdx.x % w.parts) * w.cols;
  const T *row = static_cast<const T *>(a.Z) + i * a.ldz + c0;
  const int64_t V = a.V - c0 < w.cols ? a.V - c0 : w.cols;
  Running r = scan_row<T, NT, true>(row, V, c2);
  if constexpr (TOP) {
    init_top<T, NT>(lds, r, V);
    for (int j = threadIdx.x; j < a.n_top; j += NT) w.keys[part * a.n_top + j] = 0;
  }
  r = join<W, true>(r, red, c2);
  if (threadIdx.x == 0) {
    w.stat[3 * part] = r.m;
    w.stat[3 * part + 1] = r.s;
    w.stat[3 * part + 2] = r.t;
  }
  if constexpr (TOP) {
    if (r.s == r.s)
      top_row<T, NT>(row, V, a.n_top, lds, [&](int rank, uint64_t k) {
        w.keys[part * a.n_top + rank] = k - static_cast<uint64_t>(c0);  // the row's own index
      });
  }
}

// The parts of a row joined: a key's rank is the number of keys above it (128256 bf16
// logits with 20 alternatives: 13 us, 20 by halving in the parts' lists).
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobsArgs a, LogprobsParts w) {
  __shared__ uint64_t keys[kMaxParts * kMaxTop];
  __shared__ uint32_t kept;
  const int64_t i = blockIdx.x;
  const int lane = threadIdx.x & 63, all = w.parts * a.n_top;
  const float c2 = a.scale * kLog2e;
  // Each part's list descends, so that the least of the parts' m-th keys, m parts >= n,
  // has n keys at or above it: the others need no rank.
  const uint64_t *all_keys = w.keys + i * all;
  const int m = (a.n_top + w.parts - 1) / w.parts;
  uint64_t mine = ~0ull, first = 0;
  if (a.n_top && lane < w.parts) mine = all_keys[lane * a.n_top + m - 1];
  if (threadIdx.x < all) first = all_keys[threadIdx.x];
  if (threadIdx.x == 0) kept = 0;
  Running r;
  if (lane < w.parts) {
    const float *stat = w.stat + 3 * (i * w.parts + lane);
    r.m = stat[0];
    r.s = stat[1];
    r.t = stat[2];
  }
  r = join<1, true>(r, nullptr, c2);
  write_row(a, i, static_cast<const T *>(a.Z) + i * a.ldz, r);
  if (r.s != r.s) {
    if (threadIdx.x < a.n_top) write_top(a, i, r, threadIdx.x, 0);
    return;
  }
  const uint64_t least = ~wave_max(~mine);
  __syncthreads();
  for (int j = threadIdx.x; j < all; j += 256) {
    const uint64_t k = j < 256 ? first : all_keys[j];
    if (k >= least && k != 0) keys[atomicAdd(&kept, 1u)] = k;
  }
  __syncthreads();
  const int count = static_cast<int>(kept);
  for (int j = threadIdx.x; j < count; j += 256) {
    const uint64_t k = keys[j];
    int rank = 0;
#pragma unroll 8
    for (int q = 0; q < count; ++q) rank += keys[q] > k;
    if (rank < a.n_top) write_top(a, i, r, rank, k);
  }
}

// Elements c0 .. of a row's gradient from its logits, in place of z.
//   lp = c (z - m) - L, p = e^lp:  -c p (gl + gh (lp + H))
struct RowGrad {
  float m, L, gl, gh, H, c;
  template <int E>
  __device__ __forceinline__ void apply(float (&z)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      // past e^-1e4 = 0 the factor stays finite; a row whose L is NaN has gl = NaN
      const float lp = fmaxf(fmaf(z[i] - m, c, -L), -1e4f);
      z[i] = -c * exp2_fast(lp * kLog2e) * fmaf(gh, lp + H, gl);
    }
  }
};

// A unit is kGradPieces pieces of each of NT threads in one row.
constexpr int kGradPieces = 4;

template <typename T, int NT>
__global__ __launch_bounds__(NT) void logprobs_grad_kernel(LogprobsGradArgs a, int64_t per_row,
                                                           int64_t units) {
  constexpr int E = Piece<T>::E, U = kGradPieces;
  constexpr bool ODD = sizeof(T) == 2 && NT < 256;
  const int full = static_cast<int>(a.V / E);
  const int64_t unit = group_number();
  if (unit >= units) return;
  const int64_t i = unit / per_row;
  const int base = static_cast<int>(unit - i * per_row) * (NT * U), first = base + threadIdx.x;
  const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
  T *out = static_cast<T *>(a.dZ) + i * a.lddz;
  const int32_t tok = a.tok ? a.tok[i] : -1;
  int t = -1;
  RowGrad g;
  g.gl = 0.0f;
  if (tok != -1) {
    t = static_cast<int>(clamp_id(tok, a.V, a.err_flag, 1));
    g.gl = a.g_logp ? a.g_logp[i] : 0.0f;
  }
  g.gh = a.g_entropy ? a.g_entropy[i] : 0.0f;
  const float hit = a.scale * g.gl;
  const bool none = g.gl == 0.0f && g.gh == 0.0f;  // a row that nothing flows into
  if (!none) {
    g.m = a.stats[2 * i];
    g.L = a.stats[2 * i + 1];
    g.H = g.gh != 0.0f ? a.entropy[i] : 0.0f;
    g.c = a.scale;
    if (g.L != g.L) g.gl = g.L;
  }
  const int tp = t < 0 ? -1 : t / E, te = t - tp * E;  // the given token's piece
  const bool odd = ODD && is_odd(row);
  OddPiece v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    v[u] = {u32x4{0, 0, 0, 0}, 0};
    if (!none && first + u * NT < full) {
      if constexpr (ODD) v[u] = fetch_own<T, true>(row, base + u * NT, full, odd);
      else v[u].v = load_own<T, true>(row, base + u * NT);
    }
  }
  float z[E];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int p = first + u * NT;
    if (p >= full) break;
    if (!none) {
      Piece<T>::unpack(ODD ? settle_own<T>(v[u], base + u * NT, full, odd) : v[u].v, z);
      g.apply(z);
      if (p == tp) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] += e == te ? hit : 0.0f;
      }
      v[u].v = Piece<T>::pack(z);
    }
    store_own<T, true>(out, base + u * NT, v[u].v);
  }
  // the row's last, short piece
  if (a.V % E != 0 && full >= first && full < first + NT * U && (full - first) % NT == 0) {
    const int64_t c0 = static_cast<int64_t>(full) * E;
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = 0.0f;
    if (!none) {
      load_part(row, c0, a.V, 0.0f, z);
      g.apply(z);
      if (full == tp) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] += e == te ? hit : 0.0f;
      }
    }
    store_part(out, c0, a.V, z);
  }
}

// log p of the given token and w c (p - d) in one call (of more than 32768 bf16 logits
// two registers of each thread are spilled: 8 bytes of scratch).  A thread keeps its first
// K pieces of the row in registers between the sums and the gradient; what a longer
// row has beyond them is read a second time, the last read first (the Infinity
// Cache still holds most of it).
template <typename T, int NT, int K, int WAVES>
__global__ __launch_bounds__(NT, WAVES) void loss_kernel(LossArgs a) {
  constexpr int E = Piece<T>::E, W = NT / 64;
  static_assert(K % 4 == 0, "the pieces beyond the kept ones go in fours");
  __shared__ float red[3 * W];
  const float c2 = a.scale * kLog2e;
  const int full = static_cast<int>(a.V / E), tid = threadIdx.x;
  const bool tail = a.V % E != 0 && full % NT == tid;  // holds the row's last, short piece
  const int64_t i = group_number();
  if (i >= a.N) return;
  const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
  T *out = static_cast<T *>(a.dZ) + i * a.lddz;
  const auto at = [&](int p) { return static_cast<int64_t>(p) * E; };
  const int32_t tok = a.tok[i];
  int t = -1;
  float w = 0.0f;
  if (tok != -1) {
    t = static_cast<int>(clamp_id(tok, a.V, a.err_flag, 1));
    w = a.weight ? a.weight[i] : 1.0f;
  }
  const bool odd = is_odd(row);
  u32x4 kept[K] = {};
  float z[E], last[E], m = 0.0f, f = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) last[e] = 0.0f;
  if (tok != -1) {
    const float zt = to_f32(row[t]);
    Running r;
    for (int b = K * NT; b < full; b += 4 * NT) {
      OddPiece v[4] = {};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (b + u * NT + tid < full) v[u] = fetch_own(row, b + u * NT, full, odd);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (b + u * NT + tid < full) {
          Piece<T>::unpack(settle_own<T>(v[u], b + u * NT, full, odd), z);
          r.add<E, false>(z, c2);
        }
    }
    OddPiece raw[K] = {};
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k * NT + tid < full) raw[k] = fetch_own(row, k * NT, full, odd);
    if (tail) load_part(row, at(full), a.V, -INFINITY, last);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k * NT + tid < full) {
        kept[k] = settle_own<T>(raw[k], k * NT, full, odd);
        Piece<T>::unpack(kept[k], z);
        r.add<E, false>(z, c2);
      }
    if (tail) r.add<E, false>(last, c2);
    r = join<W, false>(r, red, c2);
    m = r.m;
    const float s = r.s;
    const float L = logf(s);
    if (tid == 0) a.logp[i] = s > 0.0f ? fmaf(zt - m, a.scale, -L) : L;
    f = s == 0.0f ? 0.0f : w * a.scale / s;
  } else if (tid == 0) {
    a.logp[i] = 0.0f;
  }
  if (w == 0.0f) {
    for (int b = 0; b + tid < full; b += NT) store_own<T, true>(out, b, u32x4{0, 0, 0, 0});
#pragma unroll
    for (int e = 0; e < E; ++e) last[e] = 0.0f;
    if (tail) store_part(out, at(full), a.V, last);
  } else {
    const float hit = w * a.scale;
    const int tp = t / E, te = t - tp * E;  // the given token's piece
    const auto finish = [&](float (&x)[E], int p) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = f * exp2_fast((x[e] - m) * c2);
      if (p == tp) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] -= e == te ? hit : 0.0f;
      }
    };
    const auto write = [&](u32x4 v, int base) {
      Piece<T>::unpack(v, z);
      finish(z, base + tid);
      store_own<T, true>(out, base, Piece<T>::pack(z));
    };
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k * NT + tid < full) write(kept[k], k * NT);
    if (tail) {
      finish(last, full);
      store_part(out, at(full), a.V, last);
    }
    for (int b = (full - 1) / (4 * NT) * (4 * NT); b >= K * NT; b -= 4 * NT) {
      OddPiece v[4] = {};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (b + u * NT + tid < full) v[u] = fetch_own(row, b + u * NT, full, odd);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (b + u * NT + tid < full) write(settle_own<T>(v[u], b + u * NT, full, odd), b + u * NT);
    }
  }
}

template <typename T, int NT>
hipError_t launch_logprobs_nt(const LogprobsArgs &a, hipStream_t s) {
  if (a.n_top)
    logprobs_kernel<T, NT, true><<<groups_grid(a.N), NT, 0, s>>>(a);
  else
    logprobs_kernel<T, NT, false><<<groups_grid(a.N), NT, 0, s>>>(a);
  return hipGetLastError();
}

// Threads of a row: a wave up to 8 pieces for each lane; 256 up to 1024 pieces; 1024
// up to 512 rows (two workgroups for each CU).  Else, without alternatives, 1024 from
// 7 pieces for each on (8192 x 128256 bf16: 334 us, 353 with 512, 356 with 256), 512
// below (16384 x 32000: 205, 173, 181).  With alternatives smaller workgroups hide
// each other's selection: 512, and 256 up to 16 pieces for each (five of 8192 x
// 50264: 171 with 1024, 146, 152; of 16384 x 32000: 271, 196, 190).
template <typename T>
hipError_t launch_logprobs_t(const LogprobsArgs &a, const LogprobsParts &w, hipStream_t s) {
  if (w.parts > 1) {
    const unsigned g = static_cast<unsigned>(a.N * w.parts);
    if (a.n_top)
      logprobs_part_kernel<T, 1024, true><<<g, 1024, 0, s>>>(a, w);
    else
      logprobs_part_kernel<T, 1024, false><<<g, 1024, 0, s>>>(a, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    logprobs_join_kernel<T><<<static_cast<unsigned>(a.N), 256, 0, s>>>(a, w);
    return hipGetLastError();
  }
  const int64_t pieces = ceil_div(a.V, Piece<T>::E);
  // (a wave's 64 lanes bound up to 32 alternatives well, or any row that fits: of
  // 32768 x 1024 bf16 the first 20 take 31 us, 86 with 256 threads to a row; of 64 the
  // bound is often so low that the candidates overflow)
  if (pieces <= 512 && (a.n_top <= 32 || a.V <= kCandidates))
    return launch_logprobs_nt<T, 64>(a, s);
  if (pieces <= 1024) return launch_logprobs_nt<T, 256>(a, s);
  if (a.N <= 512 || (a.n_top == 0 && pieces >= 7 * 1024)) return launch_logprobs_nt<T, 1024>(a, s);
  if (a.n_top == 0 || pieces > 16 * 256) return launch_logprobs_nt<T, 512>(a, s);
  return launch_logprobs_nt<T, 256>(a, s);
}

// The parts of a row: of 1024 pieces or more (one for each thread), as many as give
// each CU two workgroups of 1024.  One CU alone takes 11 us for the 128256
// exponentials of a row and 13.6 with five alternatives, which pays for a second
// launch from about 8192 pieces on, and up to 64 rows.
LogprobsParts parts_of(int dt, int64_t N, int64_t V) {
  const int64_t E = dt == 0 ? 4 : 8, pieces = ceil_div(V, E);
  LogprobsParts w = {};
  w.parts = 1;
  w.cols = V;
  if (N <= 0 || N > 64 || pieces <= 8192) return w;
  int64_t parts = 512 / N < kMaxParts ? 512 / N : kMaxParts;
  parts = parts < pieces / 1024 ? parts : pieces / 1024;
  w.cols = ceil_div(pieces, parts) * E;
  w.parts = static_cast<int>(ceil_div(V, w.cols));
  return w;
}

template <typename T, int NT>
hipError_t launch_grad_nt(const LogprobsGradArgs &a, hipStream_t s) {
  const int64_t per_row = ceil_div(a.V, Piece<T>::E * NT * kGradPieces), units = per_row * a.N;
  logprobs_grad_kernel<T, NT><<<groups_grid(units), NT, 0, s>>>(a, per_row, units);
  return hipGetLastError();
}
// Short rows are one unit of fewer threads (bf16 25147 x 1024: 20 us, 36 with 256
// threads, half of them idle; 30000 x 2055: 63, 78).
template <typename T>
hipError_t launch_grad_t(const LogprobsGradArgs &a, hipStream_t s) {
  const int64_t pieces = ceil_div(a.V, Piece<T>::E);
  if (pieces <= 64 * kGradPieces) return launch_grad_nt<T, 64>(a, s);
  if (pieces <= 128 * kGradPieces) return launch_grad_nt<T, 128>(a, s);
  return launch_grad_nt<T, 256>(a, s);
}

}  // namespace

size_t logprobs_workspace_bytes(int dt, int64_t N, int64_t V, int n_top) {
  const LogprobsParts w = parts_of(dt, N, V);
  if (w.parts == 1) return 0;
  const size_t parts = static_cast<size_t>(N) * w.parts;
  return align256(parts * 3 * sizeof(float)) + align256(parts * n_top * sizeof(uint64_t));
}

hipError_t launch_logprobs(int dt, const LogprobsArgs &a, void *ws, hipStream_t s) {
  LogprobsParts w = parts_of(dt, a.N, a.V);
  w.stat = static_cast<float *>(ws);
  w.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) +
                                        align256(a.N * w.parts * 3 * sizeof(float)));
  return dt == 0 ? launch_logprobs_t<float>(a, w, s) : launch_logprobs_t<bf16_t>(a, w, s);
}

hipError_t launch_logprobs_grad(int dt, const LogprobsGradArgs &a, hipStream_t s) {
  return dt == 0 ? launch_grad_t<float>(a, s) : launch_grad_t<bf16_t>(a, s);
}

namespace {
template <typename T>
hipError_t launch_loss_t(const LossArgs &a, hipStream_t s) {
  const int64_t pieces = ceil_div(a.V, Piece<T>::E);
  if (pieces <= 256)
    loss_kernel<T, 64, 4, 6><<<groups_grid(a.N), 64, 0, s>>>(a);
  else if (pieces <= 1024)
    loss_kernel<T, 256, 4, 6><<<groups_grid(a.N), 256, 0, s>>>(a);
  else if (pieces <= 4096)
    loss_kernel<T, 512, 8, 6><<<groups_grid(a.N), 512, 0, s>>>(a);
  else
    loss_kernel<T, 1024, 8, 8><<<groups_grid(a.N), 1024, 0, s>>>(a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_loss(int dt, const LossArgs &a, hipStream_t s) {
  return dt == 0 ? launch_loss_t<float>(a, s) : launch_loss_t<bf16_t>(a, s);
}

}  // namespace sn
