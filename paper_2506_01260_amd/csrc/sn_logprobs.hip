// Token log probabilities: rows of logits z (N x V), scale c, with
//   m = max z,  x = c (z - m),  S = sum e^x,  L = log S
//   log p = x - L,  H = -sum p log p = L - (sum e^x x) / S
// for the given token's log p, the entropy H and the largest logits; the
// gradient of sum_i (gl_i log p_i[t_i] + gh_i H_i),
//   dz_j = c (gl (d_jt - p_j) - gh p_j (log p_j + H)),
// and, for a weighted loss whose weights are known beforehand, both in one call.
//
// Memory-bound: a logit costs about a dozen vector instructions (its exponential
// four of them), less than the time of its bytes.  One workgroup per row, each
// thread with a running maximum and sums of its own that are rescaled where the
// maximum grows: one pass over the row, joined over the threads at its end.
// All sums are float32 over at most V / 64 terms each, then in a tree.
#include <cfloat>

#include "sn_internal.h"
#include "sn_rows.h"

namespace sn {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Below any difference whose exponential is not 0, and far from overflow: a
// forbidden logit's difference (-inf) is taken as this where it is multiplied by
// its exponential 0.
constexpr float kFar = -1e30f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The running statistics of one thread.  m never falls below -FLT_MAX, so that
// z - m is no difference of infinities where every logit is -inf.
struct Running {
  float best = -INFINITY;  // largest logit seen
  int64_t at = 0;          // the piece that first held it
  float m = -FLT_MAX, s = 0.0f, t = 0.0f;  // sum e^x, sum e^x (z - m)

  template <int E, bool ENT>
  __device__ __forceinline__ void add(const float (&z)[E], int64_t piece, float c2) {
    float top = z[0];
#pragma unroll
    for (int i = 1; i < E; ++i) top = fmaxf(top, z[i]);
    if (top > best) {
      best = top;
      at = piece;
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
  const int64_t full = V / E;
  Running r;
  int64_t p = threadIdx.x;
  r.at = p;
  float z[E];
  for (; p + (U - 1) * NT < full; p += U * NT) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_piece(row + (p + u * NT) * E);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Piece<T>::unpack(v[u], z);
      r.add<E, ENT>(z, p + u * NT, c2);
    }
  }
  for (; p < full; p += NT) {
    Piece<T>::unpack(load_piece(row + p * E), z);
    r.add<E, ENT>(z, p, c2);
  }
  if (p * E < V) {  // the row's last, short piece
    load_part(row, p * E, V, -INFINITY, z);
    r.add<E, ENT>(z, p, c2);
  }
  return r;
}

// ---- the largest logits --------------------------------------------------------
// A 64-bit key orders logits by value, the lower index (or piece) first among
// equals: the value's bits made ascending, then the complement of the index.
__device__ __forceinline__ uint64_t order_key(float v, uint32_t index) {
  const uint32_t b = __float_as_uint(v + 0.0f);  // -0 counts as 0
  const uint32_t o = b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
  return (static_cast<uint64_t>(o) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) {
  return 0xFFFFFFFFu - static_cast<uint32_t>(k);
}

__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int mask) {
  return __shfl_xor(static_cast<unsigned long long>(v), mask);
}
// one step of a bitonic network over the wave: lane and lane ^ j exchange
__device__ __forceinline__ uint64_t exchange(uint64_t k, int j, bool larger) {
  const uint64_t o = lane_xor(k, j);
  return (o > k) == larger ? o : k;
}
// the wave's 64 keys in descending order
__device__ __forceinline__ uint64_t sort64(uint64_t k, int lane) {
#pragma unroll
  for (int n = 2; n <= 64; n <<= 1)
#pragma unroll
    for (int j = n >> 1; j; j >>= 1) k = exchange(k, j, ((lane & j) == 0) == ((lane & n) == 0));
  return k;
}
// the 64 largest of two descending lists, descending
__device__ __forceinline__ uint64_t merge64(uint64_t a, uint64_t b, int lane) {
  const uint64_t o = lane_xor(b, 63);
  uint64_t k = o > a ? o : a;
#pragma unroll
  for (int j = 32; j; j >>= 1) k = exchange(k, j, (lane & j) == 0);
  return k;
}
// the W waves' lists merged: list[0] at the end (a barrier included)
template <int W>
__device__ __forceinline__ void merge_waves(uint64_t k, uint64_t (*list)[64], int lane, int wave) {
  list[wave][lane] = k;
  __syncthreads();
#pragma unroll
  for (int h = 1; h < W; h <<= 1) {
    if ((wave & (2 * h - 1)) == 0) {
      k = merge64(k, list[wave + h][lane], lane);
      list[wave][lane] = k;
    }
    __syncthreads();
  }
}

// The n largest logits of a row, after scan_row by the same threads.  Those of
// each thread's first largest piece are ordered first: a logit outside the n
// threads that come first is smaller than n others, so only these threads'
// pieces are read again, and of them only logits not below the n-th thread's
// largest are kept.  The keys are in list[0] at the end.
template <typename T, int NT>
__device__ __forceinline__ void top_row(const T *row, int64_t V, const Running &r, int n,
                                        uint64_t (*list)[64]) {
  constexpr int E = Piece<T>::E, W = NT / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t pieces = (V + E - 1) / E;
  uint64_t k = threadIdx.x < pieces ? order_key(r.best, static_cast<uint32_t>(r.at)) : 0;
  merge_waves<W>(sort64(k, lane), list, lane, wave);
  const uint64_t least = list[0][n - 1];
  k = 0;
  for (int j = wave; j < n; j += W) {
    const uint64_t thread = list[0][j];
    if (thread == 0) break;  // fewer threads than n have a piece
    for (int64_t p = key_index(thread) % NT + NT * (lane / E);; p += NT * (64 / E)) {
      const int64_t i = p * E + lane % E;
      uint64_t mine = 0;
      if (i < V) {
        const float v = to_f32(row[i]);
        if (order_key(v, static_cast<uint32_t>(p)) >= least)
          mine = order_key(v, static_cast<uint32_t>(i));
      }
      if (__ballot(i < V) == 0) break;
      if (__ballot(mine != 0)) k = merge64(k, sort64(mine, lane), lane);
    }
  }
  __syncthreads();  // list[0] has been read
  merge_waves<W>(k, list, lane, wave);
}

// ---- kernels ---------------------------------------------------------------------

template <typename T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void logprobs_kernel(LogprobsArgs a) {
  constexpr int W = NT / 64;
  __shared__ float red[3][W];
  __shared__ uint64_t list[TOP ? W : 1][64];
  const float c2 = a.scale * kLog2e;
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
    const Running r = scan_row<T, NT, true>(row, a.V, c2);
    const float m = group_max<W>(r.m, red[0]);
    const float d = fmaxf(r.m - m, kFar), cr = exp2_fast(d * c2);
    const float s = group_sum<W>(r.s * cr, red[1]);
    const float t = group_sum<W>(cr * fmaf(r.s, d, r.t), red[2]);
    const float L = logf(s);  // -inf: nothing is allowed; NaN: a logit is NaN or +inf
    if constexpr (TOP) top_row<T, NT>(row, a.V, r, a.n_top, list);
    if (threadIdx.x == 0) {
      if (a.logp) {
        const int32_t tok = a.tok[i];
        float lp = 0.0f;
        if (tok != -1) {
          const float z = to_f32(row[clamp_id(tok, a.V, a.err_flag, 1)]);
          lp = s > 0.0f ? fmaf(z - m, a.scale, -L) : L;
        }
        a.logp[i] = lp;
      }
      a.entropy[i] = s == 0.0f ? 0.0f : L - a.scale * t / s;
      a.stats[2 * i] = s > 0.0f ? m : L;
      a.stats[2 * i + 1] = L;
    }
    if constexpr (TOP) {
      if (threadIdx.x < a.n_top) {
        const uint64_t k = list[0][threadIdx.x];
        const int64_t o = i * a.n_top + threadIdx.x;
        a.top_logp[o] = s > 0.0f ? fmaf(key_value(k) - m, a.scale, -L) : L;
        a.top_id[o] = s != s ? -1 : static_cast<int32_t>(key_index(k));
      }
    }
    if (i + gridDim.x < a.N) __syncthreads();  // the LDS is used again
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

// A unit is kPieces pieces of each of 256 threads in one row.
constexpr int kGradPieces = 4;

template <typename T>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(LogprobsGradArgs a, int64_t per_row,
                                                            int64_t units) {
  constexpr int E = Piece<T>::E, U = kGradPieces;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t i = unit / per_row, first = (unit - i * per_row) * (256 * U) + threadIdx.x;
    const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
    T *out = static_cast<T *>(a.dZ) + i * a.lddz;
    const int32_t tok = a.tok ? a.tok[i] : -1;
    int64_t t = -1;
    RowGrad g;
    g.gl = 0.0f;
    if (tok != -1) {
      t = clamp_id(tok, a.V, a.err_flag, 1);
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
    u32x4 v[U];
    if (!none) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((first + u * 256 + 1) * E <= a.V)
          v[u] = load_piece<T, true>(row + (first + u * 256) * E);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t c0 = (first + u * 256) * E;
      if (c0 >= a.V) break;
      const bool whole = c0 + E <= a.V;
      float z[E] = {};
      if (!none) {
        if (whole)
          Piece<T>::unpack(v[u], z);
        else
          load_part(row, c0, a.V, 0.0f, z);
        g.apply(z);
        if (t >= c0 && t < c0 + E) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (t == c0 + e) z[e] += hit;
        }
      }
      if (whole)
        store_piece<T, true>(out + c0, Piece<T>::pack(z));
      else
        store_part(out, c0, a.V, z);
    }
  }
}

// log p of the given token and w c (p - d) in one call: two passes over the row.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void loss_kernel(LossArgs a) {
  constexpr int E = Piece<T>::E, W = NT / 64;
  __shared__ float red[2][W];
  const float c2 = a.scale * kLog2e;
  const int64_t full = a.V / E;
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const T *row = static_cast<const T *>(a.Z) + i * a.ldz;
    T *out = static_cast<T *>(a.dZ) + i * a.lddz;
    const int32_t tok = a.tok[i];
    int64_t t = -1;
    float w = 0.0f, m = 0.0f, f = 0.0f;
    if (tok != -1) {
      t = clamp_id(tok, a.V, a.err_flag, 1);
      w = a.weight ? a.weight[i] : 1.0f;
      const float zt = to_f32(row[t]);
      const Running r = scan_row<T, NT, false>(row, a.V, c2);
      m = group_max<W>(r.m, red[0]);
      const float s = group_sum<W>(r.s * exp2_fast(fmaxf(r.m - m, kFar) * c2), red[1]);
      const float L = logf(s);
      if (threadIdx.x == 0) a.logp[i] = s > 0.0f ? fmaf(zt - m, a.scale, -L) : L;
      f = s == 0.0f ? 0.0f : w * a.scale / s;
    } else if (threadIdx.x == 0) {
      a.logp[i] = 0.0f;
    }
    const float hit = w * a.scale;
    const bool none = w == 0.0f;
    auto finish = [&](float (&z)[E], int64_t c0) {
#pragma unroll
      for (int e = 0; e < E; ++e) z[e] = f * exp2_fast((z[e] - m) * c2);
      if (t >= c0 && t < c0 + E) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (t == c0 + e) z[e] -= hit;
      }
    };
    int64_t p = threadIdx.x;
    float z[E] = {};
    if (none) {
      for (; p < full; p += NT) store_piece<T, true>(out + p * E, u32x4{0, 0, 0, 0});
      if (p * E < a.V) store_part(out, p * E, a.V, z);
    } else {
      for (; p < full; p += NT) {
        Piece<T>::unpack(load_piece(row + p * E), z);
        finish(z, p * E);
        store_piece<T, true>(out + p * E, Piece<T>::pack(z));
      }
      if (p * E < a.V) {
        load_part(row, p * E, a.V, 0.0f, z);
        finish(z, p * E);
        store_part(out, p * E, a.V, z);
      }
    }
    if (i + gridDim.x < a.N) __syncthreads();  // the LDS is used again
  }
}

unsigned grid_of(int64_t n) { return static_cast<unsigned>(n < (1 << 20) ? n : 1 << 20); }

template <typename T>
hipError_t launch_logprobs_t(const LogprobsArgs &a, hipStream_t s) {
  if (a.n_top)
    logprobs_kernel<T, 256, true><<<grid_of(a.N), 256, 0, s>>>(a);
  else
    logprobs_kernel<T, 256, false><<<grid_of(a.N), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_grad_t(const LogprobsGradArgs &a, hipStream_t s) {
  const int64_t per_row = ceil_div(a.V, Piece<T>::E * 256 * kGradPieces), units = per_row * a.N;
  logprobs_grad_kernel<T><<<grid_of(units), 256, 0, s>>>(a, per_row, units);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_logprobs(int dt, const LogprobsArgs &a, hipStream_t s) {
  return dt == 0 ? launch_logprobs_t<float>(a, s) : launch_logprobs_t<bf16_t>(a, s);
}

hipError_t launch_logprobs_grad(int dt, const LogprobsGradArgs &a, hipStream_t s) {
  return dt == 0 ? launch_grad_t<float>(a, s) : launch_grad_t<bf16_t>(a, s);
}

hipError_t launch_loss(int dt, const LossArgs &a, hipStream_t s) {
  if (dt == 0)
    loss_kernel<float, 512><<<grid_of(a.N), 512, 0, s>>>(a);
  else
    loss_kernel<bf16_t, 512><<<grid_of(a.N), 512, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sn
