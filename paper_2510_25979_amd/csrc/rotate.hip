// From a projection's rows to heads: split, normalised, rotated, and written where attention and the cache want them, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * w                       of each Q and K head, where weights are given
//   (a, b) -> amp (a cos t - b sin t, b cos t + a sin t)    of its first `rot` columns in pairs, t = position * freq[pair]
//
// Bound by memory: every element is read once from HBM and written once (K and V twice where they go to the cache, too): 32 prompts of up to 1,024 tokens,
// 48 heads of 64 (232 MB) 57 us = 4.1 TB/s on new inputs each time (38 where the same ones lie in the last-level cache), 4,000 tokens of 48 heads of 128 19.5.
// A workgroup takes a few tokens and some or all of their heads.  It forms
// the sines and cosines of its tokens once, through LDS; the other half of a pair that is not in a lane's own piece is loaded a second time (from L1).
// Few tokens are bound by latency, position -> angle -> store, 128 of one token each 5.2 us.
//
// Angles: a position is a whole number, and only the fraction of a turn counts.  freq / 2 pi is taken modulo one turn as a 64-bit
// fixed-point number, whose product with the position wraps by itself: the angle is off by 2^-52 of itself, as freq is, at any position, where
// a binary32 product would be off by a turn at 10^7.
#include "common.hpp"
#include "serve.h"

namespace ac {

struct RotateArgs {
  const void* X;
  const float *qw, *kw;
  const int32_t *pos, *slot;
  const double* freq;
  void *Q, *K, *V, *kp, *vp;
  int64_t batch_stride, row_stride, page_stride;   // elements
  int32_t S, Hq, Hkv, D, half, n_tokens, heads, n_slots, ps, begin;   // heads of a workgroup; begin: of the launch's groups of tokens
  Divider by_s, by_ps, by_half;
  float eps, amp;
  int32_t interleaved;
};

// VEC columns of a row as they lie in memory: 16 bytes, or 1 column where a row is no whole number of those.
template <typename T, int VEC>
struct RotatePiece {
  T v[VEC];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC * sizeof(T) % 16 == 0) {
      struct Words { u32x4 w[VEC * sizeof(T) / 16]; };
      *this = __builtin_bit_cast(RotatePiece, *reinterpret_cast<const Words*>(p));
    } else {
      v[0] = p[0];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (VEC * sizeof(T) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, *this), reinterpret_cast<u32x4*>(p));
    else p[0] = v[0];
  }
};

// G lanes a row, NP pieces a lane: a wave has 64 / G tokens, and a lane keeps its token and its columns, so that addresses, sines, cosines and weights are the
// lane's for all heads, of which the wave takes every fourth, U at a time.  (us, heads dealt to threads and tables of tokens in LDS / so: those prompts
// 58.2 / 57.2, from the cache 44 / 38, normalised 145 / 58; 4,000 tokens of 128 23.1 / 19.5; single tokens of 128 requests 6.2 / 5.1.)
// ODD: pairs lie apart and no whole pieces, so that their other halves are loaded one by one (of few columns, in most such models: 40 heads of 128 of which
// 20 columns turn, 2,400 tokens, 25 us; 38 with all columns one by one, 16 where pieces are whole).
template <typename T, int VEC, int G, int NP, int U, bool NORM, bool ODD>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  typedef RotatePiece<T, VEC> Piece;
  constexpr int TOKENS = kWave / G, CS = VEC > 1 ? VEC : 1;
  __shared__ float2 turn[kThreads];   // (TOKENS * half <= kThreads)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), D = a.D, half = a.half;
  const int sub = (tid & 63) / G, lane = tid % G;
  const int first = (a.begin + blockIdx.x) * TOKENS, token = min(first + sub, a.n_tokens - 1);
  const int h0 = blockIdx.y * a.heads + wave, h1 = min(blockIdx.y * a.heads + a.heads, a.Hq + 2 * a.Hkv), rotated = a.Hq + a.Hkv;
  const bool real = first + sub < a.n_tokens && a.pos[token] >= 0;
  const int b = a.by_s.div(token), s = token - b * a.S;
  const T* x = static_cast<const T*>(a.X) + b * a.batch_stride + s * a.row_stride;
  auto other = [&](int c) { return a.interleaved ? c ^ 1 : c < half ? c + half : c - half; };   // of a pair's columns
  const bool apart = !a.interleaved || VEC == 1;   // a pair's other half is not in the lane's piece
  Piece y[U][NP], z[U][NP];
  auto fetch = [&](int u, int h) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = VEC * (lane + G * i);
      if (c < D) {
        y[u][i].load(x + (int64_t)h * D + c);
        if (ODD) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) z[u][i].v[e] = h < rotated && c + e < 2 * half ? x[(int64_t)h * D + other(c + e)] : (T)0.f;
        } else if (apart && h < rotated && c < 2 * half) {
          z[u][i].load(x + (int64_t)h * D + other(c));
        }
      }
    }
  };
  // (where there are few tokens they are asked for before it is known whether they are padding)
  const bool early = gridDim.y > 1;
  if (early)
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + 4 * u < h1) fetch(u, h0 + 4 * u);
  // the weights of the lane's columns and of their pairs' other halves, of the kind of head that they were last loaded for
  RotatePiece<float, VEC> wy[NORM ? NP : 1], wz[NORM ? NP : 1];
  int weights_of = -1;
  auto weights = [&](int kind) {   // 0, 1: Q, K
    const float* w = kind == 0 ? a.qw : a.kw;
    if (!NORM || !w || weights_of == kind) return;
    weights_of = kind;
#pragma unroll
    for (int i = 0; i < (NORM ? NP : 1); ++i) {
      const int c = VEC * (lane + G * i);
      if (c < D) {
        wy[i].load(w + c);
        if (ODD) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) wz[i].v[e] = c + e < 2 * half ? w[other(c + e)] : 0.f;
        } else if (apart && c < 2 * half) {
          wz[i].load(w + other(c));
        }
      }
    }
  };
  if (h0 < rotated) weights(h0 < a.Hq ? 0 : 1);
  if (!__syncthreads_or(real)) return;   // padding
  if (real && !early)
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + 4 * u < h1) fetch(u, h0 + 4 * u);
  // one angle a thread
  if (blockIdx.y * a.heads < rotated && tid < TOKENS * half) {
    const int t = a.by_half.div(tid);
    double f = a.freq[tid - t * half] * 0.15915494309189533577;
    f -= rint(f);   // (nearest: no digit of a small negative frequency is lost to the whole turn beside it)
    const uint64_t size = (uint64_t)(fabs(f) * 18446744073709551616.0), step = f < 0 ? 0 - size : size;   // (size: up to 2^63)
    const int32_t frac = (int32_t)((step * (uint64_t)(uint32_t)max(a.pos[min(first + t, a.n_tokens - 1)], 0)) >> 32);   // of a turn, from -1/2 on
    // the nearest quarter turn is taken off while the fraction is a whole number: an eighth of a turn at most is then rounded to binary32
    const uint32_t quarter = ((uint32_t)frac + 0x20000000u) >> 30;
    float s0, c0;
    sincospif((float)(int32_t)((uint32_t)frac - (quarter << 30)) * 4.656612873077392578125e-10f, &s0, &c0);   // 2^-31: half turns
    const float sn = quarter == 0 ? s0 : quarter == 1 ? c0 : quarter == 2 ? -s0 : -c0;
    const float cn = quarter == 0 ? c0 : quarter == 1 ? -s0 : quarter == 2 ? -c0 : s0;
    turn[tid] = make_float2(cn * a.amp, sn * a.amp);
  }
  __syncthreads();
  if (!real) return;
  float2 cs[NP][CS];   // of the lane's columns; the sine's sign is the first half's
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = VEC * (lane + G * i);
    if (c < 2 * half) {
      if (ODD) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int o = other(c + e);
          cs[i][e] = make_float2(1.f, 0.f);   // (a column that does not turn)
          if (c + e < 2 * half) cs[i][e] = turn[sub * half + min(c + e, o)];
          if (c + e < o) cs[i][e].y = -cs[i][e].y;
        }
      } else if (apart) {
        const int o = other(c), pair = a.interleaved ? c >> 1 : min(c, o);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          cs[i][e] = turn[sub * half + pair + e];
          if (c < o) cs[i][e].y = -cs[i][e].y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e)
          if (c + 2 * e < 2 * half) cs[i][e] = turn[sub * half + (c >> 1) + e];
      }
    }
  }
  int64_t page = -1;
  if (a.slot) {
    const int slot = a.slot[token];
    if ((unsigned)slot < (unsigned)a.n_slots) {
      const int p = a.by_ps.div(slot);
      page = p * a.page_stride + (int64_t)(slot - p * a.ps) * D;
    }
  }
  const int64_t head = (int64_t)a.S * D, page_head = (int64_t)a.ps * D;   // elements from head to head
  T* Q = static_cast<T*>(a.Q) + (int64_t)b * a.Hq * head + (int64_t)s * D;
  const int64_t kv = (int64_t)b * a.Hkv * head + (int64_t)s * D;
  auto finish = [&](int u, int h) {   // (h, and which kind it is of, is the wave's)
    const int kind = h < a.Hq ? 0 : h < rotated ? 1 : 2, hk = h - a.Hq - (kind == 2 ? a.Hkv : 0);
    const bool weight = NORM && (kind == 0 ? a.qw : kind == 1 ? a.kw : nullptr) != nullptr;
    if (kind < 2) weights(kind);
    float inv = 1.f;
    if (weight) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (VEC * (lane + G * i) < D)
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum = fmaf((float)y[u][i].v[e], (float)y[u][i].v[e], sum);
#pragma unroll
      for (int off = G / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      inv = 1.f / sqrtf(sum / (float)D + a.eps);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = VEC * (lane + G * i);
      if (c >= D) continue;
      Piece out = y[u][i];
      if (kind < 2) {   // results are rounded once, to nearest even
        float p[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) p[e] = (float)y[u][i].v[e];
        if (weight)
#pragma unroll
          for (int e = 0; e < VEC; ++e) p[e] *= inv * wy[NORM ? i : 0].v[e];
        if (c < 2 * half) {
          if (apart) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              float q = (float)z[u][i].v[e];
              if (weight) q *= inv * wz[NORM ? i : 0].v[e];
              p[e] = p[e] * cs[i][e].x + q * cs[i][e].y;
            }
          } else if constexpr (VEC > 1) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2)
              if (c + e < 2 * half) {
                const float2 f = cs[i][e / 2];
                const float u0 = p[e], u1 = p[e + 1];
                p[e] = u0 * f.x - u1 * f.y;
                p[e + 1] = u1 * f.x + u0 * f.y;
              }
          }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) out.v[e] = (T)p[e];
      }
      if (kind == 0) {
        out.store(Q + h * head + c);
      } else {
        T* dense = static_cast<T*>(kind == 1 ? a.K : a.V);
        if (dense) out.store(dense + kv + hk * head + c);
        if (page >= 0) out.store(static_cast<T*>(kind == 1 ? a.kp : a.vp) + page + hk * page_head + c);
      }
    }
  };
  for (int h = h0; h < h1; h += 4 * U) {
    if (h != h0)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h + 4 * u < h1) fetch(u, h + 4 * u);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h + 4 * u < h1) finish(u, h + 4 * u);
  }
}

template <typename T, int VEC, int G, int NP, int U, int UN = U>   // UN: without weights
static hipError_t launch_rotate_as(RotateArgs a, hipStream_t stream) {
  constexpr int TOKENS = kWave / G;
  const int all = a.Hq + 2 * a.Hkv;
  const int64_t blocks = ((int64_t)a.n_tokens + TOKENS - 1) / TOKENS;
  // heads of a workgroup: all of them where there are many tokens, otherwise so few that there are some 2,048 workgroups
  const int64_t parts = blocks >= 2048 ? 1 : 2048 / blocks;
  int heads = (int)((all + parts - 1) / parts);
  a.heads = heads < 4 ? 4 : (heads + 3) / 4 * 4;
  const unsigned gy = (unsigned)((all + a.heads - 1) / a.heads);
  const int64_t most = 1 << 23;
  for (int64_t begin = 0; begin < blocks; begin += most) {
    a.begin = (int)begin;
    const int64_t wgs = blocks - begin < most ? blocks - begin : most;
    const bool norm = a.qw || a.kw, odd = !a.interleaved && a.half % VEC != 0;   // (VEC 1: never)
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)wgs, gy), dim3(kThreads), 0, stream, a); };
    if constexpr (VEC > 1) {
      if (odd) norm ? go(&rotate_kernel<T, VEC, G, NP, U, true, true>) : go(&rotate_kernel<T, VEC, G, NP, UN, false, true>);
    }
    if (!odd) norm ? go(&rotate_kernel<T, VEC, G, NP, U, true, false>) : go(&rotate_kernel<T, VEC, G, NP, UN, false, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_rotate(const RotateLaunch& p, hipStream_t stream) {
  RotateArgs a;
  a.X = p.X; a.qw = p.q_weight; a.kw = p.k_weight; a.pos = p.pos; a.slot = p.slot; a.freq = p.freq;
  a.Q = p.Q; a.K = p.K; a.V = p.V; a.kp = p.k_pages; a.vp = p.v_pages;
  a.batch_stride = p.batch_stride; a.row_stride = p.row_stride; a.page_stride = p.page_stride;
  a.S = p.S; a.Hq = p.Hq; a.Hkv = p.Hkv; a.D = p.D; a.half = p.rot / 2;
  a.n_tokens = p.B * p.S;
  a.n_slots = p.slot ? p.n_pages * p.page_size : 0;
  a.ps = p.slot ? p.page_size : 1;
  a.begin = 0;
  a.by_s = Divider((uint32_t)p.S);
  a.by_ps = Divider((uint32_t)a.ps);
  a.by_half = Divider((uint32_t)(a.half ? a.half : 1));
  a.eps = p.eps; a.amp = p.amplitude; a.interleaved = p.interleaved;
  if (!p.is_f32) return p.D == 64 ? launch_rotate_as<bf16_t, 8, 8, 1, 2, 3>(a, stream) : launch_rotate_as<bf16_t, 8, 16, 1, 3>(a, stream);
  if (p.D % 4 == 0) {   // (the strides are whole pieces, too)
    if (p.D <= 64) return launch_rotate_as<float, 4, 16, 1, 3>(a, stream);
    if (p.D <= 128) return launch_rotate_as<float, 4, 32, 1, 3>(a, stream);
    return launch_rotate_as<float, 4, 64, 1, 3>(a, stream);
  }
  if (p.D <= 64) return launch_rotate_as<float, 1, 64, 1, 4>(a, stream);
  if (p.D <= 128) return launch_rotate_as<float, 1, 64, 2, 4>(a, stream);
  return launch_rotate_as<float, 1, 64, 4, 2>(a, stream);
}

}  // namespace ac
