// From a projection's rows to heads: split, normalised, rotated, and written where attention and the cache want them, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * w                       of each Q and K head, where weights are given
//   (a, b) -> amp (a cos t - b sin t, b cos t + a sin t)    of its first `rot` columns in pairs, t = position * freq[pair]
//
// Bound by memory: every element is read once from HBM and written once (K and V twice where they go to the cache, too).  A workgroup
// takes a few tokens and some or all of their heads.  It forms the sines and cosines of its tokens once, in LDS; G lanes share a head, a lane
// keeps its columns, and the other half of a pair that is not in its own piece is loaded a second time (from L1).
//
// Angles: a position is a whole number, and only the fraction of a turn counts.  freq / 2 pi is taken modulo one turn as a 64-bit
// fixed-point number, whose product with the position wraps by itself: the angle is off by 2^-52 of itself, as freq is, at any position, where
// a binary32 product would be off by a turn at 10^7.
#include <type_traits>

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
  int32_t S, Hq, Hkv, D, half, n_tokens, tokens, heads, n_slots, ps, begin;   // tokens and heads of a workgroup; begin: its first token's number / tokens
  Divider by_s, by_ps, by_tokens, by_half;
  float eps, amp;
  int32_t interleaved;
};

constexpr int kRotateTokens = 16;    // most tokens of a workgroup
constexpr int kRotateAngles = 512;   // and angles (one token may have 128)

template <typename T, int VEC>
struct RotateVec {
  T v[VEC];
};
template <typename T, int VEC>
__device__ __forceinline__ void rotate_load(float (&x)[VEC], const T* p) {
  if constexpr (VEC * sizeof(T) == 16) {
    const auto r = __builtin_bit_cast(RotateVec<T, VEC>, *reinterpret_cast<const u32x4*>(p));
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)r.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (float)p[i];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void rotate_store(T* p, const float (&x)[VEC]) {
  if constexpr (VEC * sizeof(T) == 16) {
    RotateVec<T, VEC> r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = (T)x[i];   // results are rounded once, to nearest even
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = (T)x[i];
  }
}

// VEC: columns of a piece (16 bytes, or 1 where a row or a pair's other half is no whole number of those); G lanes a head; NP pieces a lane.
template <typename T, int VEC, int G, int NP>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  constexpr int RPP = kThreads / G;   // heads that the workgroup deals with at once
  __shared__ float2 turn[kRotateAngles];
  __shared__ int64_t in_at[kRotateTokens], page_at[kRotateTokens], out_b[kRotateTokens];   // out_b: the item's number, -1: nothing to do
  __shared__ int out_s[kRotateTokens];
  const int tid = threadIdx.x, lane = tid % G, sub = tid / G, D = a.D, half = a.half;
  const int t0 = (a.begin + blockIdx.x) * a.tokens, n = min(a.tokens, a.n_tokens - t0);
  const int h0 = blockIdx.y * a.heads, nh = min(a.heads, a.Hq + 2 * a.Hkv - h0);
  if (tid < n) {
    const int b = a.by_s.div(t0 + tid), s = t0 + tid - b * a.S;
    const bool real = a.pos[t0 + tid] >= 0;
    out_b[tid] = real ? b : -1;
    out_s[tid] = s;
    in_at[tid] = b * a.batch_stride + s * a.row_stride;
    int64_t at = -1;
    if (real && a.slot) {
      const int slot = a.slot[t0 + tid];
      if ((unsigned)slot < (unsigned)a.n_slots) {
        const int page = a.by_ps.div(slot);
        at = page * a.page_stride + (int64_t)(slot - page * a.ps) * D;
      }
    }
    page_at[tid] = at;
  }
  if (h0 < a.Hq + a.Hkv)
    for (int i = tid; i < n * half; i += kThreads) {
      const int t = a.by_half.div(i);
      double f = a.freq[i - t * half] * 0.15915494309189533577;
      f -= floor(f);
      const uint64_t step = (uint64_t)(f * 18446744073709551616.0);
      const int32_t frac = (int32_t)((step * (uint64_t)(uint32_t)max(a.pos[t0 + t], 0)) >> 32);   // of a turn, from -1/2 on
      float s, c;
      sincospif((float)frac * 4.656612873077392578125e-10f, &s, &c);   // 2^-31: half turns
      turn[i] = make_float2(c * a.amp, s * a.amp);
    }
  __syncthreads();
  const int rows = nh * n;
  const T* X = static_cast<const T*>(a.X);
  for (int r = sub; r < rows; r += RPP) {   // (token fastest: rows of one head and neighbouring tokens lie side by side in the outputs)
    const int hh = n == a.tokens ? a.by_tokens.div(r) : r / n, t = r - hh * n, h = h0 + hh;
    const int64_t b = out_b[t];
    if (b < 0) continue;   // (all lanes of the head)
    const T* x = X + in_at[t] + (int64_t)h * D;
    const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
    const float* w = kind == 0 ? a.qw : kind == 1 ? a.kw : nullptr;
    float y[NP][VEC], z[NP][VEC];   // a piece, and for pairs across halves the other one's
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = VEC * (lane + G * i);
#pragma unroll
      for (int e = 0; e < VEC; ++e) y[i][e] = z[i][e] = 0.f;
      if (c < D) {
        rotate_load<T, VEC>(y[i], x + c);
        if (kind < 2 && c < 2 * half) {
          if (!a.interleaved) rotate_load<T, VEC>(z[i], x + (c < half ? c + half : c - half));
          else if (VEC == 1) rotate_load<T, VEC>(z[i], x + (c ^ 1));
        }
      }
    }
    if (w) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum = fmaf(y[i][e], y[i][e], sum);
#pragma unroll
      for (int off = G / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      const float inv = 1.f / sqrtf(sum / (float)D + a.eps);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = VEC * (lane + G * i);
        if (c >= D) continue;
        const int o = a.interleaved ? c ^ 1 : c < half ? c + half : c - half;   // (read only where it is a pair's other half)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          y[i][e] *= inv * w[c + e];
          if (c < 2 * half && (!a.interleaved || VEC == 1)) z[i][e] *= inv * w[o + e];
        }
      }
    }
    const float2* cs = turn + t * half;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = VEC * (lane + G * i);
      if (c >= D) continue;
      if (kind < 2 && c < 2 * half) {
        if (!a.interleaved || VEC == 1) {
          const bool first = a.interleaved ? !(c & 1) : c < half;
          const int p = a.interleaved ? c >> 1 : first ? c : c - half;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 f = cs[p + e];
            y[i][e] = first ? y[i][e] * f.x - z[i][e] * f.y : y[i][e] * f.x + z[i][e] * f.y;
          }
        } else if constexpr (VEC > 1) {
#pragma unroll
          for (int e = 0; e < VEC; e += 2)
            if (c + e < 2 * half) {
              const float2 f = cs[(c + e) >> 1];
              const float u = y[i][e], v = y[i][e + 1];
              y[i][e] = u * f.x - v * f.y;
              y[i][e + 1] = v * f.x + u * f.y;
            }
        }
      }
      const int s = out_s[t];
      if (kind == 0) {
        rotate_store<T, VEC>(static_cast<T*>(a.Q) + ((b * a.Hq + h) * a.S + s) * D + c, y[i]);
      } else {
        const int hk = h - a.Hq - (kind == 2 ? a.Hkv : 0);
        T* dense = static_cast<T*>(kind == 1 ? a.K : a.V);
        if (dense) rotate_store<T, VEC>(dense + ((b * a.Hkv + hk) * a.S + s) * D + c, y[i]);
        if (page_at[t] >= 0)
          rotate_store<T, VEC>(static_cast<T*>(kind == 1 ? a.kp : a.vp) + page_at[t] + (int64_t)hk * a.ps * D + c, y[i]);
      }
    }
  }
}

template <typename T, int VEC, int G, int NP>
static hipError_t launch_rotate_as(RotateArgs a, hipStream_t stream) {
  const int all = a.Hq + 2 * a.Hkv, RPP = kThreads / G;
  // tokens of a workgroup: as many as there are angles for 256 threads, while there are workgroups enough
  int t = a.half ? (kThreads + a.half - 1) / a.half : kRotateTokens;
  t = t < kRotateTokens ? t : kRotateTokens;
  while (t > 1 && a.n_tokens / t < 1024) t >>= 1;
  a.tokens = t;
  // heads: all of them, or what the threads deal with at once where there are few tokens
  const int64_t blocks = ((int64_t)a.n_tokens + t - 1) / t;
  a.heads = blocks >= 1024 ? all : RPP / t > 1 ? RPP / t : 1;
  a.by_tokens = Divider((uint32_t)a.tokens);
  const unsigned gy = (unsigned)((all + a.heads - 1) / a.heads);
  const int64_t most = 1 << 23;
  for (int64_t begin = 0; begin < blocks; begin += most) {
    a.begin = (int)begin;
    const int64_t wgs = blocks - begin < most ? blocks - begin : most;
    hipLaunchKernelGGL((rotate_kernel<T, VEC, G, NP>), dim3((unsigned)wgs, gy), dim3(kThreads), 0, stream, a);
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
  const int vec = p.is_f32 ? 4 : 8;
  const bool whole = p.D % vec == 0 && p.row_stride % vec == 0 && p.batch_stride % vec == 0 &&
                     (p.interleaved || a.half % vec == 0);
  if (!p.is_f32) {
    if (whole) return p.D == 64 ? launch_rotate_as<bf16_t, 8, 8, 1>(a, stream) : launch_rotate_as<bf16_t, 8, 16, 1>(a, stream);
    return p.D == 64 ? launch_rotate_as<bf16_t, 1, 64, 1>(a, stream) : launch_rotate_as<bf16_t, 1, 64, 2>(a, stream);
  }
  if (whole) {
    if (p.D <= 64) return launch_rotate_as<float, 4, 16, 1>(a, stream);
    if (p.D <= 128) return launch_rotate_as<float, 4, 32, 1>(a, stream);
    return launch_rotate_as<float, 4, 64, 1>(a, stream);
  }
  if (p.D <= 64) return launch_rotate_as<float, 1, 64, 1>(a, stream);
  if (p.D <= 128) return launch_rotate_as<float, 1, 64, 2>(a, stream);
  return launch_rotate_as<float, 1, 64, 4>(a, stream);
}

}  // namespace ac
