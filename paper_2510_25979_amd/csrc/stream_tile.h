// What a wave does with chunks of 64 keys that lie in LDS, for 32 rows of bf16: both products transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane
// holds scores of one row and the weights go from the first product to the second in their registers.  K rows lie swizzled by k_piece_swizzle, V
// rows by v_piece_swizzle, as the copies of the kernels that use this put them (window.hip, shared.hip).
#pragma once
#include "common.hpp"

namespace ac {

constexpr int kStreamChunk = 64;
constexpr float kStreamSlack = 8.0f;   // the reference point of a row moves when a score has outgrown it by 2^8

// Copies from memory straight into LDS by buffer loads.  (The compiler takes a global load to LDS for one that may also read LDS, and lets every
// LDS read wait for all others as long as one is under way.  A buffer load it knows: reads and products wait for what they need.)
struct StreamSource {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ StreamSource(const void* from, uint32_t bytes)   // uniform; bytes behind the last read as zeros
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(from), 0, bytes, 0x00020000)) {}
  __device__ __forceinline__ void copy(void* lds, uint32_t offset) const {   // 16 bytes of each lane, side by side in LDS
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, offset, 0, 0, 0);
  }
};

enum StreamValues { kFinite, kUp, kDown };   // of chunk_of
// 2^(score - ref).  A reference point of 2^30 and more may be off by more than 2^6 from the score that it was rounded from, and a weight formed from both then by as
// many powers of two, up to an infinity or nothing at all: its rows subtract rounded scores.
__device__ __forceinline__ float stream_weight(float s, float scale_log2e, float ref) {
#pragma clang fp contract(off)
  const float scaled = s * scale_log2e;
  return __builtin_amdgcn_exp2f(fabsf(ref) < 0x1p30f ? fmaf(s, scale_log2e, -ref) : scaled - ref);
}

// x for kFinite, y for the others, without a branch for each of many values.
__device__ __forceinline__ float stream_one_of(StreamValues which, float x, float y) {
  const uint32_t first = which == kFinite ? ~0u : 0u;
  return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & first) | (__builtin_bit_cast(uint32_t, y) & ~first));
}

template <int D>
struct StreamTile {
  static constexpr int KS = D / 16, DB = D / 32;   // products of a block of 32 keys, first and second (twice DB)
  int koff[KS], voff[2][DB], kh;
  u32x4 q[KS];
  f32x16 acc[DB];
  float m, l, scale_log2e;

  // (the scale through a vector instruction: straight from a scalar load it makes the compiler wait for all LDS reads)
  __device__ __forceinline__ StreamTile(float scale, int lane)
      : kh(lane >> 5),
        scale_log2e(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, scale) + (lane & 0)))) {
    const int il = lane & 31;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = il * D + 8 * ((2 * ks + kh) ^ k_piece_swizzle<D>(il));
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int t = lane & 15, j = 4 * kh + 8 * half + (t >> 2), d0 = 32 * db + 16 * (il >> 4) + 4 * (t & 3);
        voff[half][db] = j * D + 8 * ((d0 >> 3) ^ v_piece_swizzle<D>(j)) + (d0 & 7);
      }
  }
  __device__ __forceinline__ void load_q(const bf16_t* row) {   // the lane's row
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(row + 8 * kh + 16 * ks);
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ bf16x8 kop(const bf16_t* kb, int jb, int ks) const {
    return *reinterpret_cast<const bf16x8*>(kb + koff[ks] + 32 * jb * D);
  }
  __device__ __forceinline__ bf16x8 vop(const bf16_t* vb, int jb, int s2, int db) const {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const bf16_t* at = vb + (32 * jb + 16 * s2) * D;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at + voff[0][db]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at + voff[1][db]));
    const s16x8 w = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, w);
  }
  static __device__ __forceinline__ f32x16 zeros() {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    return s;
  }
  static __device__ __forceinline__ float top(const f32x16& s) {   // of the lane's 16
    const float m01 = fmaxf(fmaxf(s[0], s[1]), s[2]), m02 = fmaxf(fmaxf(s[3], s[4]), s[5]);
    const float m03 = fmaxf(fmaxf(s[6], s[7]), s[8]), m04 = fmaxf(fmaxf(s[9], s[10]), s[11]);
    const float m05 = fmaxf(fmaxf(s[12], s[13]), s[14]);
    return fmaxf(fmaxf(fmaxf(m01, m02), m03), fmaxf(fmaxf(m04, m05), s[15]));
  }
  // The reference points of rows whose largest score has outgrown them; `largest`: of the lane's half of its row.
  __device__ __forceinline__ void follow(float largest) {
    largest *= scale_log2e;
    if (__any(largest > m + kStreamSlack)) {
      const float cand = fmaxf(m, max_with_other_half(largest));
      const float alpha = cand > m ? __builtin_amdgcn_exp2f(m - cand) : 1.f;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
      m = cand;
    }
  }
  // Offsets that the compiler does not know to be the same in every chunk: otherwise it keeps an address register for each of them and each stage.
  __device__ __forceinline__ void new_offsets() {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(koff[ks]));
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int db = 0; db < DB; ++db) asm volatile("" : "+v"(voff[half][db]));
  }
  // A chunk of 64 keys; hide(s0, s1) puts -inf in the places of keys that a row does not see.  The order is given, a product and what stands beside it at a time: LDS reads run four operands ahead of
  // the products that take them, and the weights of a block are formed between products that do not wait for them.  (In the compiler's own
  // order a product waited for each pair of reads.)
  template <typename Hide>
  __device__ __forceinline__ void chunk(const bf16_t* kb, const bf16_t* vb, Hide hide) {
    constexpr int AHEAD = 4;
    new_offsets();
    f32x16 s0 = zeros(), s1 = zeros();
    {
      bf16x8 k[2 * KS];
#pragma unroll
      for (int f = 0; f < AHEAD; ++f) k[f] = kop(kb, f / KS, f % KS);
#pragma unroll
      for (int f = 0; f < 2 * KS; ++f) {
        if (f + AHEAD < 2 * KS) k[f + AHEAD] = kop(kb, (f + AHEAD) / KS, (f + AHEAD) % KS);
        f32x16& s = f < KS ? s0 : s1;
        s = mfma_bf16(k[f], __builtin_bit_cast(bf16x8, q[f % KS]), s);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    hide(s0, s1);
    follow(fmaxf(top(s0), top(s1)));
    // Weights 2^(score - m) in bf16, the second product's operand (it takes both factors in one type, and V is bf16); their sum is over the
    // rounded ones, which V is multiplied with, so that they still add up to one.  (m = -inf: no finite score so far, all weights are zero.)  Results are off by
    // 0.0021 to 0.0024 of their size against 64 bits; with two halves a weight by 0.0016, their own rounding, and 128 heads of 4,096 tokens in a window of 1,024
    // take 366 us where they take 275, 64 answers to 16,000 tokens 50 where 44.
    typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
    const float ref = m == -INFINITY ? 0.f : m;
    u32x4 p[4];   // of 16 keys each
    auto pair = [&](int w) {   // weights 2 w and 2 w + 1 of the chunk's 32 of this lane
      const f32x16& s = w < 8 ? s0 : s1;
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * (w & 7)], scale_log2e, -ref));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * (w & 7) + 1], scale_log2e, -ref));
      const uint32_t pk = pack_bf16(e0, e1);
      p[w >> 2][w & 3] = pk;
      l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, l, false);
    };
    bf16x8 v[4 * DB];
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) v[f] = vop(vb, f / (2 * DB), f / DB % 2, f % DB);
#pragma unroll
    for (int w = 0; w < 4; ++w) pair(w);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < 4 * DB; ++f) {
      constexpr int PAIRS = 4 / DB;   // between products
      if (f + AHEAD < 4 * DB) v[f + AHEAD] = vop(vb, (f + AHEAD) / (2 * DB), (f + AHEAD) / DB % 2, (f + AHEAD) % DB);
      acc[f % DB] = mfma_bf16(v[f], __builtin_bit_cast(bf16x8, p[f / DB]), acc[f % DB]);
#pragma unroll
      for (int x = 0; x < PAIRS; ++x)
        if (4 + PAIRS * f + x < 16) pair(4 + PAIRS * f + x);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ float sum() const { return l + __shfl_xor(l, 32); }   // of the lane's row

  // A chunk where V may hold infinities and NaN that some rows see and others do not: a weight of zero does not make them vanish.  kFinite forms the sums without
  // them, by the same operations in the same order as above; kUp and kDown then count, in a row's columns, the +inf (or NaN) and the -inf (or NaN) of keys that it sees.
  template <typename Hide>
  __device__ __forceinline__ void chunk_of(StreamValues which, const bf16_t* kb, const bf16_t* vb, Hide hide) {
    new_offsets();
    // bits 15 and 31: which of two values is not finite (an exponent of ones carries)
    auto odd = [](uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
    if (which != kFinite) {   // nothing to count: most chunks
      uint32_t any = 0;
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        const u32x4 v = __builtin_bit_cast(u32x4, vop(vb, f / (2 * DB), f / DB % 2, f % DB));
        any |= odd(v[0]) | odd(v[1]) | odd(v[2]) | odd(v[3]);
        if (f % 2) __builtin_amdgcn_sched_barrier(0);
      }
      if (!__any(any)) return;
    }
    constexpr int AHEAD = D == 128 ? 4 : 1;   // reads at once: more would take more registers than the kernels have
    f32x16 s0 = zeros(), s1 = zeros();
#pragma unroll
    for (int f = 0; f < 2 * KS; ++f) {
      f32x16& s = f < KS ? s0 : s1;
      s = mfma_bf16(kop(kb, f / KS, f % KS), __builtin_bit_cast(bf16x8, q[f % KS]), s);
      if (f % AHEAD == AHEAD - 1) __builtin_amdgcn_sched_barrier(0);
    }
    hide(s0, s1);
    if (which == kFinite) follow(fmaxf(top(s0), top(s1)));   // (counts are not scaled)
    typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
    const float ref = m == -INFINITY ? 0.f : m;
    u32x4 p[4];
    auto weight = [&](float x) { return stream_one_of(which, stream_weight(x, scale_log2e, ref), x == -INFINITY ? 0.f : 1.f); };   // (-inf: hidden, or weighs nothing)
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const f32x16& s = w < 8 ? s0 : s1;
      const uint32_t pk = pack_bf16(weight(s[2 * (w & 7)]), weight(s[2 * (w & 7) + 1]));
      p[w >> 2][w & 3] = pk;
      l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, l, false);
      __builtin_amdgcn_sched_barrier(0);
    }
    auto product = [&](auto value) __attribute__((always_inline)) {   // of two values
#pragma unroll
      for (int f = 0; f < 4 * DB; ++f) {
        u32x4 v = __builtin_bit_cast(u32x4, vop(vb, f / (2 * DB), f / DB % 2, f % DB));
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = value(v[x]);
        acc[f % DB] = mfma_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p[f / DB]), acc[f % DB]);
        if (f % AHEAD == AHEAD - 1) __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (which == kFinite) {
      product([&](uint32_t w) {
        const uint32_t o = odd(w);
        return w & ~((o - (o >> 15)) | o);   // (16 bits of ones for each)
      });
    } else {
      const uint32_t wanted = which == kUp ? 0x7f80u : 0xff80u;
      auto counts = [&](uint32_t b) { return b == wanted || (b & 0x7fffu) > 0x7f80u ? 0x3f80u : 0u; };
      product([&](uint32_t w) { return counts(w & 0xffffu) | counts(w >> 16) << 16; });
    }
  }
};

}  // namespace ac
