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
  // A chunk of 64 keys; hide(s0, s1) puts -inf in the places of keys that a row does not see.  The order is given, a product and what stands beside it at a time: LDS reads run four operands ahead of
  // the products that take them, and the weights of a block are formed between products that do not wait for them.  (In the compiler's own
  // order a product waited for each pair of reads.)
  template <typename Hide>
  __device__ __forceinline__ void chunk(const bf16_t* kb, const bf16_t* vb, Hide hide) {
    constexpr int AHEAD = 4;
    // offsets that the compiler does not know to be the same in every chunk: otherwise it keeps an address register for each of them and each stage
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(koff[ks]));
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int db = 0; db < DB; ++db) asm volatile("" : "+v"(voff[half][db]));
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
    // rounded ones, which V is multiplied with, so that they still add up to one.  (m = -inf: no finite score so far, all weights are zero.)
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
};

}  // namespace ac
