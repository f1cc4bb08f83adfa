// Attention of many rows to the states of another sequence: O = softmax(scale Q K^T) V with Sq rows and Sk keys.
// Nothing is causal, so the g Sq rows of the heads that share K and V are alike: one run of R rows, which lie side by side.
//
// bf16: a workgroup owns 128 of these rows, a wave 32, and walks the keys in chunks of 64 that are copied from memory straight into
// one of two LDS stages (the next chunk under way while this one is multiplied, one barrier a chunk).  Both products are
// formed transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane holds scores of one row, and the weights go from the first
// product to the second without leaving their registers.  4 Sk D flop a row against 4 Sk D / 128 bytes: the matrix cores and, more
// so, the vector work beside them at the clock the chip grants bound it.  16 x 32 heads, 1024 x 2047 keys of 128: 555 us = 0.99 PFLOP/s (a
// library's 16384^3 product reaches 1.36 on the card, an 8192^3 one 1.25) in turn with other work, 607 to 615 where such calls follow one another: the same cycles
// at a lower clock.  The matrix pipe is busy in 54 % of them, 31 % of that together with vector work.  Both blocks of a chunk take a softmax step of their own, in an
// order that lets matrix and vector work of a wave overlap.  Raised wave priority in either product or in the exponentials: 2 to 3 % slower.
#include <type_traits>

#include "common.hpp"
#include "f32_tile.hpp"
#include "serve.h"

namespace ac {

constexpr int kCrossChunk = 64;
constexpr int kCrossRows = 128;        // rows of a workgroup
constexpr float kCrossSlack = 8.0f;    // the reference point of a row moves when a score has outgrown it by 2^8
constexpr float kCrossRange = 1e18f;   // the largest sum of weights against a point that does not move
constexpr int kCrossLong = 10;         // chunks from which on it does not

struct CrossArgs {
  const void *Q, *K, *V;
  void* O;
  const int32_t *len, *row_sel;
  int32_t Hkv, R, Sk, D, first, tiles, per;   // first: of the launch's (item, K/V head) tiles; per: workgroups of a tile
  float scale_log2e;
};

template <int D, bool STAY>   // STAY: reference points may stay where the first keys put them (below)
__global__ __launch_bounds__(kThreads, 2) void cross_bf16_kernel(const CrossArgs a) {
  constexpr int PPR = D / 8;                              // 16-byte pieces of a row
  constexpr int NCOPY = kCrossChunk * PPR / kWave / 4;    // copy instructions of a wave, tensor and chunk
  __shared__ __attribute__((aligned(16))) bf16_t kb0[kCrossChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb0[kCrossChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t kb1[kCrossChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb1[kCrossChunk * D];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int il = lane & 31, kh = lane >> 5;
  // workgroups with ids equal mod 8 (one XCD) share K and V in its L2
  const int slot = blockIdx.x >> 3, u = a.first + slot / a.per * 8 + (blockIdx.x & 7);
  if (u >= a.tiles) return;
  const int b = u / a.Hkv;
  if (a.row_sel && a.row_sel[b] >= 0) return;
  const int keys = a.len ? min(max(a.len[b], 0), a.Sk) : a.Sk;
  const int r0 = slot % a.per * kCrossRows + kRowsPerWave * wave, rows = min(kRowsPerWave, a.R - r0);
  bf16_t* O = reinterpret_cast<bf16_t*>(a.O) + ((size_t)u * a.R + r0) * D;
  if (keys == 0) {   // nothing to attend to: zeros
    for (int p = lane; p < rows * PPR; p += kWave) reinterpret_cast<u32x4*>(O)[p] = u32x4{0, 0, 0, 0};
    return;
  }
  const bf16_t* Ksrc = reinterpret_cast<const bf16_t*>(a.K) + (size_t)u * a.Sk * D;
  const bf16_t* Vsrc = reinterpret_cast<const bf16_t*>(a.V) + (size_t)u * a.Sk * D;
  // (the scale through a vector instruction: straight from a scalar load it makes the compiler wait for all LDS reads)
  const float scale_log2e = __builtin_bit_cast(
      float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a.scale_log2e) + (lane & 0)));

  // Copies: instruction i of this wave fills LDS slots [64 (wave + 4 i), ...), slot = row * PPR + position; a lane picks the
  // piece of its row that belongs there.  From one instruction to the next the row grows by 256 / PPR, which leaves the
  // permutations as they are.
  const int slot0 = kWave * wave + lane, crow = slot0 / PPR, cpos = slot0 % PPR;
  const int koff0 = crow * D + 8 * (cpos ^ k_piece_swizzle<D>(crow)), voff0 = crow * D + 8 * (cpos ^ v_piece_swizzle<D>(crow));
  auto copy = [&](bf16_t* kb, bf16_t* vb, int c) {
    const int there = keys - c * kCrossChunk;
    const bf16_t* ks = Ksrc + (size_t)c * kCrossChunk * D;
    const bf16_t* vs = Vsrc + (size_t)c * kCrossChunk * D;
    if (there >= kCrossChunk) {
#pragma unroll
      for (int i = 0; i < NCOPY; ++i) {
        __builtin_amdgcn_global_load_lds(ks + koff0 + 2048 * i, kb + kWave * 8 * (wave + 4 * i), 16, 0, 0);
        __builtin_amdgcn_global_load_lds(vs + voff0 + 2048 * i, vb + kWave * 8 * (wave + 4 * i), 16, 0, 0);
      }
    } else {
      // the last chunk: what lies behind the keys may be anything, and a weight of zero does not make a NaN vanish.  (K rows
      // repeat the last one; their scores are replaced.)
#pragma unroll
      for (int i = 0; i < NCOPY; ++i) {
        const int row = crow + 256 / PPR * i;
        __builtin_amdgcn_global_load_lds(ks + koff0 - crow * D + min(row, there - 1) * D, kb + kWave * 8 * (wave + 4 * i), 16, 0, 0);
        bf16_t* to = vb + kWave * 8 * (wave + 4 * i);
        if (row < there) __builtin_amdgcn_global_load_lds(vs + voff0 + 2048 * i, to, 16, 0, 0);
        else *reinterpret_cast<u32x4*>(to + 8 * lane) = u32x4{0, 0, 0, 0};
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // operand addresses, as the exact kernel has them: K row il, piece 2 ks + kh; V^T by the transposing read in the key order
  // in which the first product leaves the scores
  int koff[D / 16], voff[2][D / 32];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) koff[ks] = il * D + 8 * ((2 * ks + kh) ^ k_piece_swizzle<D>(il));
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const int t = lane & 15, j = 4 * kh + 8 * half + (t >> 2), d0 = 32 * db + 16 * (il >> 4) + 4 * (t & 3);
      voff[half][db] = j * D + 8 * ((d0 >> 3) ^ v_piece_swizzle<D>(j)) + (d0 & 7);
    }
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  auto vop = [&](const bf16_t* vb, int db, int jb, int s2) {
    const bf16_t* at = vb + (32 * jb + 16 * s2) * D;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at + voff[0][db]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(at + voff[1][db]));
    const s16x8 w = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, w);
  };

  copy(kb0, vb0, 0);
  u32x4 q[D / 16];
  {   // (a wave beyond the last row works on a copy of it and stores nothing: no branch of its own in the loop)
    const bf16_t* src = reinterpret_cast<const bf16_t*>(a.Q) + ((size_t)u * a.R + min(r0 + il, a.R - 1)) * D + 8 * kh;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(src + 16 * ks);
  }
  f32x16 acc[D / 32];
  float m_run, l_run;

  auto qk = [&](const bf16_t* kb, int jb) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      s = mfma_bf16(*reinterpret_cast<const bf16x8*>(kb + koff[ks] + 32 * jb * D), __builtin_bit_cast(bf16x8, q[ks]), s);
    return s;
  };
  auto hide = [&](f32x16& s, int limit) {   // keys from `limit` on
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (mfma_row(v, kh) >= limit) s[v] = -INFINITY;
  };
  auto row_max = [&](const f32x16& s) {
    const float m01 = fmaxf(fmaxf(s[0], s[1]), s[2]), m02 = fmaxf(fmaxf(s[3], s[4]), s[5]);
    const float m03 = fmaxf(fmaxf(s[6], s[7]), s[8]), m04 = fmaxf(fmaxf(s[9], s[10]), s[11]);
    const float m05 = fmaxf(fmaxf(s[12], s[13]), s[14]);
    return max_with_other_half(fmaxf(fmaxf(fmaxf(m01, m02), m03), fmaxf(fmaxf(m04, m05), s[15])));
  };
  // Weights 2^(score - m) in bf16, the second product's operand (it takes both factors in one type, and V is bf16); their sum is over the
  // rounded ones, which V is multiplied with, so that they still add up to one.  (m = -inf: no finite score so far, all weights are zero.)
  typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
  auto weights = [&](const f32x16& s, float m, u32x4(&pw)[2], float& sum) {
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * w], scale_log2e, -ref));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * w + 1], scale_log2e, -ref));
      const uint32_t pk = pack_bf16(e0, e1);
      pw[w >> 2][w & 3] = pk;
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, sum, false);
    }
  };
  auto pv = [&](const bf16_t* vb, int jb, const u32x4(&pw)[2]) {
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        acc[db] = mfma_bf16(vop(vb, db, jb, s2), __builtin_bit_cast(bf16x8, pw[s2]), acc[db]);
  };
  auto rescale = [&](float m_new) {
    const float alpha = m_new > m_run ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
  };
  // One chunk of two blocks: the scores of block 1 are requested before the exponentials of block 0, the second product of
  // block 0 before the exponentials of block 1.  `there` keys of the chunk exist (TAIL; all 64 otherwise).  FOLLOW: the reference
  // point of a row follows its largest score; otherwise it stays what it is.
  auto step = [&](const bf16_t* kb, const bf16_t* vb, int there, const bool TAIL, const bool FOLLOW) __attribute__((always_inline)) {
    const bool two = !TAIL || there > 32;
    f32x16 s0 = qk(kb, 0);
    if (TAIL) hide(s0, there);
    if (FOLLOW) {
      const float cand = fmaxf(m_run, row_max(s0) * scale_log2e);
      if (__any(cand > m_run + kCrossSlack)) {
        rescale(cand);
        m_run = cand;
      }
    }
    f32x16 s1;
    if (two) s1 = qk(kb, 1);
    u32x4 p0[2];
    float sum = 0.f;
    weights(s0, m_run, p0, sum);
    l_run += sum;
    if (two) {
      if (TAIL) hide(s1, there - 32);
      float m1 = m_run;
      bool moved = false;
      if (FOLLOW) {
        const float cand = fmaxf(m_run, row_max(s1) * scale_log2e);
        moved = __any(cand > m_run + kCrossSlack);
        if (moved) m1 = cand;
      }
      pv(vb, 0, p0);
      u32x4 p1[2];
      float sum1 = 0.f;
      weights(s1, m1, p1, sum1);
      if (moved) rescale(m1);
      m_run = m1;
      l_run += sum1;
      pv(vb, 1, p1);
    } else {
      pv(vb, 0, p0);
    }
  };
  auto publish = [&]() {   // this wave's copies have landed, then everybody's; the other stage is no longer read
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };

  const int n_chunk = (keys + kCrossChunk - 1) / kCrossChunk, full = keys / kCrossChunk;
  auto walk = [&](const bool FOLLOW) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
    if (!FOLLOW) {   // the reference point of each row: the largest score of the first 32 keys
      publish();
      m_run = row_max(qk(kb0, 0)) * scale_log2e;
    }
    int c = 0;
    for (; c + 1 < full; c += 2) {   // (two chunks a trip: the stages alternate without pointer arithmetic)
      publish();
      copy(kb1, vb1, c + 1);
      step(kb0, vb0, 0, false, FOLLOW);
      publish();
      if (c + 2 < n_chunk) copy(kb0, vb0, c + 2);
      step(kb1, vb1, 0, false, FOLLOW);
    }
    for (; c < n_chunk; ++c) {
      publish();
      bf16_t* kc = (c & 1) ? kb1 : kb0;
      bf16_t* vc = (c & 1) ? vb1 : vb0;
      if (c + 1 < n_chunk) copy((c & 1) ? kb0 : kb1, (c & 1) ? vb0 : vb1, c + 1);
      step(kc, vc, min(kCrossChunk, keys - c * kCrossChunk), true, FOLLOW);
    }
  };
  // Over many keys the reference points stay where the first keys put them: weights may grow until a sum of them reaches 10^18 (2^60),
  // and no digit is lost where later scores are larger.  A step then has a fifth fewer vector instructions and no exchange between lanes ahead of its
  // exponentials.  A workgroup of which a row's sum or result leaves the range (or is NaN), or whose
  // first keys were all -inf (no point to stay at), walks again, with points that follow: all workgroups of 16 x 32 heads, 1024 x 2047 keys
  // 1,095 us instead of 607, of 64 heads of 2048 x 4096 487 instead of 254 (calls following one another).
  // 16 x 32 heads, 1024 x 2047 keys of 128: 590 us following, 555 so; 64 heads of 2048 x 4096 539 / 504, 1024 x 1024 306 / 293, x 700 234 / 227,
  // lengths of 100 to 500 as long.  Of 64 columns both take as long, and the code for both costs short calls a tenth: kernels of their own.
  bool follow = !STAY || full < kCrossLong;
  if (STAY && !follow) {
    walk(false);
    bool again = !(l_run < kCrossRange) || m_run == -INFINITY;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) again |= !(fabsf(acc[db][v]) < INFINITY);
    follow = __syncthreads_or(again);
    if (follow) copy(kb0, vb0, 0);
  }
  if (follow) walk(true);
  __syncthreads();   // every wave is done with both stages: they now stage the output
  if (rows <= 0) return;
  const float sum = l_run + __shfl_xor(l_run, 32);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  bf16_t* ost = wave == 0 ? kb0 : wave == 1 ? vb0 : wave == 2 ? kb1 : vb1;
  if (rows == kRowsPerWave) {
    store_tile_bf16<D>(acc, inv, ost, O, lane);
  } else if (il < rows) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int vq = 0; vq < 4; ++vq)
        *reinterpret_cast<u32x2*>(O + (size_t)il * D + 32 * db + 8 * vq + 4 * kh) =
            u32x2{pack_bf16(acc[db][4 * vq] * inv, acc[db][4 * vq + 1] * inv),
                  pack_bf16(acc[db][4 * vq + 2] * inv, acc[db][4 * vq + 3] * inv)};
  }
}

// Binary32 (the layout of f32_tile.hpp): a wave owns 16 rows, four waves share stages of 32 keys in LDS, the next stage's
// rows are in registers while this one is multiplied.  Each 16-byte read of K or V feeds four products of 32 cycles, so the matrix
// cores bound it: 8 x 24 heads on 8, 1000 x 1000 keys of 128 (lengths 100 to 1000) 341 us = 112 TFLOP/s of the 154 of a large
// product.  32 rows a wave halve the reads, but leave one wave where two hide each other's exponentials: 360.  SPLIT: two waves a row, which
// add up their halves of the keys through LDS at the end (when and what it gains: at the launch).
template <int DB, int COLS, int SPLIT>   // SPLIT: waves that share 16 rows, each with its 32 / SPLIT keys of every stage
__global__ __launch_bounds__(kThreads, DB <= 2 ? 2 : 1) void cross_f32_kernel(const CrossArgs a) {
  constexpr int KC = 32, NB = KC / kF32Rows / SPLIT, WROWS = 4 / SPLIT;   // blocks of a wave and stage; waves' rows side by side
  typedef F32Stage<DB, KC, COLS> Stage;
  const int D = COLS == kAllCols ? 64 * DB : a.D;
  __shared__ __attribute__((aligned(16))) float kl[KC * Stage::LD];
  __shared__ __attribute__((aligned(16))) float vl[KC * Stage::LD];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, kq = lane >> 4, part = wave / WROWS, key0 = part * kF32Rows * NB;
  const int slot = blockIdx.x >> 3, u = a.first + slot / a.per * 8 + (blockIdx.x & 7);
  if (u >= a.tiles) return;
  const int b = u / a.Hkv;
  if (a.row_sel && a.row_sel[b] >= 0) return;
  const int keys = a.len ? min(max(a.len[b], 0), a.Sk) : a.Sk;
  const int r0 = (slot % a.per * WROWS + wave % WROWS) * kF32Rows;   // this wave's first row
  float* O = reinterpret_cast<float*>(a.O) + (size_t)u * a.R * D;
  if (keys == 0) {
    const int n = min(kF32Rows, a.R - r0) * D;
    for (int p = lane; p < n; p += kWave) O[(size_t)r0 * D + p] = 0.f;
    return;
  }
  const float* K = reinterpret_cast<const float*>(a.K) + (size_t)u * a.Sk * D;
  const float* V = reinterpret_cast<const float*>(a.V) + (size_t)u * a.Sk * D;
  f32x4 q[4 * DB], acc[4 * DB];
  {   // (rows beyond the last work on a copy of it)
    const float* src = reinterpret_cast<const float*>(a.Q) + ((size_t)u * a.R + min(r0 + i, a.R - 1)) * D;
#pragma unroll
    for (int kk = 0; kk < 4 * DB; ++kk) {
      const int c = 16 * kk + 4 * kq;
      q[kk] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (COLS == kAllCols || c + 4 <= D) {
        q[kk] = *reinterpret_cast<const f32x4_dw*>(src + c);
      } else {
#pragma unroll
        for (int x = 0; x < 3; ++x)
          if (c + x < D) q[kk][x] = src[c + x];
      }
    }
  }
#pragma unroll
  for (int x = 0; x < 4 * DB; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  Stage ks, vs;
  ks.load(K, 0, keys, D, tid);
  vs.load(V, 0, keys, D, tid);
  for (int j0 = 0; j0 < keys; j0 += KC) {
    ks.template mask<false>(j0, keys, D, tid);   // (scores of keys that are not there are replaced)
    vs.template mask<true>(j0, keys, D, tid);
    __syncthreads();   // the previous stage has been read by everybody
    ks.commit(kl, tid);
    vs.commit(vl, tid);
    __syncthreads();
    if (j0 + KC < keys) {
      ks.load(K, j0 + KC, keys, D, tid);
      vs.load(V, j0 + KC, keys, D, tid);
    }
    f32x4 s[NB];
#pragma unroll
    for (int bk = 0; bk < NB; ++bk) {
      s[bk] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float* row = kl + (key0 + kF32Rows * bk + i) * Stage::LD + 4 * kq;
      f32x4 k = *reinterpret_cast<const f32x4*>(row);
#pragma unroll
      for (int kk = 0; kk < 4 * DB; ++kk)
        if (COLS == kAllCols || 16 * kk < D) {   // uniform
          const f32x4 next = *reinterpret_cast<const f32x4*>(row + 16 * ((kk + 1) & (4 * DB - 1)));
#pragma unroll
          for (int x = 0; x < 4; ++x) s[bk] = mfma_f32(k[x], q[kk][x], s[bk]);
          k = next;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (j0 + KC > keys) {
#pragma unroll
      for (int bk = 0; bk < NB; ++bk)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (j0 + key0 + kF32Rows * bk + 4 * kq + x >= keys) s[bk][x] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int bk = 0; bk < NB; ++bk)
#pragma unroll
      for (int x = 0; x < 4; ++x) mx = fmaxf(mx, s[bk][x]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m, mx * a.scale_log2e);
    if (__any(m_new > m)) {
      const float alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
      l *= alpha;
#pragma unroll
      for (int x = 0; x < 4 * DB; ++x) acc[x] *= alpha;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m;   // no finite score so far: all weights are zero
#pragma unroll
    for (int bk = 0; bk < NB; ++bk) {
      f32x4 p;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        p[x] = __builtin_amdgcn_exp2f(fmaf(s[bk][x], a.scale_log2e, -ref));
        l += p[x];
      }
      f32_weights_v<DB>(acc, vl + (key0 + kF32Rows * bk) * Stage::LD, p, i, kq);
    }
  }
  float sum = l + __shfl_xor(l, 16);
  sum += __shfl_xor(sum, 32);
  if constexpr (SPLIT == 2) {   // the second wave's sums through the stages, which nobody reads any more
    static_assert(4 * DB * kWave * 4 * WROWS <= KC * Stage::LD, "sums of two waves");
    f32x4* sums = reinterpret_cast<f32x4*>(kl) + wave % WROWS * 4 * DB * kWave + lane;
    float* stats = vl + wave % WROWS * 2 * kWave + lane;
    __syncthreads();
    if (part > 0) {
#pragma unroll
      for (int x = 0; x < 4 * DB; ++x) sums[x * kWave] = acc[x];
      stats[0] = m;
      stats[kWave] = sum;
    }
    __syncthreads();
    if (part > 0) return;
    const float m1 = stats[0], top = fmaxf(m, m1);
    const float f0 = m < top ? __builtin_amdgcn_exp2f(m - top) : 1.f, f1 = m1 < top ? __builtin_amdgcn_exp2f(m1 - top) : 1.f;
    sum = sum * f0 + stats[kWave] * f1;
#pragma unroll
    for (int x = 0; x < 4 * DB; ++x) acc[x] = acc[x] * f0 + sums[x * kWave] * f1;
  }
  if (r0 + i < a.R)
    f32_store_row<DB, COLS, true>(O + (size_t)(r0 + i) * D, acc, sum == 0.f ? 1.f : sum, kq, D);
}

// Few rows leave most of these kernels' waves without any, and few workgroups most of the chip; decode.hip splits the keys instead,
// and reads K and V again for every 16 rows.  us, there / here.  bf16, heads x rows x keys, by units of 16 rows: 128 x 32 x 1000 (256
// units) 11.2 / 17.9 of 64, 18.4 / 25.5 of 128; 128 x 64 x 1000 (512) 18.5 / 18.0 and 32.5 / 25.9; 16 x 500 x 1500 (512) 24.2 / 22.6 and
// 45.9 / 33.7; 512 x 32 x 100 (1,024) 7.8 / 7.7 and 12.5 / 12.3; 512 x 32 x 1000 33.9 / 27.6 and 66.4 / 53.1.  Binary32, by workgroups of 32
// rows (as here where they are few): 64 x 64 x 300 of 128 (128) 14.3 / 21.1; 16 x 282 x 333, ragged (144) 16.5 / 16.9; 256 x 32 x 300 (256) 23.6 / 22.1,
// ragged 17.8 / 21.2; 128 x 64 x 500 (256) 33.7 / 32.0, x 1000 of 256 226 / 133; 64 x 282 x 333, ragged (576) 38.5 / 33.2, x 1000 62.3 / 65.8; 512 x 20 x
// 500 (512) 68 / 54.  (The host does not know the lengths: the line is where equal ones change sides, and two of the ragged sizes here lose by it.  Keys
// beyond 1,500 were not swept.)
static bool cross_by_rows(int64_t B, int64_t Hkv, int64_t R, int64_t Sk, int32_t D, int32_t is_f32) {
  const int64_t heads = B * Hkv;
  if (is_f32) return D >= 4 && R > 16 && heads * ((R + 2 * kF32Rows - 1) / (2 * kF32Rows)) >= 256;
  return !decode_fits(B, Hkv, R, Sk) || (R > 16 && heads * ((R + 15) / 16) >= 512);
}
size_t cross_workspace_bytes(int32_t B, int32_t Hkv, int32_t R, int32_t Sk, int32_t D, int32_t is_f32) {
  return cross_by_rows(B, Hkv, R, Sk, D, is_f32) ? 0 : decode_workspace_bytes(R, D);
}

// All tiles, in launches of at most 2^23 workgroups (a multiple of eight tiles each).
template <typename Kernel>
static hipError_t cross_tiles(Kernel kernel, CrossArgs a, hipStream_t stream) {
  const int64_t most = ((1 << 23) / a.per > 8 ? (1 << 23) / a.per : 8) & ~7LL;
  for (int64_t first = 0; first < a.tiles; first += most) {
    a.first = (int)first;
    const int64_t n = a.tiles - first < most ? a.tiles - first : most;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n + 7) / 8 * 8 * a.per)), dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int DB, int COLS>
static hipError_t launch_cross_f32(CrossArgs a, hipStream_t stream) {
  a.per = (a.R + 4 * kF32Rows - 1) / (4 * kF32Rows);
  // Two waves a row halve a workgroup's rows and its time, but stages of K and V serve half as many products.  us, four waves / two and two,
  // workgroups of 64 rows, keys of 128: few of them, 128 x 64 x 500 (128) 45.4 / 32.0, of 256 x 1000 228 / 133, 256 x 64 x 1000 (256) 88 / 92;
  // two a compute unit and ragged (a long one beside a long one), 64 x 282 x 333 (320) 37.5 / 33.2, 448 x 64 x 300 (448) 41.9 / 36.6, x 576
  // (576) 49.7 / 48.4, not ragged (448) 54.6 / 61.1; last workgroups at most half full, 512 x 20 x 500 (512) 85 / 54, 512 x 130 x 300 (1,536) 145 /
  // 142, 512 x 270 x 300 (2,560) 239 / 240; others, 512 x 40 x 300 (512) 55.8 / 67.4, 64 x 3000 x 1000 (3,008) 340 / 382.  (Whether lengths are given stands
  // for ragged ones, since the host does not know them: where they are all the same, 448 workgroups take 61.1 and not 54.6.)
  const int64_t wgs = (int64_t)a.tiles * a.per;
  if (wgs < 256 || (a.len && wgs < 512) || (a.R < 320 && (a.R - 1) % 64 < 32)) {
    a.per = (a.R + 2 * kF32Rows - 1) / (2 * kF32Rows);
    return cross_tiles(&cross_f32_kernel<DB, COLS, 2>, a, stream);
  }
  return cross_tiles(&cross_f32_kernel<DB, COLS, 1>, a, stream);
}

hipError_t launch_cross(const DecodeLaunch& p, hipStream_t stream) {
  if (!cross_by_rows(p.B, p.Hkv, p.R, p.Sk, p.D, p.is_f32)) return launch_decode(p, stream);
  CrossArgs a;
  a.Q = p.Q; a.K = p.K; a.V = p.V; a.O = p.O; a.len = p.len; a.row_sel = p.row_sel;
  a.Hkv = p.Hkv; a.R = p.R; a.Sk = p.Sk; a.D = p.D;
  a.first = 0;
  a.tiles = p.B * p.Hkv;
  a.per = (p.R + kCrossRows - 1) / kCrossRows;
  const float scale = p.scale == 0.f ? 1.0f / sqrtf((float)p.D) : p.scale;
  a.scale_log2e = scale * 1.44269504088896340736f;
  if (!p.is_f32)
    return p.D == 64                              ? cross_tiles(&cross_bf16_kernel<64, false>, a, stream)
           : p.Sk >= kCrossLong * kCrossChunk ? cross_tiles(&cross_bf16_kernel<128, true>, a, stream)
                                              : cross_tiles(&cross_bf16_kernel<128, false>, a, stream);
  if (p.D == 64) return launch_cross_f32<1, kAllCols>(a, stream);
  if (p.D == 128) return launch_cross_f32<2, kAllCols>(a, stream);
  if (p.D < 64) return p.D % 4 ? launch_cross_f32<1, kAnyCols>(a, stream) : launch_cross_f32<1, kVecCols>(a, stream);
  if (p.D < 128) return p.D % 4 ? launch_cross_f32<2, kAnyCols>(a, stream) : launch_cross_f32<2, kVecCols>(a, stream);
  return p.D % 4 ? launch_cross_f32<4, kAnyCols>(a, stream) : launch_cross_f32<4, kVecCols>(a, stream);
}

}  // namespace ac
