// Attention of few rows over many keys: one new token of each request over its pages, or a few query rows over an
// encoder's states.  O = softmax(scale Q K^T) V for the R rows of each (item b, K/V head), which lie side by side in Q and
// O (the g heads that share K and V, times their rows); keys j < len[b] are seen.
//
// Each byte of K and V serves few products (2 R flop a byte in bf16), so memory bounds it, and the keys of all
// requests have to be in flight on all compute units, however long or short each request is.  The work is therefore cut
// by keys, not by requests: all blocks of 32 keys (16 in binary32) of all units (item, K/V head, 32 or 16 rows) form one row of
// T blocks, and each of a fixed number of workgroups takes an equal run of it, which it finds from the lengths by itself.
// A run covers the end of one unit, some whole ones and the beginning of another.  The four waves of a workgroup deal
// out the blocks of a unit and meet in LDS; a whole unit leaves as output, the at most two others as partial results
// (row maximum, sum, sum of weighted V, binary32), which decode_join_kernel adds up.  So the workspace does not grow with the lengths,
// and the host need not know them.
//
// A wave's block: K rows go straight from memory to the lanes that multiply them (S^T = K Q^T), V rows through a
// wave-private LDS tile where the transposing read wants them (O^T = V^T P^T; binary32: straight from memory), the next
// block's on their way meanwhile.  A lane holds one key row of K and of V, so it needs one page number a block, asked for two
// blocks ahead.  Pages may end anywhere inside a block.
#include <type_traits>

#include "common.hpp"
#include "f32_tile.hpp"
#include "serve.h"
#include "split_tile.hpp"

namespace ac {

constexpr int kDecodeWaves = 4;
constexpr int kDecodeMost = 1024;   // workgroups, what the workspace is sized for
constexpr float kDecodeSlack = 8.0f;   // as in exact attention: the reference point of a row moves when it is outgrown by 2^8

struct DecodeArgs {
  const void *Q, *K, *V;
  void* O;
  const int32_t *table, *len, *row_sel;
  float *part, *stat;   // partial results [2 workgroups][rp][D] and their (maximum, sum) [2 workgroups][rp][2]
  int32_t B, Hkv, R, rbs, rp, D, Sk;   // rbs: row blocks of a K/V head; rp: rows of a partial result
  int32_t n_pages, ps, max_pages, groups;
  int64_t page_stride, head_stride;
  Divider by_ps;
  float scale_log2e;
};

// How the blocks of all units are numbered and dealt: item by item, in it K/V head, row block, key block.
template <int BK>
struct DecodeWalk {
  const DecodeArgs& a;
  int lane, per, total;
  __device__ __forceinline__ int keys(int b) const {
    if (a.row_sel && a.row_sel[b] >= 0) return 0;
    return a.len ? min(max(a.len[b], 0), a.Sk) : a.Sk;
  }
  __device__ __forceinline__ int blocks(int b) const { return (keys(b) + BK - 1) / BK; }   // of a unit of item b
  __device__ __forceinline__ DecodeWalk(const DecodeArgs& a, int lane) : a(a), lane(lane) {
    int t = 0;
    for (int b = lane; b < a.B; b += kWave) t += blocks(b);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
    total = __builtin_amdgcn_readfirstlane(t) * (a.Hkv * a.rbs);
    per = max(kDecodeWaves, (total + a.groups - 1) / a.groups);
  }
  // number of the first block of item `item`
  __device__ __forceinline__ int start(int item) const {
    int t = 0;
    for (int b = lane; b < item; b += kWave) t += blocks(b);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
    return __builtin_amdgcn_readfirstlane(t) * (a.Hkv * a.rbs);
  }
  // the item that block x < total belongs to; x becomes the block's number in it
  __device__ __forceinline__ int locate(int& x) const {
    int before = 0;
    for (int b0 = 0;; b0 += kWave) {
      int t = b0 + lane < a.B ? blocks(b0 + lane) * (a.Hkv * a.rbs) : 0;
#pragma unroll
      for (int off = 1; off < kWave; off <<= 1) {
        const int p = __shfl_up(t, off);
        if (lane >= off) t += p;
      }
      const unsigned long long beyond = __ballot(x < before + t);
      if (beyond || b0 + kWave >= a.B) {
        const int i = beyond ? __builtin_ctzll(beyond) : 0;
        const int prev = __shfl(t, max(i - 1, 0));
        x -= before + (i > 0 ? prev : 0);
        x = __builtin_amdgcn_readfirstlane(x);
        return b0 + i;
      }
      before += __builtin_amdgcn_readlane(t, kWave - 1);
    }
  }
};

// Where the K and V row of key j < keys of item b lies, in elements from its head's first row of the first page (or of the
// item); -1 where there is none.  Two steps, so that the page number can be asked for early.
template <bool PAGED>
struct DecodeRows {
  const DecodeArgs& a;
  const int32_t* pages;
  int keys, D;
  __device__ __forceinline__ int ask(int j) const {
    return PAGED && j < keys ? pages[a.by_ps.div(j)] : 0;
  }
  __device__ __forceinline__ int64_t at(int j, int page) const {
    if (j >= keys) return -1;
    if (!PAGED) return (int64_t)j * D;
    if ((unsigned)page >= (unsigned)a.n_pages) return -1;
    return page * a.page_stride + (int64_t)(j - a.by_ps.div(j) * a.ps) * D;
  }
};

// Position of piece p of row r in the V tile: the rows of a transposing read are spread over the banks as v_piece_swizzle does
// it, and, since a lane writes pieces of one row here, the eight or sixteen rows of a write too.
template <int D>
__device__ __forceinline__ int decode_v_piece(int r) {
  return v_piece_swizzle<D>(r) ^ ((r >> 2) & 3);
}

// The rows of a unit, summed over the waves: out as bf16 or binary32 (a whole unit) or as a partial result.
template <bool PAGED, int D>
__global__ __launch_bounds__(kDecodeWaves* kWave, 2) void decode_bf16_kernel(const DecodeArgs a) {
  constexpr int NW = kDecodeWaves, BK = 32, NP = D / 16;   // 16-byte pieces of a row that a lane half holds
  __shared__ __attribute__((aligned(16))) f32x4 smem[NW * (D / 8) * kWave];   // V tiles, then the waves' sums
  __shared__ float ms[NW][32], ls[NW][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int il = lane & 31, kh = lane >> 5;
  const DecodeWalk<BK> walk(a, lane);
  int x = blockIdx.x * walk.per;
  if (x >= walk.total) return;
  int left = min(walk.per, walk.total - x);
  int b = walk.locate(x);
  bf16_t* vt = reinterpret_cast<bf16_t*>(smem) + wave * 32 * D;
  while (true) {
    const int keys = __builtin_amdgcn_readfirstlane(walk.keys(b)), nb = (keys + BK - 1) / BK;
    if (nb == 0) {   // (not the item that was located: there are more blocks to come behind it)
      ++b;
      continue;
    }
    const int unit = x / nb, first = x - unit * nb, n = min(nb - first, left);
    const int hk = unit / a.rbs, row0 = 32 * (unit - hk * a.rbs), rows = min(32, a.R - row0);
    const size_t head = (size_t)b * a.Hkv + hk;
    const bf16_t* K = reinterpret_cast<const bf16_t*>(a.K) + (PAGED ? hk : head) * a.head_stride;
    const bf16_t* V = reinterpret_cast<const bf16_t*>(a.V) + (PAGED ? hk : head) * a.head_stride;
    const DecodeRows<PAGED> where{a, PAGED ? a.table + (size_t)b * a.max_pages : nullptr, keys, D};
    u32x4 q[NP], k[NP], v[NP];
    {
      const bf16_t* src = reinterpret_cast<const bf16_t*>(a.Q) + (head * a.R + row0 + min(il, rows - 1)) * D + 8 * kh;
#pragma unroll
      for (int i = 0; i < NP; ++i) q[i] = *reinterpret_cast<const u32x4*>(src + 16 * i);
    }
    const int end = first + n;
    int blk = first + wave, page = 0;
    int64_t at = -1, next_at = -1;
    auto load = [&](u32x4(&r)[NP], const bf16_t* base, int64_t where_at) {
      const bf16_t* src = base + (where_at < 0 ? 0 : where_at) + 8 * kh;   // (page 0 or row 0: there, and not used)
#pragma unroll
      for (int i = 0; i < NP; ++i) r[i] = *reinterpret_cast<const u32x4*>(src + 16 * i);
    };
    if (blk < end) {
      at = where.at(BK * blk + il, where.ask(BK * blk + il));
      load(k, K, at);
      load(v, V, at);
      if (blk + NW < end) page = where.ask(BK * (blk + NW) + il);
    }
    f32x16 acc[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    for (; blk < end; blk += NW) {
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i) s = mfma_bf16(__builtin_bit_cast(bf16x8, k[i]), __builtin_bit_cast(bf16x8, q[i]), s);
      const bool there = at >= 0, more = blk + NW < end;
      if (more) {
        next_at = where.at(BK * (blk + NW) + il, page);
        load(k, K, next_at);
        if (blk + 2 * NW < end) page = where.ask(BK * (blk + 2 * NW) + il);
      }
      const uint32_t seen = (uint32_t)__ballot(there);   // the block's 32 keys (both lane halves say the same)
      if (seen != 0xffffffffu) {   // a weight of zero does not make a NaN vanish: rows that are not there are zero
#pragma unroll
        for (int i = 0; i < NP; ++i)
          if (!there) v[i] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((seen >> mfma_row(i, kh)) & 1)) s[i] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < NP; ++i)
        *reinterpret_cast<u32x4*>(vt + il * D + 8 * ((2 * i + kh) ^ decode_v_piece<D>(il))) = v[i];
      if (more) load(v, V, next_at);
      at = next_at;
      wave_lds_fence();
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      const float cand = fmaxf(m, max_with_other_half(mx) * a.scale_log2e);
      if (__any(cand > m + kDecodeSlack)) {
        const float alpha = cand > m ? __builtin_amdgcn_exp2f(m - cand) : 1.f;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[db][i] *= alpha;
        m = cand;
      }
      const float ref = m == -INFINITY ? 0.f : m;   // no finite score so far: all weights are zero
      typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
      u32x4 p[2];
#pragma unroll
      for (int w = 0; w < 8; ++w) {   // the sum is over the rounded weights, which V is multiplied with
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[2 * w], a.scale_log2e, -ref));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[2 * w + 1], a.scale_log2e, -ref));
        const uint32_t pk = pack_bf16(e0, e1);
        p[w >> 2][w & 3] = pk;
        l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, l, false);
      }
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          s16x4 w[2];
#pragma unroll
          for (int half = 0; half < 2; ++half) {   // (the key order in which the scores lie in the registers)
            const int t = lane & 15, j = 16 * s2 + 4 * kh + 8 * half + (t >> 2);
            const int d0 = 32 * db + 16 * (il >> 4) + 4 * (t & 3);
            w[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(
                vt + j * D + 8 * ((d0 >> 3) ^ decode_v_piece<D>(j)) + (d0 & 7)));
          }
          const s16x8 vop = {w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]};
          acc[db] = mfma_bf16(__builtin_bit_cast(bf16x8, vop), __builtin_bit_cast(bf16x8, p[s2]), acc[db]);
        }
      wave_lds_fence();   // the tile is read before the next block's rows are written
    }
    l += __shfl_xor(l, 32);
    if (kh == 0) {
      ms[wave][il] = m;
      ls[wave][il] = l;
    }
    __syncthreads();   // statistics are there, V tiles are no longer read
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[w][il]);
    auto factor = [&](float mw) { return mw < top ? __builtin_amdgcn_exp2f(mw - top) : 1.f; };
#pragma unroll
    for (int w = 0; w < NW; ++w) sum = fmaf(ls[w][il], factor(ms[w][il]), sum);
    const float mine = factor(m);
    if (il < rows) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int vq = 0; vq < 4; ++vq)
          smem[(wave * (D / 8) + 4 * db + vq) * kWave + lane] =
              f32x4{acc[db][4 * vq], acc[db][4 * vq + 1], acc[db][4 * vq + 2], acc[db][4 * vq + 3]} * mine;
    }
    __syncthreads();
    const bool whole = n == nb;
    const size_t slot = (size_t)(2 * blockIdx.x + (first == 0)) * a.rp;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;   // no key at all: zeros
    if (il < rows) {
#pragma unroll
      for (int n0 = 0; n0 < D / 8; n0 += NW) {   // columns 8 i + 4 kh and three more of row il
        const int i = n0 + wave;
        f32x4 r = smem[i * kWave + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) r += smem[(w * (D / 8) + i) * kWave + lane];
        const int d = 8 * i + 4 * kh;
        if (whole)
          *reinterpret_cast<u32x2*>(reinterpret_cast<bf16_t*>(a.O) + (head * a.R + row0 + il) * D + d) =
              u32x2{pack_bf16(r[0] * inv, r[1] * inv), pack_bf16(r[2] * inv, r[3] * inv)};
        else
          *reinterpret_cast<f32x4*>(a.part + (slot + il) * D + d) = r;
      }
      if (!whole && wave == 0 && kh == 0) {
        a.stat[2 * (slot + il)] = top;
        a.stat[2 * (slot + il) + 1] = sum;
      }
    }
    left -= n;
    if (left == 0) break;
    x += n;
    if (x == nb * a.Hkv * a.rbs) {
      ++b;
      x = 0;
    }
    __syncthreads();   // the sums have been read: the next unit's V rows may be written there
  }
}

// Binary32: blocks of 16 keys, units of 16 rows, the layout of f32_tile.hpp.  D of any size: a row that is no whole number of
// 16-byte pieces is read in pieces of four that start at any 4-byte address, its end in single floats.
template <bool PAGED, int DB, bool FULL>   // FULL: D == 64 DB
__global__ __launch_bounds__(kDecodeWaves* kWave, DB <= 2 ? 2 : 1) void decode_f32_kernel(const DecodeArgs a) {
  constexpr int NW = kDecodeWaves, BK = kF32Rows;
  __shared__ __attribute__((aligned(16))) f32x4 part[NW][4 * DB][kWave];
  __shared__ float ms[NW][kF32Rows], ls[NW][kF32Rows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, kq = lane >> 4, D = FULL ? 64 * DB : a.D;
  const DecodeWalk<BK> walk(a, lane);
  int x = blockIdx.x * walk.per;
  if (x >= walk.total) return;
  int left = min(walk.per, walk.total - x);
  int b = walk.locate(x);
  // four columns from c on, zeros behind the row's end
  auto four = [&](const float* row, int c) {
    if (FULL) return *reinterpret_cast<const f32x4*>(row + c);
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (c + 4 <= D) r = *reinterpret_cast<const f32x4_dw*>(row + c);
    else
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (c + t < D) r[t] = row[c + t];
    return r;
  };
  while (true) {
    const int keys = __builtin_amdgcn_readfirstlane(walk.keys(b)), nb = (keys + BK - 1) / BK;
    if (nb == 0) {
      ++b;
      continue;
    }
    const int unit = x / nb, first = x - unit * nb, n = min(nb - first, left);
    const int hk = unit / a.rbs, row0 = kF32Rows * (unit - hk * a.rbs), rows = min(kF32Rows, a.R - row0);
    const size_t head = (size_t)b * a.Hkv + hk;
    const float* K = reinterpret_cast<const float*>(a.K) + (PAGED ? hk : head) * a.head_stride;
    const float* V = reinterpret_cast<const float*>(a.V) + (PAGED ? hk : head) * a.head_stride;
    const DecodeRows<PAGED> where{a, PAGED ? a.table + (size_t)b * a.max_pages : nullptr, keys, D};
    f32x4 q[4 * DB], k[4 * DB], v[4][DB];
    {
      const float* src = reinterpret_cast<const float*>(a.Q) + (head * a.R + row0 + min(i, rows - 1)) * D;
#pragma unroll
      for (int kk = 0; kk < 4 * DB; ++kk) q[kk] = four(src, 16 * kk + 4 * kq);
    }
    auto load_k = [&](int64_t at) {   // key i's columns 16 kk + 4 kq and three more
      const float* src = K + (at < 0 ? 0 : at);
#pragma unroll
      for (int kk = 0; kk < 4 * DB; ++kk) k[kk] = four(src, 16 * kk + 4 * kq);
    };
    auto load_v = [&](int64_t at) {   // columns 64 db + 4 i and three more of keys 4 kq ... 4 kq + 3; zeros if they are not there
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t from = __shfl((long long)at, 4 * kq + t);
        const float* src = V + (from < 0 ? 0 : from);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          v[t][db] = four(src, 64 * db + 4 * i);
          if (from < 0) v[t][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
    };
    const int end = first + n;
    int blk = first + wave, page = 0;
    int64_t at = -1, next_at = -1;
    if (blk < end) {
      at = where.at(BK * blk + i, where.ask(BK * blk + i));
      load_k(at);
      load_v(at);
      if (blk + NW < end) page = where.ask(BK * (blk + NW) + i);
    }
    f32x4 acc[4 * DB];
#pragma unroll
    for (int t = 0; t < 4 * DB; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (; blk < end; blk += NW) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4 * DB; ++kk)
        if (FULL || 16 * kk < D)
#pragma unroll
          for (int t = 0; t < 4; ++t) s = mfma_f32(k[kk][t], q[kk][t], s);
      const uint32_t seen = (uint32_t)__ballot(at >= 0) >> (4 * kq);
      const bool more = blk + NW < end;
      if (more) {
        next_at = where.at(BK * (blk + NW) + i, page);
        load_k(next_at);
        if (blk + 2 * NW < end) page = where.ask(BK * (blk + 2 * NW) + i);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (!((seen >> t) & 1)) s[t] = -INFINITY;
        mx = fmaxf(mx, s[t]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m, mx * a.scale_log2e);
      if (__any(m_new > m)) {
        const float alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < 4 * DB; ++t) acc[t] *= alpha;
        m = m_new;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      f32x4 p;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        p[t] = __builtin_amdgcn_exp2f(fmaf(s[t], a.scale_log2e, -ref));
        l += p[t];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[4 * db + c] = mfma_f32(v[t][db][c], p[t], acc[4 * db + c]);
      if (more) load_v(next_at);
      at = next_at;
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lane < kF32Rows) {
      ms[wave][lane] = m;
      ls[wave][lane] = l;
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[w][i]);
    auto factor = [&](float mw) { return mw < top ? __builtin_amdgcn_exp2f(mw - top) : 1.f; };
#pragma unroll
    for (int w = 0; w < NW; ++w) sum = fmaf(ls[w][i], factor(ms[w][i]), sum);
    const float mine = factor(m);
    if (i < rows)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          part[wave][4 * db + t][lane] = f32x4{acc[4 * db][t], acc[4 * db + 1][t], acc[4 * db + 2][t], acc[4 * db + 3][t]} * mine;
    __syncthreads();
    const bool whole = n == nb;
    const size_t slot = (size_t)(2 * blockIdx.x + (first == 0)) * a.rp;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (i < rows) {
      float* to = whole ? reinterpret_cast<float*>(a.O) + (head * a.R + row0 + i) * D : a.part + (slot + i) * D;
#pragma unroll
      for (int n0 = 0; n0 < 4 * DB; n0 += NW) {   // columns d and three more of row i
        const int c = n0 + wave, d = 64 * (c >> 2) + 16 * kq + 4 * (c & 3);
        f32x4 r = part[0][c][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) r += part[w][c][lane];
        if (whole)
#pragma unroll
          for (int t = 0; t < 4; ++t) r[t] = sum == 0.f ? 0.f : f32_divide(r[t], sum, inv);
        if (FULL || d + 4 <= D) *reinterpret_cast<f32x4_dw*>(to + d) = r;
        else
#pragma unroll
          for (int t = 0; t < 3; ++t)
            if (d + t < D) to[d + t] = r[t];
      }
      if (!whole && wave == 0 && kq == 0) {
        a.stat[2 * (slot + i)] = top;
        a.stat[2 * (slot + i) + 1] = sum;
      }
    }
    left -= n;
    if (left == 0) break;
    x += n;
    if (x == nb * a.Hkv * a.rbs) {
      ++b;
      x = 0;
    }
    __syncthreads();
  }
}

// The rows of units that several workgroups shared, and zeros for rows without a key.  NW waves add up one output row: its
// partial results are those of the workgroups whose runs touch its unit.
template <bool F32, int NW>
__global__ __launch_bounds__(NW == 1 ? kThreads : NW * kWave) void decode_join_kernel(const DecodeArgs a) {
  constexpr int BK = F32 ? kF32Rows : 32, RB = BK, COLS = F32 ? 4 : 2;   // columns of a lane: D <= 256, 128
  __shared__ float sums[NW][COLS * kWave];
  __shared__ float weight[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const DecodeWalk<BK> walk(a, lane);
  const int n_rows = a.B * a.Hkv * a.R;   // of all items
  for (int row = NW == 1 ? blockIdx.x * (kThreads / kWave) + wave : blockIdx.x; row < n_rows;
       row += NW == 1 ? gridDim.x * (kThreads / kWave) : gridDim.x) {
    const int head = row / a.R, r = row - head * a.R, b = head / a.Hkv, hk = head - b * a.Hkv;
    if (a.row_sel && a.row_sel[b] >= 0) continue;
    const int nb = __builtin_amdgcn_readfirstlane(walk.blocks(b));
    float o[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) o[c] = 0.f;
    float total = 0.f;
    if (nb > 0) {
      const int from = walk.start(b) + (hk * a.rbs + r / RB) * nb;
      const int w0 = from / walk.per, w1 = (from + nb - 1) / walk.per;
      if (w0 == w1) continue;   // one workgroup had all of it
      auto slot = [&](int w) { return (size_t)(2 * w + (w * walk.per <= from)) * a.rp + r % RB; };
      float top = -INFINITY;
      for (int w = w0 + lane; w <= w1; w += kWave) top = fmaxf(top, a.stat[2 * slot(w)]);
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
#pragma unroll 4
      for (int w = w0 + (NW == 1 ? 0 : wave); w <= w1; w += NW) {
        const size_t at = slot(w);
        const float m = a.stat[2 * at], f = m < top ? __builtin_amdgcn_exp2f(m - top) : 1.f;
        total = fmaf(a.stat[2 * at + 1], f, total);
#pragma unroll
        for (int c = 0; c < COLS; ++c)
          if (c * kWave + lane < a.D) o[c] = fmaf(a.part[at * a.D + c * kWave + lane], f, o[c]);
      }
      if (NW > 1) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) sums[wave][c * kWave + lane] = o[c];
        if (lane == 0) weight[wave] = total;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int w = 1; w < NW; ++w) {
            total += weight[w];
#pragma unroll
            for (int c = 0; c < COLS; ++c) o[c] += sums[w][c * kWave + lane];
          }
        }
        __syncthreads();
      }
    }
    if (NW > 1 && wave > 0) continue;
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      const int d = c * kWave + lane;
      if (d >= a.D) continue;
      const float r_ = total == 0.f ? 0.f : o[c] / total;
      if (F32) reinterpret_cast<float*>(a.O)[(size_t)row * a.D + d] = r_;
      else reinterpret_cast<bf16_t*>(a.O)[(size_t)row * a.D + d] = (bf16_t)r_;
    }
  }
}

size_t decode_workspace_bytes(int32_t R, int32_t D) {
  return (size_t)2 * kDecodeMost * (R < 32 ? R : 32) * (D + 2) * sizeof(float);
}
bool decode_fits(int64_t B, int64_t Hkv, int64_t R, int64_t keys) {
  // (row blocks of 16 and key blocks of 16: binary32, the smaller ones; and the rows themselves)
  const double blocks = (double)B * Hkv * ((R + 15) / 16) * ((keys + 15) / 16);
  return blocks < 2147483648.0 - 65536 && (double)B * Hkv * R < 2147483648.0 - 65536;
}

hipError_t launch_decode(const DecodeLaunch& p, hipStream_t stream) {
  const int rb = p.is_f32 ? kF32Rows : 32;
  DecodeArgs a;
  a.Q = p.Q; a.K = p.K; a.V = p.V; a.O = p.O; a.table = p.table; a.len = p.len; a.row_sel = p.row_sel;
  a.B = p.B; a.Hkv = p.Hkv; a.R = p.R; a.D = p.D; a.Sk = p.Sk;
  a.rbs = (p.R + rb - 1) / rb;
  a.rp = p.R < rb ? p.R : rb;
  a.n_pages = p.n_pages; a.ps = p.page_size; a.max_pages = p.max_pages; a.page_stride = p.page_stride;
  a.head_stride = (int64_t)(p.table ? p.page_size : p.Sk) * p.D;
  a.by_ps = Divider((uint32_t)(p.table ? p.page_size : 1));
  const float scale = p.scale == 0.f ? 1.0f / sqrtf((float)p.D) : p.scale;
  a.scale_log2e = scale * 1.44269504088896340736f;
  a.groups = 512;
  a.stat = static_cast<float*>(p.ws);
  a.part = a.stat + (size_t)2 * kDecodeMost * a.rp * 2;
  const dim3 grid((unsigned)a.groups), block(kDecodeWaves * kWave);
  auto go = [&](auto paged) {
    constexpr bool P = decltype(paged)::value;
    if (!p.is_f32) {
      if (p.D == 64) hipLaunchKernelGGL((decode_bf16_kernel<P, 64>), grid, block, 0, stream, a);
      else hipLaunchKernelGGL((decode_bf16_kernel<P, 128>), grid, block, 0, stream, a);
    } else if (p.D == 64) {
      hipLaunchKernelGGL((decode_f32_kernel<P, 1, true>), grid, block, 0, stream, a);
    } else if (p.D == 128) {
      hipLaunchKernelGGL((decode_f32_kernel<P, 2, true>), grid, block, 0, stream, a);
    } else if (p.D < 64) {
      hipLaunchKernelGGL((decode_f32_kernel<P, 1, false>), grid, block, 0, stream, a);
    } else if (p.D < 128) {
      hipLaunchKernelGGL((decode_f32_kernel<P, 2, false>), grid, block, 0, stream, a);
    } else {
      hipLaunchKernelGGL((decode_f32_kernel<P, 4, false>), grid, block, 0, stream, a);
    }
  };
  if (p.table) go(std::true_type{});
  else go(std::false_type{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)p.B * p.Hkv * p.R;
  auto join = [&](auto f32) {
    constexpr bool F = decltype(f32)::value;
    if (rows <= 1024) hipLaunchKernelGGL((decode_join_kernel<F, 8>), dim3((unsigned)rows), dim3(8 * kWave), 0, stream, a);
    else {
      const int64_t wgs = (rows + 3) / 4;
      hipLaunchKernelGGL((decode_join_kernel<F, 1>), dim3((unsigned)(wgs < 8192 ? wgs : 8192)), dim3(kThreads), 0, stream, a);
    }
  };
  if (p.is_f32) join(std::true_type{});
  else join(std::false_type{});
  return hipGetLastError();
}

}  // namespace ac
