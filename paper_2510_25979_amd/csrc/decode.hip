// Attention of few rows over many keys: one new token of each request over its pages, or a few query rows over an
// encoder's states.  O = softmax(scale Q K^T) V for the R rows of each (item b, K/V head), which lie side by side in Q and
// O (the g heads that share K and V, times their rows); keys j < len[b] are seen.
//
// Each byte of K and V serves few products (2 R flop a byte in bf16), so memory bounds it, and the keys of all requests have
// to be in flight on all compute units, however long or short each request is.
//
// decode_run_kernel cuts the work by keys, not by requests.  A unit is 16 rows of one (item, K/V head), cut into blocks of 32 keys
// (16 in binary32); all units' blocks form one row, and each of a fixed number of waves takes an equal run of it, which it
// finds from the lengths by itself.  Ending one unit and beginning the next counts as kUnitCost further blocks.  A run covers the end of
// one unit, some whole ones and the beginning of another: whole units leave as output, the at most two others as partial results (row
// maximum, sum, sum of weighted V, binary32), which decode_join_kernel adds up.  So the workspace does not grow with the lengths, and the host
// need not know them.  Waves share nothing and never meet; the next block's rows, pages and queries are on their way over the end of
// a unit, too.
//
// decode_unit_kernel gives each unit to a workgroup, whose waves deal out the blocks and meet in LDS: one launch and no workspace,
// where no unit can be large (the rule is at the launch).
//
// A wave's block: K rows go straight from memory to the lanes that multiply them (S^T = K Q^T, 16 keys x 16 rows a product), V rows
// through a wave-private LDS tile where the transposing read wants them (O^T = V^T P^T; binary32: straight from memory).  A lane
// deals with one row of Q, so maximum and sum are in-lane but for the four lanes that share it, and the weights are where the
// second product takes them.  Pages may end anywhere inside a block: each lane follows its own keys' pages.
#include <type_traits>

#include "common.hpp"
#include "f32_tile.hpp"
#include "serve.h"
#include "serve_index.h"

namespace ac {

constexpr int kDecodeRows = 16;        // rows of a unit
constexpr int kUnitCost = 2;           // what a unit costs beside its blocks, in blocks
constexpr int kDecodeWaves = 4 * 512;  // most waves of decode_run_kernel, what the workspace is sized for
constexpr float kDecodeSlack = 8.0f;   // as in exact attention: the reference point of a row moves when it is outgrown by 2^8

struct DecodeArgs {
  const void *Q, *K, *V;
  void* O;
  const int32_t *table, *len, *row_sel;
  float *part, *stat;   // partial results [2 waves][rp][D] and their (maximum, sum) [2 waves][rp][2]
  int32_t B, Hkv, R, rbs, rp, D, Sk;   // rbs: row blocks of a K/V head; rp: rows of a partial result
  int32_t n_pages, ps, max_pages, waves, join_rows;   // join_rows: output rows of a wave of the join
  int64_t page_stride, head_stride;
  Divider by_ps, by_rbs;
  float scale_log2e;
};

__device__ __forceinline__ int decode_keys(const DecodeArgs& a, int b) {
  if (a.row_sel && a.row_sel[b] >= 0) return 0;
  return a.len ? min(max(a.len[b], 0), a.Sk) : a.Sk;
}

// The same for a b that all lanes share: scalar loads, which the compiler does not take by itself in a kernel that writes, and
// which wait for no copy that is under way.
__device__ __forceinline__ int decode_keys_of(const DecodeArgs& a, int b) {
  typedef const int32_t __attribute__((address_space(4)))* scalar_ptr;
  b = __builtin_amdgcn_readfirstlane(b);
  if (a.row_sel && ((scalar_ptr)(uintptr_t)a.row_sel)[b] >= 0) return 0;
  return a.len ? min(max(((scalar_ptr)(uintptr_t)a.len)[b], 0), a.Sk) : a.Sk;
}

// How the blocks of all units are numbered and dealt: item by item, in it K/V head, row block, key block.
template <int BK>
struct DecodeWalk {
  const DecodeArgs& a;
  int lane, units, head, per, total;   // units of an item; costs of the first 64 items up to this lane's
  __device__ __forceinline__ int cost(int b) const {   // of a unit of item b
    const int keys = b < a.B ? decode_keys(a, b) : 0;
    return keys ? (keys + BK - 1) / BK + kUnitCost : 0;
  }
  __device__ __forceinline__ int upto(int t) const {   // sum over the lanes up to this one
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int p = __shfl_up(t, off);
      if (lane >= off) t += p;
    }
    return t;
  }
  // costs of the items from 64 to `end`
  __device__ __forceinline__ int further(int end) const {
    int t = 0;
    for (int b = kWave + lane; b < end; b += kWave) t += cost(b);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
    return __builtin_amdgcn_readfirstlane(t);
  }
  __device__ __forceinline__ DecodeWalk(const DecodeArgs& a, int lane) : a(a), lane(lane), units(a.Hkv * a.rbs) {
    head = upto(cost(lane));
    int t = __builtin_amdgcn_readlane(head, kWave - 1);
    if (a.B > kWave) t += further(a.B);
    total = t * units;
    per = run_length(total, a.waves);
  }
  // number of the first block of item `item`
  __device__ __forceinline__ int start(int item) const {
    if (item == 0) return 0;
    if (item <= kWave) return __builtin_amdgcn_readlane(head, item - 1) * units;
    return (__builtin_amdgcn_readlane(head, kWave - 1) + further(item)) * units;
  }
  // the item that block x < total belongs to; x becomes the block's number in it
  __device__ __forceinline__ int locate(int& x) const {
    int before = 0, t = head;
    for (int b0 = 0;; b0 += kWave) {
      const unsigned long long beyond = __ballot(x < before + t * units);
      if (beyond || b0 + kWave >= a.B) {
        const int i = beyond ? __builtin_ctzll(beyond) : 0;
        x = __builtin_amdgcn_readfirstlane(x) - before - (i > 0 ? __builtin_amdgcn_readlane(t, i - 1) * units : 0);
        return b0 + i;
      }
      before += __builtin_amdgcn_readlane(t, kWave - 1) * units;
      t = upto(cost(b0 + kWave + lane));
    }
  }
};

// Where the K and V row of key j of an item with `keys` keys lies, in elements from its head's first row of the first page (or of
// the item); -1 where there is none.  Two steps, so that the page number can be asked for early.
template <bool PAGED>
__device__ __forceinline__ int decode_ask(const DecodeArgs& a, int b, int keys, int j) {
  return PAGED && j < keys ? a.table[(size_t)b * a.max_pages + a.by_ps.div(j)] : 0;
}
template <bool PAGED>
__device__ __forceinline__ int64_t decode_at(const DecodeArgs& a, int keys, int j, int page, int D) {
  if (j >= keys) return -1;
  if (!PAGED) return (int64_t)j * D;
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return page * a.page_stride + (int64_t)(j - a.by_ps.div(j) * a.ps) * D;
}

// max over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float max_of_four(float x) {
  float lo = x, hi = x;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(lo), "+v"(hi));
  return max_with_other_half(fmaxf(lo, hi));
}
// LDS operations of one wave execute in order: only the compiler has to keep them so.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ float sum_of_four(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The work of a wave on one block.  Lane = (i, kq) = (lane % 16, lane / 16); i is its row of Q.  Results: NP pieces of four
// consecutive columns of row i, piece n from column col(n).
template <int D_>
struct DecodeBf16 {
  typedef bf16_t Elt;
  static constexpr int BK = 32, KPL = 2, NP = D_ / 16, KS = D_ / 32;   // keys of a block, of a lane; pieces
  static constexpr int OCC = 3, WGS = 2;   // waves of a SIMD the unit kernel is built for; workgroups of a compute unit with runs
  static constexpr int LDS = 32 * D_ * 2;                                      // bytes of the wave's V tile
  struct Query { u32x4 r[KS]; };
  u32x4 k[2][KS], v[2][KS];
  f32x4 acc[NP];
  float m, l;
  bf16_t* vt;
  int lane, i, kq;

  __device__ __forceinline__ DecodeBf16(const DecodeArgs&, unsigned char* lds, int lane)
      : vt(reinterpret_cast<bf16_t*>(lds)), lane(lane), i(lane & 15), kq(lane >> 4) {}
  __device__ __forceinline__ int dim() const { return D_; }
  __device__ __forceinline__ int col(int n) const { return 16 * n + 4 * kq; }
  __device__ __forceinline__ int key(int t) const { return 16 * t + i; }   // the lane's keys of a block
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NP; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void load_q(Query& q, const Elt* rows, int n_rows) const {
    const Elt* src = rows + (size_t)min(i, n_rows - 1) * D_ + 8 * kq;
#pragma unroll
    for (int s = 0; s < KS; ++s) q.r[s] = *reinterpret_cast<const u32x4*>(src + 32 * s);
  }
  __device__ __forceinline__ void rows_of(u32x4 (&r)[2][KS], const Elt* base, const int64_t (&at)[2]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Elt* src = base + (at[t] < 0 ? 0 : at[t]) + 8 * kq;   // (row 0: there, and not used)
#pragma unroll
      for (int s = 0; s < KS; ++s) r[t][s] = *reinterpret_cast<const u32x4*>(src + 32 * s);
    }
  }
  __device__ __forceinline__ void load_k(const Elt* base, const int64_t (&at)[2]) { rows_of(k, base, at); }
  __device__ __forceinline__ void load_v(const Elt* base, const int64_t (&at)[2]) { rows_of(v, base, at); }
  // scores^T: keys 16 t + 4 kq + x of row i
  typedef f32x4 Scores[2];
  __device__ __forceinline__ void scores(Scores& s, const Query& q) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KS; ++c)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][c]),
                                                       __builtin_bit_cast(bf16x8, q.r[c]), s[t], 0, 0, 0);
    }
  }
  // Position of piece p of row r in the V tile: sixteen rows of a write, and eight rows of a transposing read of two pieces
  // each, fall on different banks.
  static __device__ __forceinline__ int piece(int r) {
    return D_ == 128 ? 4 * (r & 3) ^ 2 * ((r >> 2) & 1) ^ ((r >> 3) & 1) : 2 * ((r >> 1) & 3) ^ ((r >> 3) & 1);
  }
  // Rows that are not there: no score, and zeros in V, since a weight of zero does not make a NaN vanish.
  __device__ __forceinline__ void hide(Scores& s, const int64_t (&at)[2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t seen = (uint32_t)__ballot(at[t] >= 0);
      if ((seen & 0xffff) != 0xffff) {
#pragma unroll
        for (int c = 0; c < KS; ++c)
          if (at[t] < 0) v[t][c] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (!((seen >> (4 * kq + x)) & 1)) s[t][x] = -INFINITY;
      }
    }
  }
  __device__ __forceinline__ void stage_v() const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KS; ++c)
        *reinterpret_cast<u32x4*>(vt + key(t) * D_ + 8 * ((4 * c + kq) ^ piece(i))) = v[t][c];
  }
  __device__ __forceinline__ void add(Scores& s, float scale_log2e) {
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                     fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    const float cand = fmaxf(m, max_of_four(mx) * scale_log2e);
    if (__any(cand > m + kDecodeSlack)) {
      const float alpha = cand > m ? __builtin_amdgcn_exp2f(m - cand) : 1.f;
      l *= alpha;
#pragma unroll
      for (int n = 0; n < NP; ++n) acc[n] *= alpha;
      m = cand;
    }
    const float ref = m == -INFINITY ? 0.f : m;   // no finite score so far: all weights are zero
    typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
    u32x4 p;
    // Weights are rounded to bf16: the matrix product takes both factors in one type, and V is bf16; two halves a weight would double it.
    // The sum is over the rounded ones, which V is multiplied with, so that they still add up to one.  Against 64 bits results are off by
    // 0.0020 to 0.0023 of their size (root mean square, the measured cases), by 0.0017 from their own rounding alone.
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[w >> 1][2 * (w & 1)], scale_log2e, -ref));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s[w >> 1][2 * (w & 1) + 1], scale_log2e, -ref));
      const uint32_t pk = pack_bf16(e0, e1);
      p[w] = pk;
      l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, l, false);
    }
    // contraction slot e of lane quarter kq is key 16 (e / 4) + 4 kq + e % 4, where the first product left the scores; lane i of a
    // group of 16 names key 4 kq + i / 4 and four columns, and receives its own column of the four keys
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      s16x4 w[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int j = 4 * kq + (i >> 2), d0 = 16 * n + 4 * (i & 3);
        w[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(
            vt + (16 * t + j) * D_ + 8 * ((d0 >> 3) ^ piece(j)) + (d0 & 7)));
      }
      const s16x8 vop = {w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]};
      acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop), __builtin_bit_cast(bf16x8, p), acc[n], 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void store(Elt* to, const f32x4 r, float inv, int, int) {
    *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(r[0] * inv, r[1] * inv), pack_bf16(r[2] * inv, r[3] * inv)};
  }
};

// Binary32, D <= 64 DB.  A row that is no whole number of 16-byte pieces is read in pieces of four that start at any 4-byte
// address, its end in single floats.
template <int DB, bool FULL>   // FULL: D == 64 DB
struct DecodeF32 {
  typedef float Elt;
  static constexpr int BK = 16, KPL = 1, NP = 4 * DB, OCC = DB <= 2 ? 2 : 1, WGS = 1;
  static constexpr int LDS = 0;
  struct Query { f32x4 r[4 * DB]; };
  f32x4 k[4 * DB], v[4][DB];
  f32x4 acc[4 * DB];   // [4 b + c][x]: column 64 b + 16 kq + 4 x + c
  float m, l;
  int D, lane, i, kq;

  __device__ __forceinline__ DecodeF32(const DecodeArgs& a, unsigned char*, int lane)
      : D(FULL ? 64 * DB : a.D), lane(lane), i(lane & 15), kq(lane >> 4) {}
  __device__ __forceinline__ int dim() const { return FULL ? 64 * DB : D; }
  __device__ __forceinline__ int col(int n) const { return 64 * (n >> 2) + 16 * kq + 4 * (n & 3); }
  __device__ __forceinline__ int key(int) const { return i; }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < 4 * DB; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ f32x4 four(const float* row, int c) const {   // columns c ... c + 3, zeros behind the row's end
    if (FULL) return *reinterpret_cast<const f32x4*>(row + c);
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (c + 4 <= D) {
      r = *reinterpret_cast<const f32x4_dw*>(row + c);
    } else {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (c + t < D) r[t] = row[c + t];
    }
    return r;
  }
  __device__ __forceinline__ void load_q(Query& q, const Elt* rows, int n_rows) const {
    const float* src = rows + (size_t)min(i, n_rows - 1) * dim();
#pragma unroll
    for (int s = 0; s < 4 * DB; ++s) q.r[s] = four(src, 16 * s + 4 * kq);
  }
  __device__ __forceinline__ void load_k(const Elt* base, const int64_t (&at)[1]) {
    const float* src = base + (at[0] < 0 ? 0 : at[0]);
#pragma unroll
    for (int s = 0; s < 4 * DB; ++s) k[s] = four(src, 16 * s + 4 * kq);
  }
  // columns 64 b + 4 i and three more of keys 4 kq ... 4 kq + 3; zeros if they are not there
  __device__ __forceinline__ void load_v(const Elt* base, const int64_t (&at)[1]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t from = __shfl((long long)at[0], 4 * kq + t);
      const float* src = base + (from < 0 ? 0 : from);
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        v[t][b] = four(src, 64 * b + 4 * i);
        if (from < 0) v[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  }
  typedef f32x4 Scores[1];
  __device__ __forceinline__ void scores(Scores& s, const Query& q) const {
    s[0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4 * DB; ++c)
      if (FULL || 16 * c < D)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[0] = mfma_f32(k[c][t], q.r[c][t], s[0]);
  }
  __device__ __forceinline__ void hide(Scores& s, const int64_t (&at)[1]) {
    const uint32_t seen = (uint32_t)__ballot(at[0] >= 0) >> (4 * kq);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (!((seen >> x) & 1)) s[0][x] = -INFINITY;
  }
  __device__ __forceinline__ void stage_v() const {}
  __device__ __forceinline__ void add(Scores& s, float scale_log2e) {
    const float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
    const float m_new = fmaxf(m, max_of_four(mx) * scale_log2e);
    if (__any(m_new > m)) {
      const float alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
      l *= alpha;
#pragma unroll
      for (int n = 0; n < 4 * DB; ++n) acc[n] *= alpha;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    f32x4 p;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      p[x] = __builtin_amdgcn_exp2f(fmaf(s[0][x], scale_log2e, -ref));
      l += p[x];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[4 * b + c] = mfma_f32(v[x][b][c], p[x], acc[4 * b + c]);
  }
  static __device__ __forceinline__ void store(Elt* to, f32x4 r, float inv, int d, int D) {
#pragma unroll
    for (int t = 0; t < 4; ++t) r[t] *= inv;
    if (FULL || d + 4 <= D) {
      *reinterpret_cast<f32x4_dw*>(to) = r;
    } else {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (d + t < D) to[t] = r[t];
    }
  }
};
// piece n of a lane's results
template <int D>
__device__ __forceinline__ f32x4 decode_piece(const DecodeBf16<D>& c, int n) { return c.acc[n]; }
template <int DB, bool FULL>
__device__ __forceinline__ f32x4 decode_piece(const DecodeF32<DB, FULL>& c, int n) {
  const int b = n >> 2, x = n & 3;
  return f32x4{c.acc[4 * b][x], c.acc[4 * b + 1][x], c.acc[4 * b + 2][x], c.acc[4 * b + 3][x]};
}
__device__ __forceinline__ void store_partial(float* to, const f32x4 r, int d, int D) {
  if (d + 4 <= D) *reinterpret_cast<f32x4_dw*>(to) = r;
  else
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (d + t < D) to[t] = r[t];
}

// A block of a run: its item, unit of the item and number in the unit, and what is left of the run from it on.
struct DecodeItem {
  int b, unit, blk, keys, nb, left;
};

template <class Core, bool PAGED>
__global__ __launch_bounds__(kThreads, Core::WGS) void decode_run_kernel(const DecodeArgs a) {
  typedef typename Core::Elt Elt;
  constexpr int BK = Core::BK, KPL = Core::KPL;
  __shared__ __attribute__((aligned(16))) unsigned char lds[Core::LDS ? 4 * Core::LDS : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int run = blockIdx.x * 4 + wave;
  const DecodeWalk<BK> walk(a, lane);
  if (run >= a.waves) return;
  int x = run * walk.per;
  if (x >= walk.total) return;
  Core core(a, lds + wave * Core::LDS, lane);
  const int D = core.dim();

  auto item = [&](DecodeItem& it, int b) {   // the first block of the first item from b on that has any (there is one)
    int keys = decode_keys_of(a, b);
    while (keys == 0 && b + 1 < a.B) {   // (64 a step: millions of items may have none)
      const int other = b + 1 + lane;
      const unsigned long long some = __ballot(other < a.B && decode_keys(a, other) > 0);
      b = some ? b + 1 + (int)__builtin_ctzll(some) : min(b + kWave, a.B - 1);
      keys = decode_keys_of(a, b);
    }
    it.b = b;
    it.unit = 0;
    it.keys = keys;
    it.nb = (keys + BK - 1) / BK;
  };
  auto next = [&](DecodeItem& it) {   // false: the run ends
    const bool last = it.blk + 1 == it.nb;
    it.left -= last ? 1 + kUnitCost : 1;
    it.blk = last ? 0 : it.blk + 1;
    it.unit += last ? 1 : 0;
    if (it.unit == walk.units && it.left > 0) item(it, it.b + 1);
    return it.left > 0;
  };
  DecodeItem now, then, later;
  {
    const int left = min(walk.per, walk.total - x);
    item(now, walk.locate(x));
    now.left = left;
    now.unit = x / (now.nb + kUnitCost);
    now.blk = x - now.unit * (now.nb + kUnitCost);
    if (now.blk >= now.nb) {   // behind a unit's last block
      now.left -= now.nb + kUnitCost - now.blk - 1;
      now.blk = now.nb - 1;
      now.left += kUnitCost;
      if (!next(now)) return;
    }
  }
  auto ask = [&](const DecodeItem& it, int(&page)[KPL]) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) page[t] = decode_ask<PAGED>(a, it.b, it.keys, BK * it.blk + core.key(t));
  };
  auto place = [&](const DecodeItem& it, const int(&page)[KPL], int64_t(&at)[KPL]) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) at[t] = decode_at<PAGED>(a, it.keys, BK * it.blk + core.key(t), page[t], D);
  };
  auto base_of = [&](const void* p, const DecodeItem& it) {
    const int hk = a.by_rbs.div(it.unit);
    return static_cast<const Elt*>(p) + (PAGED ? (size_t)hk : (size_t)it.b * a.Hkv + hk) * a.head_stride;
  };
  // the unit's first row in Q and O, and how many there are
  auto rows_of = [&](const DecodeItem& it, size_t& row0) {
    const int hk = a.by_rbs.div(it.unit), r0 = kDecodeRows * (it.unit - hk * a.rbs);
    row0 = ((size_t)it.b * a.Hkv + hk) * a.R + r0;
    return min(kDecodeRows, a.R - r0);
  };
  auto load_q = [&](typename Core::Query& q, const DecodeItem& it) {
    size_t row0;
    const int rows = rows_of(it, row0);
    core.load_q(q, static_cast<const Elt*>(a.Q) + row0 * D, rows);
  };

  typename Core::Query q, q_then;
  int page[KPL];
  int64_t at[KPL], at_then[KPL];
  ask(now, page);
  load_q(q, now);
  then = now;
  bool more = next(then);
  place(now, page, at);
  core.load_k(base_of(a.K, now), at);
  core.load_v(base_of(a.V, now), at);
  if (more) ask(then, page);
  core.reset();
  int begin = now.blk;
  while (true) {
    typename Core::Scores s;
    core.scores(s, q);
    const bool last = now.blk + 1 == now.nb;   // of its unit
    later = then;
    bool more_later = false;
    if (more) {
      place(then, page, at_then);
      if (last) load_q(q_then, then);
      core.load_k(base_of(a.K, then), at_then);
      more_later = next(later);
      if (more_later) ask(later, page);
    }
    core.hide(s, at);
    core.stage_v();
    if (Core::LDS && more) core.load_v(base_of(a.V, then), at_then);
    if (Core::LDS) wave_fence();
    core.add(s, a.scale_log2e);
    if (Core::LDS) wave_fence();   // the tile is read before the next block's rows are written
    if (!Core::LDS && more) core.load_v(base_of(a.V, then), at_then);
    if (last || !more) {
      const float sum = sum_of_four(core.l);
      size_t row0;
      const int rows = rows_of(now, row0);
      const bool whole = begin == 0 && last;
      const size_t slot = (size_t)(2 * run + (begin == 0)) * a.rp;   // as partial_of has it
      if (core.i < rows) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // no key at all: zeros
        Elt* o = static_cast<Elt*>(a.O) + (row0 + core.i) * D;
#pragma unroll
        for (int n = 0; n < Core::NP; ++n) {
          const int d = core.col(n);
          if (whole) Core::store(o + d, decode_piece(core, n), inv, d, D);
          else store_partial(a.part + (slot + core.i) * D + d, decode_piece(core, n), d, D);
        }
        if (!whole && core.kq == 0) {
          a.stat[2 * (slot + core.i)] = core.m;
          a.stat[2 * (slot + core.i) + 1] = sum;
        }
      }
      if (!more) break;
      core.reset();
      q = q_then;
      begin = 0;
    }
    now = then;
    then = later;
    more = more_later;
#pragma unroll
    for (int t = 0; t < KPL; ++t) at[t] = at_then[t];
  }
}

// A workgroup per unit, its waves deal out the blocks.
template <class Core, bool PAGED, int NW>
__global__ __launch_bounds__(NW* kWave, Core::OCC) void decode_unit_kernel(const DecodeArgs a) {
  typedef typename Core::Elt Elt;
  constexpr int BK = Core::BK, KPL = Core::KPL, NP = Core::NP;
  constexpr int TILES = NW * Core::LDS, SUMS = NW * NP * kWave * 16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[TILES > SUMS ? TILES : SUMS];
  __shared__ float ms[NW][kDecodeRows], ls[NW][kDecodeRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the row blocks of a head are workgroups with ids equal mod 8 (one XCD): K and V come from its L2 after the first
  const int slot = blockIdx.x >> 3, group = a.by_rbs.div(slot), rb = slot - group * a.rbs;
  const int head = a.rbs == 1 ? blockIdx.x : 8 * group + (blockIdx.x & 7);
  if (head >= a.B * a.Hkv) return;
  const int b = head / a.Hkv, hk = head - b * a.Hkv;
  if (a.row_sel && a.row_sel[b] >= 0) return;
  const int keys = decode_keys_of(a, b), nb = (keys + BK - 1) / BK;
  Core core(a, lds + wave * Core::LDS, lane);
  const int D = core.dim(), i = core.i, rows = min(kDecodeRows, a.R - kDecodeRows * rb);
  const size_t row0 = (size_t)head * a.R + kDecodeRows * rb;
  const Elt* K = static_cast<const Elt*>(a.K) + (PAGED ? (size_t)hk : (size_t)head) * a.head_stride;
  const Elt* V = static_cast<const Elt*>(a.V) + (PAGED ? (size_t)hk : (size_t)head) * a.head_stride;
  typename Core::Query q;
  int page[KPL];
  int64_t at[KPL], at_then[KPL];
  auto ask = [&](int blk) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) page[t] = decode_ask<PAGED>(a, b, keys, BK * blk + core.key(t));
  };
  auto place = [&](int blk, int64_t(&to)[KPL]) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) to[t] = decode_at<PAGED>(a, keys, BK * blk + core.key(t), page[t], D);
  };
  core.reset();
  int blk = wave;
  if (blk < nb) {
    ask(blk);
    core.load_q(q, static_cast<const Elt*>(a.Q) + row0 * D, rows);
    place(blk, at);
    core.load_k(K, at);
    core.load_v(V, at);
    if (blk + NW < nb) ask(blk + NW);
  }
  for (; blk < nb; blk += NW) {
    typename Core::Scores s;
    core.scores(s, q);
    const bool more = blk + NW < nb;
    if (more) {
      place(blk + NW, at_then);
      core.load_k(K, at_then);
      if (blk + 2 * NW < nb) ask(blk + 2 * NW);
    }
    core.hide(s, at);
    core.stage_v();
    if (Core::LDS && more) core.load_v(V, at_then);
    if (Core::LDS) wave_fence();
    core.add(s, a.scale_log2e);
    if (Core::LDS) wave_fence();
    if (!Core::LDS && more) core.load_v(V, at_then);
#pragma unroll
    for (int t = 0; t < KPL; ++t) at[t] = at_then[t];
  }
  const float l = sum_of_four(core.l);
  if (core.kq == 0) {
    ms[wave][i] = core.m;
    ls[wave][i] = l;
  }
  __syncthreads();   // statistics are there, V tiles are no longer read
  f32x4* sums = reinterpret_cast<f32x4*>(lds);
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[w][i]);
  auto factor = [&](float mw) { return mw < top ? __builtin_amdgcn_exp2f(mw - top) : 1.f; };
#pragma unroll
  for (int w = 0; w < NW; ++w) sum = fmaf(ls[w][i], factor(ms[w][i]), sum);
  const float mine = factor(core.m);
  if (i < rows)
#pragma unroll
    for (int n = 0; n < NP; ++n) sums[(wave * NP + n) * kWave + lane] = decode_piece(core, n) * mine;
  __syncthreads();
  if (i < rows) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int n = wave; n < NP; n += NW) {
      f32x4 r = sums[n * kWave + lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) r += sums[(w * NP + n) * kWave + lane];
      const int d = core.col(n);
      Core::store(static_cast<Elt*>(a.O) + (row0 + i) * D + d, r, inv, d, D);
    }
  }
}

// The rows of units that several waves shared, and zeros for rows without a key.  NW waves add up one output row: its partial
// results are those of the waves whose runs touch its unit, dealt to the waves here in turn.  A lane holds four columns, G lanes a
// partial result; a wave knows the weights of 64 of them at once, one a lane.  Bound by latency: lengths -> statistics -> sums.
template <bool F32, int G, int NW>
__global__ __launch_bounds__(NW == 1 ? kThreads : NW * kWave) void decode_join_kernel(const DecodeArgs a) {
  typedef typename std::conditional<F32, float, bf16_t>::type Elt;
  constexpr int BK = F32 ? 16 : 32, SUB = kWave / G;
  __shared__ __attribute__((aligned(16))) f32x4 sums[NW][G];
  __shared__ float ms[NW], ls[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = lane / G, d = 4 * (lane % G), D = a.D;
  const DecodeWalk<BK> walk(a, lane);
  const int n_rows = a.B * a.Hkv * a.R;   // of all items
  // A wave has consecutive rows and goes from item to item with them: it looks through the items before its first row once, not for each.
  const int mine = NW == 1 ? blockIdx.x * (kThreads / kWave) + wave : blockIdx.x, each = NW == 1 ? a.join_rows : 1;
  const int row0 = mine * each;
  int item = -1, first_block = -1, cost = 0;   // first_block: the item's, -1 until one is asked for; cost of its units
  for (int row = row0; row < min(n_rows, row0 + each); ++row) {
    const int head = row / a.R, r = row - head * a.R, b = head / a.Hkv, hk = head - b * a.Hkv;
    const int keys = decode_keys_of(a, b), nb = (keys + BK - 1) / BK;
    if (b != item && first_block >= 0) first_block += cost * walk.units;
    item = b;
    cost = keys ? nb + kUnitCost : 0;
    if (a.row_sel && a.row_sel[b] >= 0) continue;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;
    if (keys > 0) {
      if (first_block < 0) first_block = walk.start(b);
      const int from = first_block + (hk * a.rbs + r / kDecodeRows) * cost;
      const int w0 = from / walk.per, w1 = (from + nb - 1) / walk.per;
      if (w0 == w1) continue;   // one wave had all of it
      const int first = w0 + (NW == 1 ? 0 : wave);
      for (int w = first; w <= w1; w += NW * kWave) {
        const size_t slot = (size_t)partial_of(min(w + NW * lane, w1), walk.per, from) * a.rp + r % kDecodeRows;
        float m = -INFINITY, l = 0.f;
        if (w + NW * lane <= w1) {
          m = a.stat[2 * slot];
          l = a.stat[2 * slot + 1];
        }
        float t = fmaxf(top, m);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) t = fmaxf(t, __shfl_xor(t, off));
        const float old = top < t ? __builtin_amdgcn_exp2f(top - t) : 1.f, f = m < t ? __builtin_amdgcn_exp2f(m - t) : 1.f;
        top = t;
        total *= old;
        o *= old;
        l *= f;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
        total += l;
        const int n = min(kWave, (w1 - w) / NW + 1);
        for (int k0 = 0; k0 < n; k0 += 4 * SUB) {   // four loads of a lane on their way at once
          f32x4 x[4];
          float weight[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int k = k0 + j * SUB + sub, from_lane = min(k, n - 1);
            const float w_j = __shfl(f, from_lane);
            weight[j] = k < n ? w_j : 0.f;
            const float* src = a.part + (size_t)__shfl((int)slot, from_lane) * D + d;
            x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (k >= n || d >= D) continue;
            if (!F32 || d + 4 <= D) {
              x[j] = *reinterpret_cast<const f32x4_dw*>(src);
            } else {
#pragma unroll
              for (int c = 0; c < 3; ++c)
                if (d + c < D) x[j][c] = src[c];
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) o += x[j] * weight[j];
        }
      }
#pragma unroll
      for (int off = G; off < kWave; off <<= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] += __shfl_xor(o[c], off);
      if (NW > 1) {
        if (lane < G) sums[wave][lane] = o;
        if (lane == 0) {
          ms[wave] = top;
          ls[wave] = total;
        }
        __syncthreads();
        if (wave == 0) {
          for (int w = 1; w < NW; ++w) top = fmaxf(top, ms[w]);
          total = 0.f;
          o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < NW; ++w) {
            const float f = ms[w] < top ? __builtin_amdgcn_exp2f(ms[w] - top) : 1.f;
            total = fmaf(ls[w], f, total);
            o += sums[w][lane % G] * f;
          }
        }
      }
    }
    if (wave == 0 || NW == 1) {
      if (sub == 0 && d < D) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        Elt* to = static_cast<Elt*>(a.O) + (size_t)row * D + d;
        if constexpr (F32) store_partial(to, o * inv, d, D);
        else DecodeBf16<64>::store(to, o, inv, d, D);
      }
    }
    if (NW > 1) __syncthreads();
  }
}

size_t decode_workspace_bytes(int32_t R, int32_t D) {
  return (size_t)2 * kDecodeWaves * (R < kDecodeRows ? R : kDecodeRows) * (D + 2) * sizeof(float);
}
bool decode_fits(int64_t B, int64_t Hkv, int64_t R, int64_t keys) {
  // blocks of 16 rows and 16 keys (binary32, the smaller ones), and the rows themselves; keys <= 2^30, so their numbers are far from the end
  const double units = (double)B * Hkv * ((R + kDecodeRows - 1) / kDecodeRows);
  return units * ((keys + 15) / 16 + kUnitCost) < 2147483648.0 - 65536 && (double)B * Hkv * R < 2147483648.0 - 65536;
}

template <class Core, bool PAGED>
static hipError_t launch_decode_core(DecodeArgs& a, hipStream_t stream) {
  constexpr bool F32 = Core::BK == 16;
  const int64_t units = (int64_t)a.B * a.Hkv * a.rbs, rows = (int64_t)a.B * a.Hkv * a.R;
  const int blocks = (int)(((int64_t)a.Sk + Core::BK - 1) / Core::BK);   // the most of a unit
  // One launch where no unit can be large: it is then over before a second launch would be.  Up to 256 KB of K and V, what one compute unit
  // reads in the time of that launch, 512 KB where there are 128 units, 64 blocks where there are units for the whole chip.  us, runs and
  // join / units, bf16 on pages: 4 x 8 heads of 64, up to 1,008 tokens (256 KB) 8.8 / 8.4, up to 2,000 9.8 / 12.3; of 128, up to 500 (250 KB) 9.9 /
  // 9.3, up to 700 9.9 / 11.0; 64 units of 128, 500 tokens 13.2 / 11.6, 1,000 17.1 / 19.1; 128 units, 1,000 (512 KB) 21.2 / 19.4, 2,000 31.9 /
  // 33.2; 256 units, 2,000 (63 blocks) 65.9 / 49.4; 1,024 units, 128 to 4,096 tokens (128) 129 / 156, all 4,000 711 / 685; binary32, 32 units of 128,
  // 200 tokens (208 KB) 10.5 / 11.0, 500 13.4 / 19.1.  Eight waves a unit / four: the first 8.5 / 9.2, 128 units 19.5 / 19.7, 512 units of 500
  // tokens 26.3 / 23.2.  The host knows the most keys an item can have, not how many it has: 256 units of 2,000 tokens take 49.4 in a table
  // of up to 2,048 tokens and 65.9 in a wider one.  Binary32 units of 200 tokens (208 KB) are on the wrong side by 5 %.
  const int64_t unit_bytes = 2LL * blocks * Core::BK * a.D * (int64_t)sizeof(typename Core::Elt);
  const bool small = units >= 256 ? blocks <= 64 : unit_bytes <= (units >= 128 ? 512 : 256) * 1024;
  if (small && units <= (1 << 22)) {
    const int64_t heads = (int64_t)a.B * a.Hkv;
    const dim3 grid((unsigned)(a.rbs == 1 ? heads : (heads + 7) / 8 * 8 * a.rbs));
    if constexpr (Core::NP <= 8)
      if (units <= 128) {
        hipLaunchKernelGGL((decode_unit_kernel<Core, PAGED, 8>), grid, dim3(8 * kWave), 0, stream, a);
        return hipGetLastError();
      }
    hipLaunchKernelGGL((decode_unit_kernel<Core, PAGED, 4>), grid, dim3(4 * kWave), 0, stream, a);
    return hipGetLastError();
  }
  a.waves = 4 * 256 * Core::WGS;
  hipLaunchKernelGGL((decode_run_kernel<Core, PAGED>), dim3((unsigned)(a.waves / 4)), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // waves of an output row: 32 rows of 64 partial results each take eight, thousands of two or three one (1,024 rows with eight 9.3 us
  // of launching waves, 2,048 with one 5.4)
  constexpr int G = Core::NP * 4;
  if (rows <= 256) {
    hipLaunchKernelGGL((decode_join_kernel<F32, G, 8>), dim3((unsigned)rows), dim3(8 * kWave), 0, stream, a);
  } else if (rows <= 1024) {
    hipLaunchKernelGGL((decode_join_kernel<F32, G, 4>), dim3((unsigned)rows), dim3(4 * kWave), 0, stream, a);
  } else {
    a.join_rows = rows_of_a_wave((int)rows, 4 * 8192);
    const int64_t waves = (rows + a.join_rows - 1) / a.join_rows;
    hipLaunchKernelGGL((decode_join_kernel<F32, G, 1>), dim3((unsigned)((waves + 3) / 4)), dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_decode(const DecodeLaunch& p, hipStream_t stream) {
  DecodeArgs a;
  a.Q = p.Q; a.K = p.K; a.V = p.V; a.O = p.O; a.table = p.table; a.len = p.len; a.row_sel = p.row_sel;
  a.B = p.B; a.Hkv = p.Hkv; a.R = p.R; a.D = p.D; a.Sk = p.Sk;
  a.rbs = (p.R + kDecodeRows - 1) / kDecodeRows;
  a.rp = p.R < kDecodeRows ? p.R : kDecodeRows;
  a.n_pages = p.n_pages; a.ps = p.page_size; a.max_pages = p.max_pages; a.page_stride = p.page_stride;
  a.head_stride = (int64_t)(p.table ? p.page_size : p.Sk) * p.D;
  a.by_ps = Divider((uint32_t)(p.table ? p.page_size : 1));
  a.by_rbs = Divider((uint32_t)a.rbs);
  const float scale = p.scale == 0.f ? 1.0f / sqrtf((float)p.D) : p.scale;
  a.scale_log2e = scale * 1.44269504088896340736f;
  a.waves = 0;
  a.join_rows = 1;
  a.stat = static_cast<float*>(p.ws);
  a.part = a.stat + (size_t)2 * kDecodeWaves * a.rp * 2;
  auto go = [&](auto paged) {
    constexpr bool P = decltype(paged)::value;
    if (!p.is_f32)
      return p.D == 64 ? launch_decode_core<DecodeBf16<64>, P>(a, stream) : launch_decode_core<DecodeBf16<128>, P>(a, stream);
    if (p.D == 64) return launch_decode_core<DecodeF32<1, true>, P>(a, stream);
    if (p.D == 128) return launch_decode_core<DecodeF32<2, true>, P>(a, stream);
    if (p.D < 64) return launch_decode_core<DecodeF32<1, false>, P>(a, stream);
    if (p.D < 128) return launch_decode_core<DecodeF32<2, false>, P>(a, stream);
    return launch_decode_core<DecodeF32<4, false>, P>(a, stream);
  };
  return p.table ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace ac
