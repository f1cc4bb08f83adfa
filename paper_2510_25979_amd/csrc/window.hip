// Attention of prompts within a sliding window: row t sees keys j <= t with j > t - window or j < sinks, of the item's first key_len.
//
// Rows are cut into units of 32 tokens (binary32: 16) of one head; the units of the g heads that share K and V are numbered token block first, head
// second, and four consecutive ones are a workgroup, so that its waves see (nearly) the same keys: with four heads on one K and V a
// workgroup reads no key that only some of its waves need.  It walks the blocks of 32 keys (16) that hold a first token or lie in the window of one
// of its rows, and compares keys with rows only where some see them and some do not.
//
// bf16: two blocks at a time straight into one of two LDS stages, by buffer loads whose bounds are the item's last key; both products of stream_tile.h.
// Bound by the softmax's vector work and the matrix pipe at the clock that the chip grants them: 128 heads of 128, 4,096 tokens, window 1,024, 276 us (0.88
// PFLOP/s; 309 to 370 where nothing else runs between), the pipe busy in 48 % of the cycles.  Blocks of 32 keys and not chunks of 64 spare 5 % at a window's two
// edges.  Passing over pairs that a wave does not see takes 6 % off rows of one head a workgroup and a window of 64 (66 / 62), and adds 1 to 2 %
// everywhere else: not done.
//
// A hidden key must not touch a row even if its V is infinite or NaN, which a product over a block cannot avoid (0 * inf): a workgroup of which a wave ends with such
// a result walks its keys three times more.  That wave then forms its sums without what is not finite, and counts who sees a +inf, and who a -inf (StreamTile::chunk_of).
// us, 16 heads of 128 (bf16 / binary32), 1,500 tokens, window 700: 22 / 90; with NaN in Q's last 500 rows 22 / 88, in a first token's V 113 / 490, in all of V 200 / 490;
// key by key each of the four took 14,900 / 7,600.
#include <type_traits>

#include "common.hpp"
#include "f32_tile.hpp"
#include "serve.h"
#include "stream_tile.h"

namespace ac {

constexpr int kWindowChunk = kStreamChunk;

struct WindowArgs {
  const void *Q, *K, *V;
  void* O;
  const int32_t *len, *row_sel;
  int32_t Hkv, g, S, D, window, sinks, first, tiles, per, units;   // first: of the launch's tiles; per, units: workgroups, units of a tile
  float scale_log2e;
  Divider by_g, by_per;
};

// Blocks of C keys that a workgroup with tokens [lo, hi) looks at: `head` of them from the first on, then `count - head` from `from` on.
template <int C>
struct WindowBlocks {
  int head, from, count;
  __device__ __forceinline__ WindowBlocks(const WindowArgs& a, int lo, int hi, int keys) {
    const int end = (min(hi, keys) + C - 1) / C, seen = min(a.sinks, min(hi, keys));
    head = (seen + C - 1) / C;
    from = max(head, max(0, lo - a.window + 1) / C);
    count = head + max(0, end - from);
  }
  __device__ __forceinline__ int at(int i) const { return i < head ? i : i - head + from; }
};
// What rows [t0, t0 + R) see of keys [k0, k0 + C).
enum WindowBlock { kNone, kSome, kEvery };
template <int R, int C>
__device__ __forceinline__ WindowBlock window_block(const WindowArgs& a, int t0, int k0, int keys) {
  if (k0 > t0 + R - 1 || k0 >= keys || (k0 + C - 1 <= t0 - a.window && k0 >= a.sinks)) return kNone;
  return k0 + C - 1 <= t0 && k0 + C <= keys && (k0 > t0 + R - 1 - a.window || k0 + C <= a.sinks) ? kEvery : kSome;
}
__device__ __forceinline__ bool window_hides(const WindowArgs& a, int t, int key, int keys) {
  return key > t || key >= keys || (key <= t - a.window && key >= a.sinks);
}

// Whether what a row came to may have been touched by what it does not see: sums that are not finite beside a sum of weights that is a number.  (The
// latter knows nothing of V: if it is NaN, a score that the row sees is, or is +inf, and so is the row.)  Or its scores are of 2^30 and more: stream_weight.
__device__ __forceinline__ bool window_doubtful(float m, float sum, float rest) {   // rest: NaN if a sum is not finite, otherwise 0
  const bool odd = rest != rest && sum == sum, far = fabsf(m) >= 0x1p30f && fabsf(m) < INFINITY;
  return odd || far;
}

template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 4 : 2) void window_bf16_kernel(const WindowArgs a) {
  constexpr int PPR = D / 8;                             // 16-byte pieces of a row
  constexpr int NCOPY = kWindowChunk * PPR / kWave / 4;  // copy instructions of a wave, tensor and chunk
  __shared__ __attribute__((aligned(16))) bf16_t kb0[kWindowChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb0[kWindowChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t kb1[kWindowChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb1[kWindowChunk * D];
  __shared__ int doubt;   // of some wave, about its results
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid == 0) doubt = 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int il = lane & 31, kh = lane >> 5;
  // workgroups with ids equal mod 8 (one XCD) share K and V in its L2
  const int slot = blockIdx.x >> 3, group = a.by_per.div(slot), u = a.first + group * 8 + (blockIdx.x & 7);
  if (u >= a.tiles) return;
  const int b = u / a.Hkv, hk = u - b * a.Hkv;
  if (a.row_sel && a.row_sel[b] >= 0) return;
  const int keys = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  const int unit0 = 4 * (slot - group * a.per), last = min(unit0 + 3, a.units - 1);
  const int unit = min(unit0 + wave, last), tb = a.by_g.div(unit), t0 = kRowsPerWave * tb;
  const bool live = unit0 + wave <= last;
  const size_t row0 = ((size_t)(b * a.Hkv + hk) * a.g + (unit - tb * a.g)) * a.S;   // the head's first row
  const int rows = min(kRowsPerWave, a.S - t0);
  const WindowBlocks<32> blocks(a, kRowsPerWave * a.by_g.div(unit0), min(a.S, kRowsPerWave * (a.by_g.div(last) + 1)), keys);
  const bf16_t* Ksrc = reinterpret_cast<const bf16_t*>(a.K) + (size_t)u * a.S * D;
  const bf16_t* Vsrc = reinterpret_cast<const bf16_t*>(a.V) + (size_t)u * a.S * D;
  bf16_t* O = reinterpret_cast<bf16_t*>(a.O) + (row0 + t0) * D;
  StreamTile<D> tile(a.scale_log2e, lane);
  // copies as in cross.hip
  const int slot0 = kWave * wave + lane, crow = slot0 / PPR, cpos = slot0 % PPR;
  const int kpiece = 8 * (cpos ^ k_piece_swizzle<D>(crow)), vpiece = 8 * (cpos ^ v_piece_swizzle<D>(crow));
  // A chunk is two blocks of 32 keys that follow one another in the workgroup's list; the second of the last may be missing.
  constexpr int NROW = NCOPY / 2;        // copies of a block
  uint32_t kfrom[NROW], vfrom[NROW];     // bytes from a block's first row
#pragma unroll
  for (int i = 0; i < NROW; ++i) {
    kfrom[i] = 2 * ((crow + 256 / PPR * i) * D + kpiece);
    vfrom[i] = 2 * ((crow + 256 / PPR * i) * D + vpiece);
  }
  auto copy = [&](bf16_t* kb, bf16_t* vb, int c) {   // (rows behind the keys are not read; in the place of a missing block lies the one before it)
#pragma unroll
    for (int jb = 0; jb < 2; ++jb) {
      const int k0 = kRowsPerWave * blocks.at(min(2 * c + jb, blocks.count - 1));
      const uint32_t bytes = min(keys - k0, 32) * D * 2;
      const StreamSource ks(Ksrc + (size_t)k0 * D, bytes), vs(Vsrc + (size_t)k0 * D, bytes);
#pragma unroll
      for (int i = 0; i < NROW; ++i) {
        ks.copy(kb + 32 * D * jb + kWave * 8 * (wave + 4 * i), kfrom[i]);
        vs.copy(vb + 32 * D * jb + kWave * 8 * (wave + 4 * i), vfrom[i]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const int n_chunk = (blocks.count + 1) / 2;
  if (n_chunk > 0) copy(kb0, vb0, 0);
  tile.load_q(reinterpret_cast<const bf16_t*>(a.Q) + (row0 + min(t0 + il, a.S - 1)) * D);
  tile.reset();
  // (mfma_row(v, 0) is a key's place in its block but for the lane's part of it, a constant of the register)
  auto hide = [&](f32x16& s, int k0) {
    const int mine = k0 + 4 * kh, t = t0 + il;
    if (k0 + 31 > min(t0, keys - 1)) {   // keys behind the row or the item's last
      const int hi = min(t, keys - 1) - mine;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = mfma_row(v, 0) > hi ? -INFINITY : s[v];
    }
    if (k0 <= t0 + kRowsPerWave - 1 - a.window && k0 + 32 > a.sinks) {   // keys in the gap
      const int from = a.sinks - mine;
      const unsigned n = (unsigned)max(t - a.window - a.sinks + 1, 0);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = (unsigned)(mfma_row(v, 0) - from) < n ? -INFINITY : s[v];
    }
  };
  auto hide_both = [&](int c) {
    return [&, c](f32x16& s0, f32x16& s1) {
      hide(s0, 32 * blocks.at(2 * c));
      hide(s1, 2 * c + 1 < blocks.count ? 32 * blocks.at(2 * c + 1) : keys);
    };
  };
  auto publish = [&]() {   // this wave's copies have landed, then everybody's; the other stage is no longer read
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };
  auto walk = [&](auto step) __attribute__((always_inline)) {
#pragma unroll 1
    for (int c = 0; c < n_chunk; c += 2) {   // (two a trip: the stages alternate without pointer arithmetic)
      publish();
      if (c + 1 < n_chunk) copy(kb1, vb1, c + 1);
      step(kb0, vb0, c);
      if (c + 1 >= n_chunk) break;
      publish();
      if (c + 2 < n_chunk) copy(kb0, vb0, c + 2);
      step(kb1, vb1, c + 1);
    }
  };
  walk([&](const bf16_t* kb, const bf16_t* vb, int c) __attribute__((always_inline)) { tile.chunk(kb, vb, hide_both(c)); });
  f32x16(&acc)[D / 32] = tile.acc;
  float sum = tile.sum();
  float rest[4] = {0.f, 0.f, 0.f, 0.f};   // NaN where a sum is not finite (a comparison each waits for scalar registers: 0.3 us)
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) rest[v & 3] = fmaf(acc[db][v], 0.f, rest[v & 3]);
  const bool again = __any(live && il < rows && window_doubtful(tile.m, sum, (rest[0] + rest[1]) + (rest[2] + rest[3])));
  if (again && lane == 0) doubt = 1;
  __syncthreads();   // every wave is done with both stages: they now stage the output
  auto store = [&]() {
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
  };
  if (live) store();   // (doubtful rows, too, and over them later)
  if (__builtin_expect(!__builtin_amdgcn_readfirstlane(doubt), 1)) return;
#pragma unroll 1
  for (int which = kFinite; which <= kDown; ++which) {
    __syncthreads();   // the stages are no longer read
    copy(kb0, vb0, 0);
    tile.reset();
    walk([&](const bf16_t* kb, const bf16_t* vb, int c) __attribute__((always_inline)) {
      if (again) tile.chunk_of((StreamValues)which, kb, vb, hide_both(c));
    });
    sum = tile.sum();
    if (!again || il >= rows) continue;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    bf16_t* o = O + (size_t)il * D + 4 * kh;
    auto each = [&](auto f) {   // (a lane's columns are always the same: it reads what it wrote)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) f(o + 32 * db + mfma_row(v, 0), acc[db][v]);
    };
    const float such = which == kUp ? INFINITY : -INFINITY;
    if (which == kFinite) each([&](bf16_t* o, float x) { *o = (bf16_t)(x * inv); });
    else each([&](bf16_t* o, float x) { if (x > 0.f) *o = (bf16_t)((float)*o + such); });
  }
}

// f32_weights_v of the values that StreamTile::chunk_of takes.
template <int DB, int LD>
__device__ __forceinline__ void window_weights_v_of(StreamValues which, f32x4 (&acc)[4 * DB], const float* __restrict__ v, const f32x4 w, int i, int kq) {
  const float wanted = which == kUp ? INFINITY : -INFINITY;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const f32x4 r = *reinterpret_cast<const f32x4*>(v + (4 * kq + x) * LD + 64 * b + 4 * i);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float count = r[t] == wanted || r[t] != r[t] ? 1.f : 0.f;
        acc[4 * b + t] = mfma_f32(stream_one_of(which, fabsf(r[t]) < INFINITY ? r[t] : 0.f, count), w[x], acc[4 * b + t]);
      }
      __builtin_amdgcn_sched_barrier(0);   // (reads that run ahead would take more registers than the kernel has)
    }
}

// Binary32 (the layout of f32_tile.hpp): four waves share stages of 16 keys for each wave of a row.  Heads of 64 and 128 columns go straight from memory
// into two stages in turn (K's pieces swizzled, V's not: both are then read without bank conflicts); others through registers, in which the next stage is while
// this one is multiplied.  The vector units form these products themselves, so that what the softmax takes comes on top of them, and its reference
// points move only when a score has outgrown them by 2^8.  us, 24 heads of 128, 16 items of up to 333 tokens, window 100: 78 with stages of 32 keys
// a wave, 75 of 16, 74 straight into LDS, 72 with reference points that stay; waves that load their keys for themselves, without stages or barriers, read
// them four times: 96; eight waves, two for each row: 82.  Bound by products and softmax (47 us of it; four times the items take 216) and, where a
// chip's few rounds of workgroups end unevenly, by the last ones.
template <int DB, int COLS, int SPLIT>   // SPLIT: waves that share 16 rows, each with 16 keys of every stage
__global__ __launch_bounds__(kThreads, DB == 4 && COLS == kAllCols && SPLIT == 2 ? 1 : 2) void window_f32_kernel(const WindowArgs a) {
  constexpr int KC = kF32Rows * SPLIT, UNITS = 4 / SPLIT;   // keys of a stage; units of a workgroup
  constexpr bool DIRECT = COLS == kAllCols;   // rows go straight to LDS, into two stages in turn
  typedef F32Stage<DB, KC, COLS> Stage;
  const int D = COLS == kAllCols ? 64 * DB : a.D;
  constexpr int LD = DIRECT ? 64 * DB : Stage::LD;
  __shared__ __attribute__((aligned(16))) float kl[KC * LD];
  __shared__ __attribute__((aligned(16))) float vl[KC * LD];
  __shared__ __attribute__((aligned(16))) float kl1[DIRECT ? KC * LD : 4];
  __shared__ __attribute__((aligned(16))) float vl1[DIRECT ? KC * LD : 4];
  __shared__ __attribute__((aligned(16))) int doubt[4];   // of a wave, about its results
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < 4) doubt[tid] = 0;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, kq = lane >> 4, part = wave / UNITS, key0 = part * kF32Rows;
  const int slot = blockIdx.x >> 3, group = a.by_per.div(slot), u = a.first + group * 8 + (blockIdx.x & 7);
  if (u >= a.tiles) return;
  const int b = u / a.Hkv, hk = u - b * a.Hkv;
  if (a.row_sel && a.row_sel[b] >= 0) return;
  const int keys = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  const int unit0 = UNITS * (slot - group * a.per), last = min(unit0 + UNITS - 1, a.units - 1);
  const int unit = min(unit0 + wave % UNITS, last), tb = a.by_g.div(unit), t0 = kF32Rows * tb;
  const bool live = unit0 + wave % UNITS <= last;
  const size_t row0 = ((size_t)(b * a.Hkv + hk) * a.g + (unit - tb * a.g)) * a.S;
  const WindowBlocks<KC> chunks(a, kF32Rows * a.by_g.div(unit0), min(a.S, kF32Rows * (a.by_g.div(last) + 1)), keys);
  const float* K = reinterpret_cast<const float*>(a.K) + (size_t)u * a.S * D;
  const float* V = reinterpret_cast<const float*>(a.V) + (size_t)u * a.S * D;
  const float* Q = reinterpret_cast<const float*>(a.Q) + row0 * D;
  float* O = reinterpret_cast<float*>(a.O) + row0 * D;
  f32x4 q[4 * DB], acc[4 * DB];
  {
    const float* src = Q + (size_t)min(t0 + i, a.S - 1) * D;
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
  float m, ref, l;
  auto reset = [&]() {
#pragma unroll
    for (int x = 0; x < 4 * DB; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    ref = l = 0.f;
  };
  auto block = [&](const float* kl, const float* vl, int j0, auto apart, int which) __attribute__((always_inline)) {   // apart: the values that `which` says
    const int k0 = j0 + key0;
    const WindowBlock bl = window_block<kF32Rows, kF32Rows>(a, t0, k0, keys);
    if (bl == kNone) return;   // uniform
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    auto piece = [&](int kk) { return *reinterpret_cast<const f32x4*>(kl + (key0 + i) * LD + (DIRECT ? 4 * ((4 * kk + kq) ^ i) : 16 * kk + 4 * kq)); };
    f32x4 k = piece(0);
#pragma unroll
    for (int kk = 0; kk < 4 * DB; ++kk)
      if (COLS == kAllCols || 16 * kk < D) {   // uniform
        const f32x4 next = piece((kk + 1) & (4 * DB - 1));
#pragma unroll
        for (int x = 0; x < 4; ++x) s = mfma_f32(k[x], q[kk][x], s);
        k = next;
        __builtin_amdgcn_sched_barrier(0);
      }
    if (bl == kSome) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (window_hides(a, t0 + i, k0 + 4 * kq + x, keys)) s[x] = -INFINITY;
    }
    const float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * a.scale_log2e;
    if ((!apart || which == kFinite) && __any(mx > m + kStreamSlack)) {   // (counts are not scaled)
      float top = fmaxf(mx, __shfl_xor(mx, 16));
      top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), m);
      const float alpha = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.f;
      l *= alpha;
#pragma unroll
      for (int x = 0; x < 4 * DB; ++x) acc[x] *= alpha;
      m = top;
      ref = m == -INFINITY ? 0.f : m;   // no finite score so far: all weights are zero
    }
    f32x4 p;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if constexpr (apart) p[x] = stream_one_of((StreamValues)which, stream_weight(s[x], a.scale_log2e, ref), s[x] == -INFINITY ? 0.f : 1.f);
      else p[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2e, -ref));
      l += p[x];
    }
    if constexpr (apart) window_weights_v_of<DB, LD>((StreamValues)which, acc, vl + key0 * LD, p, i, kq);
    else f32_weights_v<DB, LD>(acc, vl + key0 * LD, p, i, kq);
  };
  auto walk = [&](bool mine, auto apart, int which, int tid, int D) __attribute__((always_inline)) {   // all keys; mine: of this wave's row block, too
    if constexpr (DIRECT) {
      constexpr int PPR = 16 * DB, NCOPY = KC * PPR / kThreads;   // 16-byte pieces of a row, of a thread
      uint32_t kfrom[NCOPY], vfrom[NCOPY];   // bytes from a stage's first row; piece p of K's row r lies at p ^ r % 16
#pragma unroll
      for (int n = 0; n < NCOPY; ++n) {
        const int r = tid / PPR + n * (kThreads / PPR), p = tid % PPR;
        kfrom[n] = 16 * (r * PPR + (p ^ (r & 15)));
        vfrom[n] = 16 * (r * PPR + p);
      }
      auto copy = [&](float* kl, float* vl, int n) {   // (rows behind the keys: zeros)
        const int j0 = KC * chunks.at(n);
        const uint32_t bytes = min(keys - j0, KC) * LD * 4;
        const StreamSource ks(K + (size_t)j0 * LD, bytes), vs(V + (size_t)j0 * LD, bytes);
#pragma unroll
        for (int x = 0; x < NCOPY; ++x) {
          ks.copy(kl + 4 * kWave * (wave + 4 * x), kfrom[x]);
          vs.copy(vl + 4 * kWave * (wave + 4 * x), vfrom[x]);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      auto publish = [&]() {   // this wave's copies have landed, then everybody's; the other stage is no longer read
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
      };
      if (chunks.count > 0) copy(kl, vl, 0);
#pragma unroll 1
      for (int n = 0; n < chunks.count; n += 2) {
        publish();
        if (n + 1 < chunks.count) copy(kl1, vl1, n + 1);
        if (mine) block(kl, vl, KC * chunks.at(n), apart, which);
        if (n + 1 >= chunks.count) break;
        publish();
        if (n + 2 < chunks.count) copy(kl, vl, n + 2);
        if (mine) block(kl1, vl1, KC * chunks.at(n + 1), apart, which);
      }
    } else {
      Stage ks, vs;
      if (chunks.count > 0) {
        ks.load(K, KC * chunks.at(0), keys, D, tid);
        vs.load(V, KC * chunks.at(0), keys, D, tid);
      }
      for (int n = 0; n < chunks.count; ++n) {
        const int j0 = KC * chunks.at(n);
        ks.template mask<false>(j0, keys, D, tid);   // (scores of keys that are not there are replaced)
        vs.template mask<true>(j0, keys, D, tid);
        __syncthreads();   // the previous stage has been read by everybody
        ks.commit(kl, tid);
        vs.commit(vl, tid);
        __syncthreads();
        if (n + 1 < chunks.count) {
          ks.load(K, KC * chunks.at(n + 1), keys, D, tid);
          vs.load(V, KC * chunks.at(n + 1), keys, D, tid);
        }
        if (mine) block(kl, vl, j0, apart, which);
      }
    }
  };
  float sum;
  auto join = [&](bool mine) __attribute__((always_inline)) {   // what the row's lanes and waves have
    const float all = l + __shfl_xor(l, 16);
    if (mine) sum = all + __shfl_xor(all, 32);
    if constexpr (SPLIT == 2) {   // the second wave's sums through the stages, which nobody reads any more
      static_assert(4 * DB * kWave * 4 * UNITS <= KC * LD, "sums of two waves");
      f32x4* sums = reinterpret_cast<f32x4*>(kl) + wave % UNITS * 4 * DB * kWave + lane;
      float* stats = vl + wave % UNITS * 2 * kWave + lane;
      __syncthreads();
      if (mine && part > 0) {
#pragma unroll
        for (int x = 0; x < 4 * DB; ++x) sums[x * kWave] = acc[x];
        stats[0] = m;
        stats[kWave] = sum;
      }
      __syncthreads();
      if (mine && part == 0) {
        const float m1 = stats[0], top = fmaxf(m, m1);
        const float f0 = m < top ? __builtin_amdgcn_exp2f(m - top) : 1.f, f1 = m1 < top ? __builtin_amdgcn_exp2f(m1 - top) : 1.f;
        sum = sum * f0 + stats[kWave] * f1;
        m = top;
#pragma unroll
        for (int x = 0; x < 4 * DB; ++x) acc[x] = acc[x] * f0 + sums[x * kWave] * f1;
      }
    }
  };
  const int rows = min(kF32Rows, a.S - t0);
  reset();
  walk(live, std::false_type{}, kFinite, tid, D);
  // (sums end here for the compiler: carried on to the stores in the registers that suit those, they took 24 more and a copy after every product)
#pragma unroll
  for (int x = 0; x < 4 * DB; ++x) asm volatile("" : "+v"(acc[x]));
  join(true);
  f32x4 rest = {0.f, 0.f, 0.f, 0.f};   // as above
#pragma unroll
  for (int x = 0; x < 4 * DB; ++x)
#pragma unroll
    for (int t = 0; t < 4; ++t) rest[t] = fmaf(acc[x][t], 0.f, rest[t]);
  bool again = part == 0 && __any(live && i < rows && window_doubtful(m, sum, (rest[0] + rest[1]) + (rest[2] + rest[3])));
  if (again && lane == 0) doubt[wave] = 1;
  if (part == 0 && live && i < rows) f32_store_row<DB, COLS, true>(O + (size_t)(t0 + i) * D, acc, sum == 0.f ? 1.f : sum, kq, D);
  __syncthreads();
  if (__builtin_expect(!__builtin_amdgcn_readfirstlane(doubt[0] | doubt[1] | doubt[2] | doubt[3]), 1)) return;
  if (SPLIT == 2) again = __builtin_amdgcn_readfirstlane(doubt[wave % UNITS]);   // both waves of a row
#pragma unroll 1
  for (int which = kFinite; which <= kDown; ++which) {
    __syncthreads();   // the stages are no longer read
    reset();
    // (what the first walk knows of its copies need not be kept for these: the compiler forms it again)
    int tid_ = tid, D_ = D;
    asm volatile("" : "+v"(tid_), "+s"(D_));
    walk(again, std::true_type{}, which, tid_, COLS == kAllCols ? D : D_);
    join(again);
    if (part > 0 || !again || i >= rows) continue;
    float* o = O + (size_t)(t0 + i) * D + 16 * kq;   // (an address of its own in every turn: the compiler would keep one a column)
    asm volatile("" : "+v"(o));
    const int cols = D_ - 16 * kq;
    const float by = sum == 0.f ? 1.f : sum, inv = 1.f / by;
    auto each = [&](auto f) {   // (a lane's columns are always the same: it reads what it wrote)
#pragma unroll
      for (int n = 0; n < 4 * DB; ++n)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int d = 64 * (n >> 2) + 4 * (n & 3) + t;
          if (d < cols) f(o + d, acc[4 * (n >> 2) + t][n & 3]);
        }
    };
    const float such = which == kUp ? INFINITY : -INFINITY;
    if (which == kFinite) each([&](float* o, float x) { *o = f32_divide(x, by, inv); });
    else each([&](float* o, float x) { if (x > 0.f) *o += such; });
  }
}

// All tiles, in launches of at most 2^23 workgroups (a multiple of eight tiles each).
template <typename Kernel>
static hipError_t window_tiles(Kernel kernel, WindowArgs a, int rows, int units, hipStream_t stream) {   // rows of a unit, units of a workgroup
  a.units = (a.S + rows - 1) / rows * a.g;
  a.per = (a.units + units - 1) / units;
  a.by_per = Divider((uint32_t)a.per);
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

// Two waves a row where workgroups of 64 rows would not give every CU one: a wave's chain of keys is what such a call takes (24 heads on 8 of K and
// V, 333 tokens, 128 workgroups: 20 -> 15 us; 8 heads, 1,000 tokens, all seen, 256: 61 -> 49).  With more, half as many rows a workgroup read every
// key twice as often and nothing is gained (576 workgroups: 24 -> 25; 2,688: 79 -> 89).
constexpr int64_t kWindowSplit = 256;

template <int DB, int COLS>
static hipError_t launch_window_f32(const WindowArgs& a, hipStream_t stream) {
  const int64_t workgroups = ((int64_t)((a.S + kF32Rows - 1) / kF32Rows) * a.g + 3) / 4 * a.tiles;
  return workgroups <= kWindowSplit ? window_tiles(&window_f32_kernel<DB, COLS, 2>, a, kF32Rows, 2, stream)
                                    : window_tiles(&window_f32_kernel<DB, COLS, 1>, a, kF32Rows, 4, stream);
}

hipError_t launch_window(const WindowLaunch& p, hipStream_t stream) {
  WindowArgs a;
  a.Q = p.Q; a.K = p.K; a.V = p.V; a.O = p.O; a.len = p.key_len; a.row_sel = p.row_sel;
  a.Hkv = p.Hkv; a.g = p.Hq / p.Hkv; a.S = p.S; a.D = p.D;
  a.window = p.window < p.S ? p.window : p.S;   // (t - window stays in 32 bits)
  a.sinks = p.sinks < p.S ? p.sinks : p.S;
  a.tiles = p.B * p.Hkv;
  a.by_g = Divider((uint32_t)a.g);
  const float scale = p.scale == 0.f ? 1.0f / sqrtf((float)p.D) : p.scale;
  a.scale_log2e = scale * 1.44269504088896340736f;
  if (!p.is_f32) return p.D == 64 ? window_tiles(&window_bf16_kernel<64>, a, 32, 4, stream) : window_tiles(&window_bf16_kernel<128>, a, 32, 4, stream);
  if (p.D == 64) return launch_window_f32<1, kAllCols>(a, stream);
  if (p.D == 128) return launch_window_f32<2, kAllCols>(a, stream);
  if (p.D < 4) return launch_window_f32<1, kFewCols>(a, stream);
  if (p.D < 64) return p.D % 4 ? launch_window_f32<1, kAnyCols>(a, stream) : launch_window_f32<1, kVecCols>(a, stream);
  if (p.D < 128) return p.D % 4 ? launch_window_f32<2, kAnyCols>(a, stream) : launch_window_f32<2, kVecCols>(a, stream);
  if (p.D == 256) return launch_window_f32<4, kAllCols>(a, stream);
  return p.D % 4 ? launch_window_f32<4, kAnyCols>(a, stream) : launch_window_f32<4, kVecCols>(a, stream);
}

}  // namespace ac
