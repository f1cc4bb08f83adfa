// Attention of one new token of each request over its pages, where requests share long prefixes: K and V of a prefix are read once for all
// requests of its group, not once for each.
//
// A group is consecutive rows of the batch whose first P tokens are the same.  The work is a list of items, first the groups' prefixes (the g heads of
// all the group's requests on P keys), then each request's own keys behind its prefix (g heads on n - P keys); a request that shares nothing has all its
// keys there.  Every item's result is partial: row maximum, sum, sum of weighted V, in binary32; a row's two items are added up at the end.
//
// The list says who is in which group, what each item has and where its blocks are numbered.  Up to 256 requests and 255 groups each workgroup makes it
// for itself, in LDS; otherwise shared_plan_kernel writes it before.
// shared_prefix (bf16) forms prefixes of many rows: workgroups of 128 rows that share chunks of 64 keys in LDS (stream_tile.h), each an equal
//   run of all such chunks, so that few groups fill the chip and many short ones do, too.
// shared_run forms everything else in units of 32 rows (binary32 16) of one (item, K/V head), cut into equal runs of blocks by wave, as decode.hip.
// shared_join_kernel adds up an output row's parts.
//
// 64 requests of 32 heads on 8 of 128 that share 16,000 tokens 45 us, of which the list takes 5, the prefix 31 -- 16 chunks of some 1.3 us one after another in each
// workgroup: products, page numbers and copies each need about as long, and neither without the others' wait is much faster (36 without the copies, 33 without
// the products) --, the join 7.  134 requests that share little: bound by memory, 44 of 50 us in the runs.
#include <type_traits>

#include "decode_tile.h"
#include "stream_tile.h"

namespace ac {

constexpr int kSharedRows = 128, kSharedChunk = kStreamChunk;   // of a workgroup of shared_prefix
constexpr int kSharedWgs = 512;                       // most workgroups
constexpr int kSharedLeast = 4, kSharedMost = 16;     // chunks of a run: at least; at most while there is one for each compute unit (see the plan)
constexpr int kSharedUnitCost = 1;                    // what a unit of it costs beside its chunks

struct SharedItem {
  int keys, key0, row;     // keys [key0, key0 + keys) of the request whose table has them
  int b0, R;               // rows of a K/V head: the g heads of requests b0, b0 + 1, ...
  int rbs, start;          // row blocks of a K/V head; number of the first block
  int group;               // of a request: its group's number, -1: shares nothing; of a group: 1 if shared_prefix forms it
};

struct SharedArgs {
  DecodeArgs d;            // Q, K, V, O, table, len and sizes
  const int32_t *share_first, *share_len;
  int32_t *sums, *first, *leader, *count, *start, *start1;   // sums: blocks of all items, chunks of all prefixes, chunks of a run
  SharedItem* item;        // [G + B]
  float *part, *stat;      // partial results: rows' own whole ones, rows' prefixes' whole ones, two of each run
  int32_t G, g, own_rbs, big_rows, big_keys, wgs;   // see shared_is_big
  Divider by_g;
};

// Whether shared_prefix forms a prefix: one of more than 32 rows, or of more than 16 where it is long and a head has 128 columns.  us, 32 rows a wave / workgroups of 128:
// 64 rows a group, prefixes of 16,000 tokens 43.4 / 28.8, eight of 2,000 53.1 / 40.7, 16 of 4,000 of 64 columns 69.3 / 57.4; 48 rows, eight of 2,000 48.7 /
// 38.2; 96 rows 70.6 / 51.7; 32 rows, one of 16,000 34.2 / 26.7, eight of 4,000 55.5 / 46.1, four of 1,000 23.4 / 25.3, 64 of 500 107 / 112; of 64 columns
// 16 of 4,000 45.3 / 44.5, of 24 rows 41.9 / 43.8; 20 rows, one of 16,000 31.1 / 25.4.
__device__ __forceinline__ int shared_is_big(const SharedArgs& a, int R, int keys) {
  return R > a.big_rows || (R > kDecodeRows && keys >= a.big_keys);
}

// A wave's work on a block for two blocks of 16 rows, which share the keys' way from memory (the second may be empty): a prefix of eight requests of
// four heads is read once and not twice.
template <int D_>
struct SharedBf16 : DecodeBf16<D_> {
  typedef DecodeBf16<D_> One;
  static constexpr int RB = 2;
  f32x4 acc1[One::NP];
  float m1, l1;
  using One::One;
  __device__ __forceinline__ void reset() {
    One::reset();
#pragma unroll
    for (int n = 0; n < One::NP; ++n) acc1[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    m1 = -INFINITY;
    l1 = 0.f;
  }
  __device__ __forceinline__ void add1(typename One::Scores& s, float scale_log2e) { One::add(s, scale_log2e, acc1, m1, l1); }
  __device__ __forceinline__ f32x4 piece1(int n) const { return acc1[n]; }
};
template <int DB, bool FULL>
struct SharedF32 : DecodeF32<DB, FULL> {
  typedef DecodeF32<DB, FULL> One;
  static constexpr int RB = 1;
  float m1 = 0.f, l1 = 0.f;
  using One::One;
  __device__ __forceinline__ void add1(typename One::Scores&, float) {}
  __device__ __forceinline__ f32x4 piece1(int) const { return f32x4{0.f, 0.f, 0.f, 0.f}; }
};

// Records: own whole results [B Hq], prefixes' [B Hq], of runs [2 waves][unit], of workgroups [2 wgs][128].
__device__ __forceinline__ size_t shared_rows(const SharedArgs& a) { return (size_t)a.d.B * a.d.Hkv * a.g; }

template <int NT, typename Op>
__device__ __forceinline__ int shared_scan(int x, int& all, int* part, Op op, int none) {   // inclusive, over the workgroup
  constexpr int NW = NT / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int p = __shfl_up(x, off);
    if (lane >= off) x = op(x, p);
  }
  if (lane == kWave - 1) part[wave] = x;
  __syncthreads();
  int before = none;
  all = none;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int p = part[w];
    if (w < wave) before = op(before, p);
    all = op(all, p);
  }
  __syncthreads();
  return op(x, before);
}

// What the list adds up to: blocks of shared_run, chunks of shared_prefix, chunks of a run of the latter, waves of the former.
// One workgroup of prefixes a compute unit up to 16 chunks each, beside it one that has runs, then two.  Each leaves up to two partial results of 128
// rows, so that more of them cost the join what they save: 64 requests of a prefix of 16,000 tokens (4,016 chunks) in 502 runs of 8 66.6 us, in
// 251 of 16 61.8, and 58.4 with the runs on the other half of the workgroups.
__device__ __forceinline__ int shared_sum(const SharedArgs& a, int blocks, int chunks, int which) {
  if (which < 2) return which ? chunks : blocks;
  if (which == 3) return (int64_t)chunks * 128 >= (int64_t)blocks * a.d.D ? a.d.waves / 2 : a.d.waves;
  const int one = chunks > 0 ? (chunks - 1) / (a.wgs / 2) + 1 : 0, two = chunks > 0 ? (chunks - 1) / a.wgs + 1 : 0;
  return max(max(one < kSharedMost ? one : kSharedMost, two), kSharedLeast);
}

// Groups of the plan: in LDS while each has a thread, otherwise in the workspace, where what this launch has written is read past the
// first-level cache.
template <bool LDS>
__device__ __forceinline__ int shared_peek(const int* p) {
  return LDS ? *p : __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Bound by latency: lengths and groups -> who shares -> sums -> list.  64 requests 14.3 us with the groups in the workspace, 6.0 so.
template <int BK, int UNIT, int NT, bool LDS>   // keys of a block, rows of a unit, threads
__global__ __launch_bounds__(NT) void shared_plan_kernel(const SharedArgs a) {
  __shared__ int part[NT / kWave], part1[NT / kWave];
  __shared__ int s_first[LDS ? NT + 1 : 1], s_leader[LDS ? NT : 1], s_count[LDS ? NT : 1], s_len[LDS ? NT : 1];
  const int tid = threadIdx.x, B = a.d.B, G = a.G, cap = a.d.Sk;
  int* first = LDS ? s_first : a.first;
  int* leader = LDS ? s_leader : a.leader;
  int* count = LDS ? s_count : a.count;
  auto add = [](int x, int y) { return x + y; };
  auto top = [](int x, int y) { return max(x, y); };
  auto tokens = [&](int b) { return min(max(a.d.len[b], 0), cap); };
  int mine = tid < B ? tokens(tid) : 0;   // of the first requests: asked for at once
  // where groups begin: in order, whatever is given
  int before = 0;
  for (int c = 0; c <= G; c += NT) {
    const int i = c + tid;
    if (LDS && i < G) s_len[i] = min(max(a.share_len[i], 0), cap);
    int all;
    const int f = shared_scan<NT>(i <= G ? min(max(a.share_first[i], 0), B) : 0, all, part, top, 0);
    if (i <= G) first[i] = max(before, f);
    if (i < G) {
      leader[i] = B;
      count[i] = 0;
    }
    before = max(before, all);
  }
  if (!LDS) __threadfence();
  __syncthreads();
  auto prefix = [&](int q) { return LDS ? s_len[q] : min(max(a.share_len[q], 0), cap); };
  auto group_of = [&](int b) {   // the last group that begins at b or before it, if b is in it
    int lo = -1, hi = G;         // first[lo] <= b < first[hi], but for the ends
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (shared_peek<LDS>(first + mid) <= b) lo = mid;
      else hi = mid;
    }
    return lo >= 0 && b < shared_peek<LDS>(first + lo + 1) ? lo : -1;
  };
  int group = -1;   // of this thread's request among the first
  for (int b = tid; b < B; b += NT) {
    const int q = group_of(b), n = b == tid ? mine : tokens(b);
    if (b == tid) group = q;
    if (q < 0) continue;
    const int P = prefix(q);
    if (P > 0 && n >= P) {   // shorter ones have their keys for themselves
      atomicMin(&leader[q], b);
      atomicAdd(&count[q], 1);
    }
  }
  if (!LDS) __threadfence();
  __syncthreads();
  // First the groups, then the requests: the same thread has a request here and above.
  int begun = 0, begun1 = 0;
  for (int c = 0; c < G; c += NT) {
    const int i = c + tid;
    SharedItem it = {0, 0, 0, 0, 0, 1, 0, 0};
    int cost = 0, cost1 = 0;
    if (i < G && shared_peek<LDS>(count + i) > 1) {
      const int f = shared_peek<LDS>(first + i), n = shared_peek<LDS>(first + i + 1) - f;
      it.keys = prefix(i);
      it.row = shared_peek<LDS>(leader + i);
      it.b0 = f;
      it.R = n * a.g;
      it.group = shared_is_big(a, it.R, it.keys);
      if (it.group) {
        it.rbs = (it.R + kSharedRows - 1) / kSharedRows;
        cost1 = a.d.Hkv * it.rbs * ((it.keys + kSharedChunk - 1) / kSharedChunk + kSharedUnitCost);
      } else {
        it.rbs = (it.R + UNIT - 1) / UNIT;
        cost = a.d.Hkv * it.rbs * ((it.keys + BK - 1) / BK + kUnitCost);
      }
    }
    int all, all1;
    const int upto = begun + shared_scan<NT>(cost, all, part, add, 0), upto1 = begun1 + shared_scan<NT>(cost1, all1, part1, add, 0);
    if (i < G) {
      it.start = it.group ? upto1 - cost1 : upto - cost;
      a.item[i] = it;
      a.start[i] = upto - cost;
      a.start1[i] = upto1 - cost1;
    }
    begun += all;
    begun1 += all1;
  }
  for (int c = 0; c < B; c += NT) {
    const int b = c + tid;
    SharedItem it = {0, 0, 0, 0, 0, 1, 0, -1};
    int cost = 0;
    if (b < B) {
      const int q = c == 0 ? group : group_of(b), n = c == 0 ? mine : tokens(b);
      it.group = q;
      if (q >= 0) {
        const int P = prefix(q);
        if (n >= P && shared_peek<LDS>(count + q) > 1) it.key0 = P;
      }
      it.keys = n - it.key0;
      it.row = it.b0 = b;
      it.R = a.g;
      it.rbs = a.own_rbs;
      if (it.keys > 0) cost = a.d.Hkv * it.rbs * ((it.keys + BK - 1) / BK + kUnitCost);
    }
    int all;
    const int upto = begun + shared_scan<NT>(cost, all, part, add, 0);
    if (b < B) {
      it.start = upto - cost;
      a.item[G + b] = it;
      a.start[G + b] = upto - cost;
    }
    begun += all;
  }
  if (tid < 4) a.sums[tid] = shared_sum(a, begun, begun1, tid);
}

// The list of few requests and groups, in LDS: each workgroup makes its own and needs no launch before it.
constexpr int kSmall = 256;
struct SharedSmall {
  int first[kSmall + 1], leader[kSmall], count[kSmall], len[kSmall], start1[kSmall];
  int tokens[kSmall], key0[kSmall], group[kSmall], start[2 * kSmall];
  int sums[4], part[kThreads / kWave], part1[kThreads / kWave];
};

// The last of n items that begins at block x or before it (items without a block begin where the next one does).  64 looked at a step.
__device__ __forceinline__ int shared_locate(const int32_t* start, int n, int x, int lane) {
  int lo = 0, hi = n;   // it is in [lo, hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const unsigned long long up = __ballot(at < hi && start[at] <= x);   // (lane 0 always)
    const int last = 63 - (int)__builtin_clzll(up);
    const int from = lo + last * step;
    hi = min(hi, from + step);
    lo = from;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ SharedItem shared_item(const SharedItem* items, int i) {   // by scalar loads
  typedef const SharedItem __attribute__((address_space(4)))* scalar_ptr;
  scalar_ptr p = (scalar_ptr)(uintptr_t)(items + __builtin_amdgcn_readfirstlane(i));
  SharedItem it;
  it.keys = p->keys; it.key0 = p->key0; it.row = p->row; it.b0 = p->b0; it.R = p->R; it.rbs = p->rbs; it.start = p->start; it.group = p->group;
  return it;
}
// What a kernel knows of the list: from the workspace, or (SMALL) from its own.
template <int BK, int UNIT, bool SMALL>
struct SharedList {
  const SharedArgs& a;
  SharedSmall* s;
  __device__ __forceinline__ int sum(int k) const { return SMALL ? __builtin_amdgcn_readfirstlane(s->sums[k]) : a.sums[k]; }
  __device__ __forceinline__ int start(int i) const { return SMALL ? s->start[i] : a.start[i]; }
  __device__ __forceinline__ int locate(int x, int lane) const {
    return SMALL ? shared_locate(s->start, a.G + a.d.B, x, lane) : shared_locate(a.start, a.G + a.d.B, x, lane);
  }
  __device__ __forceinline__ int locate1(int x, int lane) const {
    return SMALL ? shared_locate(s->start1, a.G, x, lane) : shared_locate(a.start1, a.G, x, lane);
  }
  __device__ __forceinline__ SharedItem group(int i) const {   // SMALL
    SharedItem it = {0, 0, 0, 0, 0, 1, 0, 0};
    if (s->count[i] > 1) {
      it.keys = s->len[i];
      it.row = s->leader[i];
      it.b0 = s->first[i];
      it.R = (s->first[i + 1] - it.b0) * a.g;
      it.group = shared_is_big(a, it.R, it.keys);
      it.rbs = it.group ? (it.R + kSharedRows - 1) / kSharedRows : (it.R + UNIT - 1) / UNIT;
    }
    it.start = it.group ? s->start1[i] : s->start[i];
    return it;
  }
  __device__ __forceinline__ SharedItem request(int b) const {   // SMALL
    const int key0 = s->key0[b];
    return SharedItem{s->tokens[b] - key0, key0, b, b, a.g, a.own_rbs, s->start[a.G + b], s->group[b]};
  }
  __device__ __forceinline__ SharedItem item(int i) const {   // uniform
    if (!SMALL) return shared_item(a.item, i);
    SharedItem it = i < a.G ? group(i) : request(i - a.G);
    int* f = reinterpret_cast<int*>(&it);
#pragma unroll
    for (int k = 0; k < (int)(sizeof(it) / 4); ++k) f[k] = __builtin_amdgcn_readfirstlane(f[k]);
    return it;
  }
  __device__ __forceinline__ int cost(const SharedItem& it) const {   // blocks of an item that shared_run forms
    return it.keys > 0 ? a.d.Hkv * it.rbs * ((it.keys + BK - 1) / BK + kUnitCost) : 0;
  }
  __device__ __forceinline__ int cost1(const SharedItem& it) const {   // chunks of one that shared_prefix forms
    return a.d.Hkv * it.rbs * ((it.keys + kSharedChunk - 1) / kSharedChunk + kSharedUnitCost);
  }
  // B <= kSmall, G < kSmall, kThreads threads.  `write`: into the workspace, too, for the join.
  __device__ __forceinline__ void plan(bool write) {
    const int tid = threadIdx.x, B = a.d.B, G = a.G, cap = a.d.Sk;
    const int n = tid < B ? min(max(a.d.len[tid], 0), cap) : 0;
    const int P = tid < G ? min(max(a.share_len[tid], 0), cap) : 0;
    const int f = tid <= G ? min(max(a.share_first[tid], 0), B) : 0;
    auto add = [](int x, int y) { return x + y; };
    auto top = [](int x, int y) { return max(x, y); };
    int all, all1;
    const int first = shared_scan<kThreads>(f, all, s->part, top, 0);
    s->len[tid] = P;
    s->leader[tid] = B;
    s->count[tid] = 0;
    s->tokens[tid] = n;
    if (tid <= G) s->first[tid] = first;
    __syncthreads();
    int q = -1;
    if (tid < B) {
      int lo = -1, hi = G;   // as in shared_plan_kernel
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s->first[mid] <= tid) lo = mid;
        else hi = mid;
      }
      if (lo >= 0 && tid < s->first[lo + 1]) q = lo;
      if (q >= 0 && s->len[q] > 0 && n >= s->len[q]) {
        atomicMin(&s->leader[q], tid);
        atomicAdd(&s->count[q], 1);
      }
    }
    s->group[tid] = q;
    __syncthreads();
    SharedItem it = {0, 0, 0, 0, 0, 1, 0, 0};
    if (tid < G) it = group(tid);   // (its start is not known yet)
    const int c = it.group ? 0 : cost(it), c1 = it.group ? cost1(it) : 0;
    const int upto = shared_scan<kThreads>(c, all, s->part, add, 0), upto1 = shared_scan<kThreads>(c1, all1, s->part1, add, 0);
    if (tid < G) {
      it.start = it.group ? upto1 - c1 : upto - c;
      s->start[tid] = upto - c;
      s->start1[tid] = upto1 - c1;
      if (write) a.item[tid] = it;
    }
    SharedItem own = {0, 0, 0, 0, 0, 1, 0, -1};
    s->key0[tid] = q >= 0 && n >= s->len[q] && s->count[q] > 1 ? s->len[q] : 0;
    if (tid < B) own = request(tid);
    const int co = tid < B ? cost(own) : 0;
    int all_own;
    const int own_upto = all + shared_scan<kThreads>(co, all_own, s->part, add, 0);
    if (tid < B) {
      own.start = own_upto - co;
      s->start[G + tid] = own.start;
      if (write) a.item[G + tid] = own;
    }
    if (tid < 4) {
      const int v = shared_sum(a, all + all_own, all1, tid);
      s->sums[tid] = v;
      if (write) a.sums[tid] = v;
    }
    __syncthreads();
  }
};

// Row r of K/V head hk of an item, in Q, O and the records.
__device__ __forceinline__ size_t shared_row(const SharedArgs& a, int b0, int hk, int r) {
  const int n = a.by_g.div(r);
  return ((size_t)(b0 + n) * a.d.Hkv + hk) * a.g + (r - n * a.g);
}

// ---- units of 16 rows
struct SharedBlock {
  int i, unit, blk, nb, left;   // item, its unit, block of the unit, blocks of a unit, what is left of the run
  SharedItem it;
};

template <class Core, class List>
__device__ __forceinline__ void shared_run(const SharedArgs& a, const List& list, unsigned char* lds) {   // lds: the wave's Core::LDS bytes
  typedef typename Core::Elt Elt;
  constexpr int BK = Core::BK, KPL = Core::KPL, RB = Core::RB, UNIT = RB * kDecodeRows;
  const DecodeArgs& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // where prefixes are most of the work, the second half of the workgroups has the runs
  const int waves = list.sum(3), n_items = a.G + d.B, run = blockIdx.x * 4 + wave - (d.waves - waves);
  const int total = list.sum(0), per = run_length(total, waves);
  if (run < 0 || (int64_t)run * per >= total) return;
  Core core(d, lds, lane);
  const int D = core.dim();

  auto item = [&](SharedBlock& s, int i) {
    s.i = i;
    s.it = list.item(i);
    s.unit = 0;
    s.nb = (s.it.keys + BK - 1) / BK;
  };
  auto next = [&](SharedBlock& s) {   // false: the run ends
    const bool last = s.blk + 1 == s.nb;
    s.left -= last ? 1 + kUnitCost : 1;
    s.blk = last ? 0 : s.blk + 1;
    s.unit += last ? 1 : 0;
    if (last && s.left > 0 && s.unit == d.Hkv * s.it.rbs) {   // the next item that has a block
      const int done = s.it.start + s.unit * (s.nb + kUnitCost);
      int i = s.i + 1;
      for (;; i += kWave) {   // (there is one)
        const unsigned long long up = __ballot(i + lane + 1 >= n_items || list.start(i + lane + 1) > done);
        if (up) {
          i += (int)__builtin_ctzll(up);
          break;
        }
      }
      item(s, i);
    }
    return s.left > 0;
  };
  SharedBlock now, then, later;
  {
    const int x = run * per;
    item(now, list.locate(x, lane));
    now.left = min(per, total - x);
    const int in = x - now.it.start, cost = now.nb + kUnitCost;
    now.unit = in / cost;
    now.blk = in - now.unit * cost;
    if (now.blk >= now.nb) {   // behind a unit's last block
      now.left -= now.nb + kUnitCost - now.blk - 1;
      now.blk = now.nb - 1;
      now.left += kUnitCost;
      if (!next(now)) return;
    }
  }
  auto ask = [&](const SharedBlock& s, int(&page)[KPL]) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) {
      const int j = BK * s.blk + core.key(t);
      page[t] = j < s.it.keys ? d.table[(size_t)s.it.row * d.max_pages + d.by_ps.div(s.it.key0 + j)] : 0;
    }
  };
  auto place = [&](const SharedBlock& s, const int(&page)[KPL], int64_t(&at)[KPL]) {
#pragma unroll
    for (int t = 0; t < KPL; ++t) {
      const int j = BK * s.blk + core.key(t), token = s.it.key0 + j;
      at[t] = j < s.it.keys && (unsigned)page[t] < (unsigned)d.n_pages
                  ? page[t] * d.page_stride + (int64_t)(token - d.by_ps.div(token) * d.ps) * D : -1;
    }
  };
  auto head_of = [&](const SharedBlock& s) { return s.it.rbs == 1 ? s.unit : s.unit / s.it.rbs; };
  auto base_of = [&](const void* p, const SharedBlock& s) { return static_cast<const Elt*>(p) + (size_t)head_of(s) * d.head_stride; };
  auto row_of = [&](const SharedBlock& s) { return UNIT * (s.unit - head_of(s) * s.it.rbs) + core.i; };   // the lane's, of the item's rows
  auto both = [&](const SharedBlock& s) { return RB == 2 && UNIT * (s.unit - head_of(s) * s.it.rbs) + kDecodeRows < s.it.R; };   // uniform
  auto load_q = [&](typename Core::Query& q, const SharedBlock& s, int x) {   // of row block x
    core.load_row(q, static_cast<const Elt*>(d.Q) + shared_row(a, s.it.b0, head_of(s), min(row_of(s) + kDecodeRows * x, s.it.R - 1)) * D);
  };

  typename Core::Query q, q1, q_then;   // (q1 is not asked for ahead: registers)
  int page[KPL];
  int64_t at[KPL], at_then[KPL];
  ask(now, page);
  load_q(q, now, 0);
  if (both(now)) load_q(q1, now, 1);
  then = now;
  bool more = next(then);
  place(now, page, at);
  core.load_k(base_of(d.K, now), at);
  core.load_v(base_of(d.V, now), at);
  if (more) ask(then, page);
  core.reset();
  int begin = now.blk;
  while (true) {
    typename Core::Scores s, s1;
    const bool two = both(now);
    core.scores(s, q);
    if (RB == 2 && two) core.scores(s1, q1);
    const bool last = now.blk + 1 == now.nb;   // of its unit
    later = then;
    bool more_later = false;
    if (more) {
      place(then, page, at_then);
      if (last) load_q(q_then, then, 0);
      core.load_k(base_of(d.K, then), at_then);
      more_later = next(later);
      if (more_later) ask(later, page);
    }
    core.hide(s, at);
    if (RB == 2 && two) core.hide(s1, at);
    core.stage_v();
    if (Core::LDS && more) core.load_v(base_of(d.V, then), at_then);
    if (Core::LDS) wave_fence();
    core.add(s, d.scale_log2e);
    if (RB == 2 && two) core.add1(s1, d.scale_log2e);
    if (Core::LDS) wave_fence();   // the tile is read before the next block's rows are written
    if (!Core::LDS && more) core.load_v(base_of(d.V, then), at_then);
    if (last || !more) {
      const int hk = head_of(now);
      const size_t rows = shared_rows(a);
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        const float sum = sum_of_four(x ? core.l1 : core.l);
        const int r = row_of(now) + kDecodeRows * x;
        if (r >= now.it.R) continue;
        const size_t rec = begin == 0 && last ? (now.i < a.G ? rows : 0) + shared_row(a, now.it.b0, hk, r)
                                              : 2 * rows + (size_t)(2 * run + (begin == 0)) * UNIT + kDecodeRows * x + core.i;   // as partial_of has it
#pragma unroll
        for (int n = 0; n < Core::NP; ++n) {
          const int c = core.col(n);
          store_partial(a.part + rec * D + c, x ? core.piece1(n) : decode_piece(static_cast<const typename Core::One&>(core), n), c, D);
        }
        if (core.kq == 0) {
          a.stat[2 * rec] = x ? core.m1 : core.m;
          a.stat[2 * rec + 1] = sum;
        }
      }
      if (!more) break;
      core.reset();
      q = q_then;
      if (both(then)) load_q(q1, then, 1);
      begin = 0;
    }
    now = then;
    then = later;
    more = more_later;
#pragma unroll
    for (int t = 0; t < KPL; ++t) at[t] = at_then[t];
  }
}

// ---- prefixes of many rows
// FAR: the cache is larger than a buffer load's 32 bits reach.
template <int D, bool FAR, class List>
__device__ __forceinline__ void shared_prefix(const SharedArgs& a, const List& list, bf16_t* kb0, bf16_t* vb0, bf16_t* kb1, bf16_t* vb1) {
  constexpr int PPR = D / 8, NCOPY = kSharedChunk * PPR / kWave / 4, UNIT = SharedBf16<D>::RB * kDecodeRows;
  typedef typename std::conditional<FAR, int64_t, uint32_t>::type Place;   // elements from the head's first row of the first page; FAR or bytes
  const DecodeArgs& d = a.d;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int il = lane & 31, kh = lane >> 5;
  const int total = list.sum(1), per = list.sum(2);
  const int run = blockIdx.x;   // (neighbouring runs on one XCD, which then share K and V in its L2: as long, at two row blocks a head and at eight)
  if ((int64_t)run * per >= total) return;
  // copies as in cross.hip
  const int slot0 = kWave * wave + lane, crow = slot0 / PPR, cpos = slot0 % PPR;
  const int kpiece = 8 * (cpos ^ k_piece_swizzle<D>(crow)), vpiece = 8 * (cpos ^ v_piece_swizzle<D>(crow));
  StreamTile<D> tile(d.scale_log2e, lane);
  const uint32_t bytes = FAR ? 0 : (uint32_t)(((int64_t)(d.n_pages - 1) * d.page_stride + d.head_stride) * 2);   // of a head, in all pages

  int x = run * per;
  const int end = min(total, x + per);
  int i = list.locate1(x, lane);
  while (x < end) {
    const SharedItem it = list.item(i);
    const int nc = (it.keys + kSharedChunk - 1) / kSharedChunk, cost = nc + kSharedUnitCost;
    const int in = x - it.start, unit = in / cost, c0 = in - unit * cost, c1 = min(nc, c0 + end - x);
    if (unit >= d.Hkv * it.rbs) {   // the next group that has chunks
      i = list.locate1(x, lane);
      continue;
    }
    if (c0 >= nc) {   // behind a unit's last chunk
      x += cost - c0;
      continue;
    }
    const int hk = unit / it.rbs, r = kSharedRows * (unit - hk * it.rbs) + kRowsPerWave * wave + il;
    const bf16_t* K = uniform_ptr(static_cast<const bf16_t*>(d.K) + (size_t)hk * d.head_stride);
    const bf16_t* V = uniform_ptr(static_cast<const bf16_t*>(d.V) + (size_t)hk * d.head_stride);
    const StreamSource ks(K, bytes), vs(V, bytes);
    // Lane l asks for the page of key l of a chunk, two chunks ahead of the products; a chunk ahead it knows the key's place and hands it to the lanes that
    // copy its row.
    auto ask = [&](int c) {
      const int j = c * kSharedChunk + lane;
      return j < it.keys ? d.table[(size_t)it.row * d.max_pages + d.by_ps.div(j)] : -1;
    };
    struct Rows { Place at[NCOPY]; unsigned long long there; };
    auto place = [&](Rows& w, int c, int page) {
      const int j = c * kSharedChunk + lane;
      const bool is = (unsigned)page < (unsigned)d.n_pages;
      const int64_t at = is ? page * d.page_stride + (int64_t)(j - d.by_ps.div(j) * d.ps) * D : 0;   // (0: there, and not used)
      w.there = __ballot(is);
#pragma unroll
      for (int n = 0; n < NCOPY; ++n) {
        if constexpr (FAR) w.at[n] = __shfl((long long)at, crow + 256 / PPR * n);
        else w.at[n] = (uint32_t)__shfl((int)(uint32_t)(2 * at), crow + 256 / PPR * n);
      }
    };
    auto copy = [&](bf16_t* kb, bf16_t* vb, const Rows& w) {
#pragma unroll
      for (int n = 0; n < NCOPY; ++n) {
        bf16_t* to = kb + kWave * 8 * (wave + 4 * n);
        if constexpr (FAR) __builtin_amdgcn_global_load_lds(K + w.at[n] + kpiece, to, 16, 0, 0);
        else ks.copy(to, w.at[n] + 2 * kpiece);
      }
      auto values = [&](int n) {
        bf16_t* to = vb + kWave * 8 * (wave + 4 * n);
        if constexpr (FAR) __builtin_amdgcn_global_load_lds(V + w.at[n] + vpiece, to, 16, 0, 0);
        else vs.copy(to, w.at[n] + 2 * vpiece);
      };
      if (w.there == ~0ull) {   // uniform
#pragma unroll
        for (int n = 0; n < NCOPY; ++n) values(n);
      } else {   // a weight of zero does not make a NaN vanish
#pragma unroll
        for (int n = 0; n < NCOPY; ++n) {
          if ((w.there >> (crow + 256 / PPR * n)) & 1) values(n);
          else *reinterpret_cast<u32x4*>(vb + kWave * 8 * (wave + 4 * n) + 8 * lane) = u32x4{0, 0, 0, 0};
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](const bf16_t* kb, const bf16_t* vb, unsigned long long there) __attribute__((always_inline)) {
      tile.chunk(kb, vb, [&](f32x16& s0, f32x16& s1) {
        if (there != ~0ull) {   // uniform
          const uint32_t lo = (uint32_t)there >> (4 * kh), hi = (uint32_t)(there >> 32) >> (4 * kh);
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            s0[v] = (lo >> mfma_row(v, 0)) & 1 ? s0[v] : -INFINITY;
            s1[v] = (hi >> mfma_row(v, 0)) & 1 ? s1[v] : -INFINITY;
          }
        }
      });
    };
    auto publish = [&]() {   // this wave's copies have landed, then everybody's; the other stage is no longer read
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
    };
    __syncthreads();   // the stages are no longer read
    Rows now, next;
    int page = ask(c0);
    tile.load_q(static_cast<const bf16_t*>(d.Q) + shared_row(a, it.b0, hk, min(r, it.R - 1)) * D);
    place(now, c0, page);
    copy(kb0, vb0, now);
    if (c0 + 1 < c1) place(next, c0 + 1, ask(c0 + 1));
    tile.reset();
#pragma unroll 1
    for (int c = c0; c < c1; c += 2) {   // now: what lies in the first stage; next: the chunk behind it
      publish();
      if (c + 1 < c1) copy(kb1, vb1, next);
      if (c + 2 < c1) page = ask(c + 2);
      step(kb0, vb0, now.there);
      if (c + 1 >= c1) break;
      if (c + 2 < c1) place(now, c + 2, page);
      publish();
      if (c + 2 < c1) copy(kb0, vb0, now);
      if (c + 3 < c1) page = ask(c + 3);
      step(kb1, vb1, next.there);
      if (c + 3 < c1) place(next, c + 3, page);
    }
    const float sum = tile.sum();
    if (r < it.R) {
      const size_t rows = shared_rows(a);
      const size_t rec = c0 == 0 && c1 == nc ? rows + shared_row(a, it.b0, hk, r)
                                             : 2 * rows + (size_t)2 * d.waves * UNIT +
                                                   (size_t)(2 * run + (c0 == 0)) * kSharedRows + kRowsPerWave * wave + il;
      float* to = a.part + rec * D + 4 * kh;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int vq = 0; vq < 4; ++vq) {
          const f32x16& t = tile.acc[db];
          *reinterpret_cast<f32x4*>(to + 32 * db + 8 * vq) = f32x4{t[4 * vq], t[4 * vq + 1], t[4 * vq + 2], t[4 * vq + 3]};
        }
      if (kh == 0) {
        a.stat[2 * rec] = tile.m;
        a.stat[2 * rec + 1] = sum;
      }
    }
    x += c1 - c0 + (c1 == nc ? kSharedUnitCost : 0);
  }
}

template <class Core>
using SharedListOf = SharedList<Core::BK, Core::RB * kDecodeRows, true>;
template <class Core>
using SharedListIn = SharedList<Core::BK, Core::RB * kDecodeRows, false>;

template <class Core, bool SMALL>
__global__ __launch_bounds__(kThreads, Core::WGS) void shared_run_kernel(const SharedArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[Core::LDS ? 4 * Core::LDS : 16];
  unsigned char* mine = lds + (Core::LDS ? (threadIdx.x >> 6) * Core::LDS : 0);
  if constexpr (SMALL) {
    __shared__ SharedSmall small;
    SharedListOf<Core> list{a, &small};
    list.plan(blockIdx.x == 0);
    shared_run<Core>(a, list, mine);
  } else {
    shared_run<Core>(a, SharedListIn<Core>{a, nullptr}, mine);
  }
}
// Both in one launch: a workgroup has its share of the one and of the other.
template <int D, bool FAR, bool SMALL>
__global__ __launch_bounds__(kThreads, 2) void shared_both_kernel(const SharedArgs a) {
  typedef SharedBf16<D> Core;
  __shared__ __attribute__((aligned(16))) bf16_t kb0[kSharedChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb0[kSharedChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t kb1[kSharedChunk * D];
  __shared__ __attribute__((aligned(16))) bf16_t vb1[kSharedChunk * D];
  static_assert(Core::LDS <= (int)sizeof(kb0), "a wave's V tile in a stage");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* mine = reinterpret_cast<unsigned char*>(wave == 0 ? kb0 : wave == 1 ? vb0 : wave == 2 ? kb1 : vb1);
  auto both = [&](const auto& list) __attribute__((always_inline)) {
    shared_prefix<D, FAR>(a, list, kb0, vb0, kb1, vb1);
    __syncthreads();
    shared_run<Core>(a, list, mine);
  };
  if constexpr (SMALL) {
    __shared__ SharedSmall small;
    SharedListOf<Core> list{a, &small};
    list.plan(blockIdx.x == 0);
    both(list);
  } else {
    both(SharedListIn<Core>{a, nullptr});
  }
}

// ---- parts of an output row
constexpr int kSharedManyRows = 6144;   // from here on shared_rows_kernel
// NW waves add up one row (or, NW 1, a wave each): a lane holds four columns, G lanes a partial result; a wave knows the weights of 64 at once.
template <bool F32, int G, int NW>
__global__ __launch_bounds__(NW == 1 ? kThreads : NW * kWave) void shared_join_kernel(const SharedArgs a) {
  typedef typename std::conditional<F32, float, bf16_t>::type Elt;
  constexpr int BK = F32 ? 16 : 32, UNIT = F32 ? 16 : 32, SUB = kWave / G;
  __shared__ __attribute__((aligned(16))) f32x4 sums[NW][G];
  __shared__ float ms[NW], ls[NW];
  const DecodeArgs& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = lane / G, col = 4 * (lane % G), D = d.D;
  const size_t rows = shared_rows(a);
  const size_t row = NW == 1 ? (size_t)blockIdx.x * (kThreads / kWave) + wave : blockIdx.x;
  if (row >= rows) return;   // (all of the workgroup's waves, where they meet)
  const int head = (int)(row / a.g), x = (int)(row - (size_t)head * a.g), b = head / d.Hkv, hk = head - b * d.Hkv;
  const int per = run_length(a.sums[0], a.sums[3]), per1 = a.sums[2];
  // the parts of an item's row: of runs [w0, w0 + n), or (whole) one by itself
  struct Parts {
    int n, w0, per, from;
    size_t base;     // record of the first part, or of run 0
    int stride;      // records of a run; 0: whole
  };
  auto parts_of = [&](const SharedItem& it, int r, bool big, size_t whole) {
    Parts p = {0, 0, 1, 0, whole, 0};
    const int br = big ? kSharedRows : UNIT, blocks = big ? (it.keys + kSharedChunk - 1) / kSharedChunk : (it.keys + BK - 1) / BK;
    if (blocks == 0) return p;
    p.per = big ? per1 : per;
    p.from = it.start + (hk * it.rbs + r / br) * (blocks + (big ? kSharedUnitCost : kUnitCost));
    p.w0 = p.from / p.per;
    p.n = (p.from + blocks - 1) / p.per - p.w0 + 1;
    if (p.n > 1) {
      p.base = 2 * rows + (big ? (size_t)2 * d.waves * UNIT : 0) + r % br;
      p.stride = br;
    }
    return p;
  };
  const SharedItem own = shared_item(a.item, a.G + b);
  const Parts mine = parts_of(own, x, false, row);
  Parts theirs = {0, 0, 1, 0, 0, 0};
  if (own.key0 > 0) {
    const SharedItem pre = shared_item(a.item, own.group);
    theirs = parts_of(pre, (b - pre.b0) * a.g + x, pre.group != 0, rows + row);
  }
  const int n = mine.n + theirs.n;
  auto record = [&](int e) {
    const Parts& p = e < mine.n ? mine : theirs;
    const int w = p.w0 + (e < mine.n ? e : e - mine.n);
    return p.base + (p.stride ? (size_t)partial_of(w, p.per, p.from) * p.stride : 0);
  };
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, total = 0.f;
  for (int e0 = NW == 1 ? 0 : wave; e0 < n; e0 += NW * kWave) {
    const int e = min(e0 + NW * lane, n - 1);
    const size_t rec = record(e);
    const int here = min(kWave, (n - 1 - e0) / NW + 1);
    // the first parts are asked for beside their maxima and sums; four loads of a lane are on their way at once
    f32x4 y[4];
    auto parts = [&](int k0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + j * SUB + sub;
        const float* src = a.part + (size_t)__shfl((long long)rec, min(k, here - 1)) * D + col;
        y[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (k >= here || col >= D) continue;
        if (!F32 || col + 4 <= D) {
          y[j] = *reinterpret_cast<const f32x4_dw*>(src);
        } else {
#pragma unroll
          for (int c = 0; c < 3; ++c)
            if (col + c < D) y[j][c] = src[c];
        }
      }
    };
    float m = -INFINITY, l = 0.f;
    if (e0 + NW * lane < n) {
      m = a.stat[2 * rec];
      l = a.stat[2 * rec + 1];
    }
    parts(0);
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
    for (int k0 = 0; k0 < here;) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + j * SUB + sub;
        const float weight = __shfl(f, min(k, here - 1));
        o += y[j] * (k < here ? weight : 0.f);
      }
      k0 += 4 * SUB;
      if (k0 < here) parts(k0);
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
    if (wave > 0) return;
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
  if (sub == 0 && col < D) {
    const float inv = total == 0.f ? 0.f : 1.f / total;   // no key at all: zeros
    Elt* to = static_cast<Elt*>(d.O) + row * D + col;
    if constexpr (F32) store_partial(to, o * inv, col, D);
    else DecodeBf16<64>::store(to, o, inv, col, D);
  }
}

// Many rows: G lanes have one, and look at its parts one after another.
template <bool F32, int G>
__global__ __launch_bounds__(kThreads) void shared_rows_kernel(const SharedArgs a) {
  typedef typename std::conditional<F32, float, bf16_t>::type Elt;
  constexpr int BK = F32 ? 16 : 32, UNIT = F32 ? 16 : 32, AT_ONCE = 4;
  const DecodeArgs& d = a.d;
  const int col = 4 * (threadIdx.x % G), D = d.D;
  const size_t rows = shared_rows(a), row = (size_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  if (row >= rows) return;
  const int per = run_length(a.sums[0], a.sums[3]), per1 = a.sums[2];
  const Divider by_per((uint32_t)max(per, 1)), by_per1((uint32_t)max(per1, 1)), by_heads((uint32_t)d.Hkv);
  const int head = a.by_g.div((int)row), x = (int)row - head * a.g, b = by_heads.div(head), hk = head - b * d.Hkv;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, total = 0.f;
  auto item = [&](const SharedItem& it, int r, bool big, size_t whole) {
    const int br = big ? kSharedRows : UNIT, blocks = big ? (it.keys + kSharedChunk - 1) / kSharedChunk : (it.keys + BK - 1) / BK;
    if (blocks == 0) return;
    const int p = big ? per1 : per, from = it.start + (hk * it.rbs + r / br) * (blocks + (big ? kSharedUnitCost : kUnitCost));
    const int w0 = big ? by_per1.div(from) : by_per.div(from), n = (big ? by_per1.div(from + blocks - 1) : by_per.div(from + blocks - 1)) - w0 + 1;
    const size_t base = 2 * rows + (big ? (size_t)2 * d.waves * UNIT : 0) + r % br;
    for (int e0 = 0; e0 < n; e0 += AT_ONCE) {
      f32x4 y[AT_ONCE];
      float m[AT_ONCE], l[AT_ONCE], t = top;
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        m[e] = -INFINITY;
        l[e] = 0.f;
        y[e] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (e0 + e < n) {
          const size_t rec = n == 1 ? whole : base + (size_t)partial_of(w0 + e0 + e, p, from) * br;
          const float* src = a.part + rec * D + col;
          m[e] = a.stat[2 * rec];
          l[e] = a.stat[2 * rec + 1];
          if (!F32 || col + 4 <= D) {
            y[e] = *reinterpret_cast<const f32x4_dw*>(src);
          } else {
#pragma unroll
            for (int c = 0; c < 3; ++c)
              if (col + c < D) y[e][c] = src[c];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) t = fmaxf(t, m[e]);
      const float old = top < t ? __builtin_amdgcn_exp2f(top - t) : 1.f;
      top = t;
      total *= old;
      o *= old;
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        const float f = m[e] < t ? __builtin_amdgcn_exp2f(m[e] - t) : 1.f;
        total = fmaf(l[e], f, total);
        o += y[e] * f;
      }
    }
  };
  const SharedItem own = a.item[a.G + b];
  item(own, x, false, row);
  if (own.key0 > 0) {
    const SharedItem pre = a.item[own.group];
    item(pre, (b - pre.b0) * a.g + x, pre.group != 0, rows + row);
  }
  if (col >= D) return;
  const float inv = total == 0.f ? 0.f : 1.f / total;   // no key at all: zeros
  Elt* to = static_cast<Elt*>(d.O) + row * D + col;
  if constexpr (F32) store_partial(to, o * inv, col, D);
  else DecodeBf16<64>::store(to, o, inv, col, D);
}

// ---- nothing shared, little of it
template <class Core>
__global__ __launch_bounds__(kThreads, Core::OCC) void shared_wave_kernel(const DecodeArgs a) { decode_wave<Core, kPages>(a); }

// ---- launches
static size_t shared_ints(int64_t B, int64_t G) {   // sums, first, leader, count, start, start1, items; in whole pieces of 16 bytes
  return (size_t)((4 + (G + 1) + G + G + (G + B) + G + 3) / 4 * 4 + (G + B) * (int64_t)(sizeof(SharedItem) / 4));
}
static bool shared_big(int64_t B, int32_t g, int32_t D) { return (D == 64 || D == 128) && B * g > kDecodeRows; }   // some group may have many rows
static size_t shared_records(int64_t B, int64_t Hq, int32_t g, int32_t D) {
  return (size_t)(2 * B * Hq) + (size_t)2 * kDecodeWaves * 2 * kDecodeRows + (shared_big(B, g, D) ? (size_t)2 * kSharedWgs * kSharedRows : 0);
}
size_t shared_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t G) {
  return 4 * shared_ints(B, G) + shared_records(B, Hq, Hq / Hkv, D) * (size_t)(D + 2) * sizeof(float);
}
bool shared_fits(int64_t B, int64_t Hkv, int64_t g, int64_t G, int64_t keys) {
  // own items' blocks and prefixes' (a group's last row block may be a single row)
  const double units = (double)Hkv * (B * (double)((g + kDecodeRows - 1) / kDecodeRows) + (double)B * g / kDecodeRows + G);
  return units * ((keys + 15) / 16 + kUnitCost) < 2147483648.0 - 65536 && (double)B * Hkv * g <= 33554432.0;   // (the join's grid)
}

template <class Core>
static hipError_t launch_shared_as(SharedArgs& a, bool big, hipStream_t stream) {
  constexpr bool F32 = Core::BK == 16;
  constexpr int G = Core::NP * 4, UNIT = Core::RB * kDecodeRows;
  a.d.waves = 4 * 256 * Core::WGS;
  a.own_rbs = (a.g + UNIT - 1) / UNIT;
  const bool small = a.d.B <= kSmall && a.G < kSmall;
  hipError_t e = hipSuccess;
  if (!small) {
    if (a.G <= 1024) hipLaunchKernelGGL((shared_plan_kernel<Core::BK, UNIT, 1024, true>), dim3(1), dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL((shared_plan_kernel<Core::BK, UNIT, 1024, false>), dim3(1), dim3(1024), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  auto go = [&](auto kernel, int wgs) { hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(kThreads), 0, stream, a); };
  const int wgs = a.d.waves / 4;
  if constexpr (!F32) {
    static_assert(Core::WGS == 2, "a workgroup has a share of both");
    constexpr int D = Core::NP * 16;
    const bool far = (double)a.d.n_pages * (double)a.d.page_stride * 2 >= 4294967296.0;
    if (big && far) small ? go(&shared_both_kernel<D, true, true>, a.wgs) : go(&shared_both_kernel<D, true, false>, a.wgs);
    else if (big) small ? go(&shared_both_kernel<D, false, true>, a.wgs) : go(&shared_both_kernel<D, false, false>, a.wgs);
    else small ? go(&shared_run_kernel<Core, true>, wgs) : go(&shared_run_kernel<Core, false>, wgs);
  } else {
    small ? go(&shared_run_kernel<Core, true>, wgs) : go(&shared_run_kernel<Core, false>, wgs);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)a.d.B * a.d.Hkv * a.g;
  // us, four waves a row / one: 408 rows of 30 parts 24.7 / 24.9, 2,048 of 17 52.5 / 50.8 (the chip starts some 420 workgroups a us), 4,288 of few 63.8 / 55.1;
  // one / G lanes: 2,048 49.6 / 52.3, 4,288 51.0 / 54.0, 4,816 51.4 / 51.8, 7,056 32.6 / 29.9, 8,736 36.1 / 34.0, 16,384 65.0 / 58.2, 41,280 71.4 / 52.4
  if (rows <= 1024) hipLaunchKernelGGL((shared_join_kernel<F32, G, 4>), dim3((unsigned)rows), dim3(4 * kWave), 0, stream, a);
  else if (rows < kSharedManyRows) hipLaunchKernelGGL((shared_join_kernel<F32, G, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((shared_rows_kernel<F32, G>), dim3((unsigned)((rows * G + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// Where K and V of the most tokens that all requests can have are at most 64 MiB, reading them for each request by itself (mostly from the caches) takes
// less time than finding out what is shared and adding up its parts.  us, shared / by itself: two answers to 16 tokens 10.9 / 4.8, 60 to 200 (61 MiB) 23.2 / 10.0,
// 240 requests on eight heads to 16 tokens 27.1 / 6.5, 64 to 910 tokens (60 MiB) 21.2 / 18.8, 8 to 15,000 (60 MiB) 18.7 / 22.0, 17 in binary32 on eight heads of
// 128 to 1,270 (169 MiB) 21.6 / 26.9, 141 of 64 columns to 1,168 (80 MiB) 15.5 / 20.6, 23 on 12 heads to 768 (104 MiB) 23.3 / 16.5.  Up to 128 tokens that holds for
// any number of requests: 748 on 12 heads of 64, prefixes of 12 tokens 67 / 44, of 102 46 / 43; 256 on eight of 128 38 / 20, 33 / 21; to 256 tokens, prefixes of
// 25 99 / 70 and 49 / 33, of 204 51 / 68 and 36 / 36.  The host knows how many tokens requests can have, not how many they have or share.
constexpr int64_t kSharedWorth = 64LL << 20;
constexpr int kSharedTokens = 128;

hipError_t launch_shared(const SharedLaunch& p, hipStream_t stream) {
  if (p.G == 0 || p.d.Sk <= kSharedTokens || (double)p.d.B * p.d.Hkv * p.d.Sk * p.d.D * (p.d.is_f32 ? 8 : 4) <= (double)kSharedWorth) {
    const DecodeArgs d = decode_args(p.d);
    return decode_with_core(p.d, [&](auto c) {
      typedef typename decltype(c)::Core Core;
      if (!decode_by_wave<Core>(d)) return launch_decode(p.d, stream);
      hipLaunchKernelGGL((shared_wave_kernel<Core>), dim3((unsigned)(((int64_t)d.B * d.Hkv * d.rbs + 3) / 4)), dim3(kThreads), 0, stream, d);
      return hipGetLastError();
    });
  }
  SharedArgs a;
  a.d = decode_args(p.d);
  a.g = p.d.R; a.G = p.G;
  a.share_first = p.share_first; a.share_len = p.share_len;
  a.by_g = Divider((uint32_t)a.g);
  const bool big = !p.d.is_f32 && shared_big(p.d.B, a.g, p.d.D);
  a.big_rows = big ? 2 * kDecodeRows : 0x7fffffff;
  a.big_keys = big && p.d.D == 128 ? 2048 : 0x7fffffff;
  a.wgs = kSharedWgs;
  const int64_t B = p.d.B, G = p.G;
  int32_t* ws = static_cast<int32_t*>(p.d.ws);
  a.sums = ws;
  a.first = ws + 4;
  a.leader = a.first + G + 1; a.count = a.leader + G; a.start = a.count + G; a.start1 = a.start + G + B;
  const size_t ints = shared_ints(B, G);
  a.item = reinterpret_cast<SharedItem*>(ws + ints - (size_t)(G + B) * (sizeof(SharedItem) / 4));
  a.part = reinterpret_cast<float*>(ws + ints);
  const size_t records = shared_records(B, (int64_t)p.d.Hkv * a.g, a.g, p.d.D);
  a.stat = a.part + records * p.d.D;
  if (!p.d.is_f32) return p.d.D == 64 ? launch_shared_as<SharedBf16<64>>(a, big, stream) : launch_shared_as<SharedBf16<128>>(a, big, stream);
  if (p.d.D == 64) return launch_shared_as<SharedF32<1, true>>(a, big, stream);
  if (p.d.D == 128) return launch_shared_as<SharedF32<2, true>>(a, big, stream);
  if (p.d.D < 64) return launch_shared_as<SharedF32<1, false>>(a, big, stream);
  if (p.d.D < 128) return launch_shared_as<SharedF32<2, false>>(a, big, stream);
  if (p.d.D == 256) return launch_shared_as<SharedF32<4, true>>(a, big, stream);
  return launch_shared_as<SharedF32<4, false>>(a, big, stream);
}

}  // namespace ac
