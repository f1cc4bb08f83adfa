// Rows of a paged cache that become other rows: beams that change places, answers that begin at one prompt, requests that end, and
// pages that a window has left behind.
//
// Row b becomes what row from[b] was.  Full pages are shared: the new row names the same ones.  The page in which a row ends will be written, so
// one row keeps it (the row itself if it goes on, otherwise the first that takes it) and each other takes a page from the ring and copies its
// tokens.  A page is free when some row had it and no row has it: two bitmaps of the pages, before and after, say so without a count a page.
//
// Bookkeeping of up to 1,024 rows, 8,192 entries and 65,536 pages is one workgroup's work, in LDS; then the tokens are copied by the whole chip.
// Otherwise three launches, since each needs all of the one before: the rows (who keeps, who copies, which of the ring's pages; one workgroup,
// which looks at 1,024 rows a step, while others clear the bitmaps), tables and bitmaps, then the ring (one workgroup, pages in order of their
// number) beside the copies and the way back of tables that are replaced in place.
#include "common.hpp"
#include "serve.h"
#include "serve_index.h"

namespace ac {

struct ForkArgs {
  const int32_t *from, *seq_len, *state, *table;
  int32_t *ring, *table_out, *seq_out, *state_out;
  void *kp, *vp;
  // workspace: of each row its source (-1: none), tokens and entry of the ring (-1: no copy), of each source who keeps its last page; copies
  // (from page, to page, tokens), their number and the ring's first entry and number; bitmaps; new tables that replace their source
  int32_t *src, *len, *take, *keeper, *sums, *staged;
  int4* copy;
  uint32_t *had, *has;
  int32_t B, H, max_pages, n, ps, sinks, window, words, segs, row_pieces, wgs, flat;   // wgs: workgroups that copy; flat: entries of one of fork_flat_kernel
  int64_t page_stride;   // pieces
  Divider by_ps, by_segs, by_max_pages;
};

constexpr int kForkRows = 1024;   // threads of the workgroup that plans
constexpr int kForkEntries = 4 * kThreads;   // entries of a table that a workgroup deals with
constexpr int kForkSmallWords = 2048;        // most of a bitmap in LDS

__device__ __forceinline__ int fork_pages_of(const ForkArgs& a, int tokens) { return tokens > 0 ? a.by_ps.div(tokens - 1) + 1 : 0; }
__device__ __forceinline__ int fork_tokens(const ForkArgs& a, int b) { return min(max(a.seq_len[b], 0), a.max_pages * a.ps); }
// Entry j of a row of len tokens: no token after them sees its page.
__device__ __forceinline__ bool fork_gone(const ForkArgs& a, int len, int j) {
  return a.window > 0 && (int64_t)(j + 1) * a.ps <= (int64_t)len - a.window && (int64_t)j * a.ps >= a.sinks;
}

// Inclusive sum over the workgroup's threads, and the total.
template <int NT>
__device__ __forceinline__ int fork_sum(int x, int& all, int* part) {
  constexpr int NW = NT / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int p = __shfl_up(x, off);
    if (lane >= off) x += p;
  }
  if (lane == kWave - 1) part[wave] = x;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int p = part[w];
    if (w < wave) before += p;
    all += p;
  }
  __syncthreads();
  return x + before;
}

__global__ __launch_bounds__(kForkRows) void fork_rows_kernel(const ForkArgs a) {
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {   // had and has lie side by side
    const int64_t step = (int64_t)(gridDim.x - 1) * kForkRows;
    for (int64_t w = (int64_t)(blockIdx.x - 1) * kForkRows + tid; w < 2LL * a.words; w += step) a.had[w] = 0;
    return;
  }
  __shared__ int part[kForkRows / kWave];
  __shared__ int s_keeper[kForkRows];
  __shared__ int s_taken;
  const int first = ring_first(a.state[0], a.n), count = min(max(a.state[1], 0), a.n);
  const bool few = a.B <= kForkRows;   // keepers in LDS: no fences (100 rows 10.4 us with them, 3.4 so)
  if (tid == 0) s_taken = 0;
  if (few) {
    s_keeper[tid] = a.B;
  } else {
    for (int b = tid; b < a.B; b += kForkRows) a.keeper[b] = a.B;
    __threadfence();
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kForkRows) {
    const int f = a.from[b];
    if ((unsigned)f < (unsigned)a.B) atomicMin(few ? &s_keeper[f] : &a.keeper[f], f == b ? -1 : b);
  }
  if (!few) __threadfence();
  __syncthreads();
  int before = 0;
  for (int c = 0; c < a.B; c += kForkRows) {
    const int b = c + tid;
    int f = -1, len = 0;
    bool copies = false;
    if (b < a.B) {
      f = a.from[b];
      if ((unsigned)f >= (unsigned)a.B) f = -1;
      if (f >= 0) {
        len = fork_tokens(a, f);
        // (as the atomics left it, past the first-level cache)
        const int k = few ? s_keeper[f] : __hip_atomic_load(&a.keeper[f], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        copies = len - a.by_ps.div(len) * a.ps > 0 && (k == -1 ? f : k) != b;
      }
    }
    int all;
    const int upto = before + fork_sum<kForkRows>(copies, all, part);
    if (b < a.B) {
      const bool served = !copies || upto <= count;
      a.src[b] = served ? f : -1;
      a.len[b] = f < 0 ? 0 : served ? len : -1;
      a.take[b] = copies && served ? upto - 1 : -1;
      if (copies && served) atomicMax(&s_taken, upto);
    }
    before += all;
  }
  __syncthreads();
  if (tid == 0) {
    a.sums[0] = first;
    a.sums[1] = count;
    a.sums[2] = s_taken;
  }
}

__device__ __forceinline__ int fork_ring_page(const ForkArgs& a, int first, int i) {   // entry i of the free pages
  const unsigned at = (unsigned)first + (unsigned)i;
  return a.ring[at >= (unsigned)a.n ? at - a.n : at];
}

__global__ __launch_bounds__(kThreads) void fork_tables_kernel(const ForkArgs a) {
  const int tid = threadIdx.x;
  const int b = a.by_segs.div(blockIdx.x), j0 = (blockIdx.x - b * a.segs) * kForkEntries + tid;
  const int held = fork_pages_of(a, fork_tokens(a, b)), src = a.src[b], len = a.len[b], take = a.take[b];
  const int now = src >= 0 ? fork_pages_of(a, len) : 0;
  const int32_t* mine = a.table + (size_t)b * a.max_pages;
  const int32_t* theirs = a.table + (size_t)max(src, 0) * a.max_pages;
  int32_t* out = (a.table_out == a.table ? a.staged : a.table_out) + (size_t)b * a.max_pages;
  auto mark = [&](uint32_t* bits, int page) {
    if ((unsigned)page < (unsigned)a.n) atomicOr(&bits[page >> 5], 1u << (page & 31));
  };
#pragma unroll
  for (int i = 0; i < kForkEntries / kThreads; ++i) {
    const int j = j0 + i * kThreads;
    if (j < held) mark(a.had, mine[j]);
    if (j < now) {
      int page = theirs[j];
      if (j == now - 1 && take >= 0) {
        const int fresh = fork_ring_page(a, a.sums[0], take);
        a.copy[take] = make_int4(page, fresh, len - j * a.ps, 0);
        page = fresh;
      }
      if (fork_gone(a, len, j)) page = -1;
      out[j] = page;
      mark(a.has, page);
    }
  }
}

// The same where the bitmaps fit LDS: workgroups mark a.flat entries each there, and then words at a time in the workspace, where atomics on a few lines
// take turns (24,000 entries 16 us one by one, 5 so).
__global__ __launch_bounds__(kThreads) void fork_flat_kernel(const ForkArgs a) {
  __shared__ uint32_t s_had[kForkSmallWords], s_has[kForkSmallWords];
  const int tid = threadIdx.x;
  for (int w = tid; w < a.words; w += kThreads) s_had[w] = s_has[w] = 0;
  __syncthreads();
  auto mark = [&](uint32_t* bits, int page) {
    if ((unsigned)page < (unsigned)a.n) atomicOr(&bits[page >> 5], 1u << (page & 31));
  };
  int32_t* out = a.table_out == a.table ? a.staged : a.table_out;
  const int e0 = blockIdx.x * a.flat, e1 = e0 + min(a.flat, a.B * a.max_pages - e0);
#pragma unroll 4
  for (int e = e0 + tid; e < e1; e += kThreads) {
    const int b = a.by_max_pages.div(e), j = e - b * a.max_pages, src = a.src[b], len = a.len[b];
    const int now = src >= 0 ? fork_pages_of(a, len) : 0;
    if (j < fork_pages_of(a, fork_tokens(a, b))) mark(s_had, a.table[e]);
    if (j < now) {
      int page = a.table[(size_t)src * a.max_pages + j];
      if (j == now - 1 && a.take[b] >= 0) {
        const int fresh = fork_ring_page(a, a.sums[0], a.take[b]);
        a.copy[a.take[b]] = make_int4(page, fresh, len - j * a.ps, 0);
        page = fresh;
      }
      if (fork_gone(a, len, j)) page = -1;
      out[e] = page;
      mark(s_has, page);
    }
  }
  __syncthreads();
  for (int w = tid; w < a.words; w += kThreads) {
    if (s_had[w]) atomicOr(&a.had[w], s_had[w]);
    if (s_has[w]) atomicOr(&a.has[w], s_has[w]);
  }
}

// The whole plan by one workgroup.  Everything is read before anything is written, since outputs may be inputs.
// us, one workgroup / three launches, replayed and called: 8,000 entries of 16 rows 11.2 / 11.2, 12.2 / 13.9, of 128 rows 12.7 / 12.4, 13.3 / 14.8; 9,600 of 320
// rows 15.3 / 12.9, 15.8 / 14.7; 16,000 of 32 rows 14.1 / 10.9, 14.7 / 13.8; 4,000 of 32 9.9 / 11.3, 11.5 / 14.3.
constexpr int kForkSmallEntries = 8192;
__global__ __launch_bounds__(kForkRows) void fork_small_kernel(const ForkArgs a) {
  constexpr int N = kForkSmallEntries / kForkRows, NW = kForkSmallWords / kForkRows;
  __shared__ int s_keeper[kForkRows], s_src[kForkRows], s_len[kForkRows], s_take[kForkRows], s_held[kForkRows];
  __shared__ uint32_t s_had[kForkSmallWords], s_has[kForkSmallWords];
  __shared__ int part[kForkRows / kWave];
  __shared__ int s_taken;
  const int tid = threadIdx.x;
  const int first = ring_first(a.state[0], a.n), count = min(max(a.state[1], 0), a.n);
  int f = -1, len = 0;
  if (tid < a.B) {
    f = a.from[tid];
    if ((unsigned)f >= (unsigned)a.B) f = -1;
    len = fork_tokens(a, tid);
  }
  s_len[tid] = len;
  s_held[tid] = fork_pages_of(a, len);
  s_keeper[tid] = a.B;
  for (int w = tid; w < a.words; w += kForkRows) s_had[w] = s_has[w] = 0;
  if (tid == 0) s_taken = 0;
  __syncthreads();
  if (f >= 0) {
    atomicMin(&s_keeper[f], f == tid ? -1 : tid);
    len = s_len[f];
  }
  __syncthreads();
  int all;
  const bool copies = f >= 0 && len - a.by_ps.div(len) * a.ps > 0 && (s_keeper[f] == -1 ? f : s_keeper[f]) != tid;
  const int upto = fork_sum<kForkRows>(copies, all, part);
  const bool served = !copies || upto <= count;
  len = f < 0 ? 0 : served ? len : -1;
  s_src[tid] = served ? f : -1;
  s_take[tid] = copies && served ? upto - 1 : -1;
  s_len[tid] = len;
  if (copies && served) atomicMax(&s_taken, upto);
  __syncthreads();
  const int entries = a.B * a.max_pages;
  int page[N];
  auto mark = [&](uint32_t* bits, int q) {   // (rows share pages: most bits are there already, and atomics on one word take turns)
    if ((unsigned)q < (unsigned)a.n && !((bits[q >> 5] >> (q & 31)) & 1)) atomicOr(&bits[q >> 5], 1u << (q & 31));
  };
#pragma unroll
  for (int i = 0; i < N; ++i) {   // (what no row has stays: -2)
    page[i] = -2;
    const int e = i * kForkRows + tid;
    if (i * kForkRows < entries && e < entries) {
      const int b = a.by_max_pages.div(e), j = e - b * a.max_pages, src = s_src[b];
      if (j < s_held[b]) mark(s_had, a.table[e]);
      if (src >= 0 && j < s_held[src]) {
        int q = a.table[src * a.max_pages + j];
        const int take = s_take[b];
        if (take >= 0 && j == s_held[src] - 1) {
          const int fresh = fork_ring_page(a, first, take);
          a.copy[take] = make_int4(q, fresh, s_len[b] - j * a.ps, 0);
          q = fresh;
        }
        if (fork_gone(a, s_len[b], j)) q = -1;
        page[i] = q == -2 ? -1 : q;
        mark(s_has, q);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (page[i] != -2) a.table_out[i * kForkRows + tid] = page[i];
  const unsigned end = ((unsigned)first + (unsigned)count) % (unsigned)a.n;
  uint32_t free[NW];
  int n = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int at = tid * NW + w;
    free[w] = at < a.words ? s_had[at] & ~s_has[at] : 0;
    n += __popc(free[w]);
  }
  unsigned at = (unsigned)(fork_sum<kForkRows>(n, all, part) - n);
#pragma unroll
  for (int w = 0; w < NW; ++w)
    while (free[w]) {
      const int bit = __ffs(free[w]) - 1;
      free[w] &= free[w] - 1;
      a.ring[end + at < (unsigned)a.n ? end + at : end + at - a.n] = 32 * (tid * NW + w) + bit;   // (at < n: each page once)
      ++at;
    }
  if (tid < a.B) a.seq_out[tid] = len;
  if (tid == 0) {
    a.sums[2] = s_taken;
    a.state_out[0] = (int)(((unsigned)first + (unsigned)s_taken) % (unsigned)a.n);
    a.state_out[1] = (int)min((unsigned)a.n, (unsigned)(count - s_taken) + (unsigned)all);
  }
}

// Tokens: workgroup w of W serves copy w mod (their number), pieces of it in turn with the others that do.  T: a piece of a row, 16 bytes,
// or 4 where rows are no whole number of those.
template <typename T>
__device__ __forceinline__ void fork_copy(const ForkArgs& a, int w, int W) {
  const int tid = threadIdx.x, taken = a.sums[2];
  if (taken == 0) return;
  for (int i = w % taken; i < taken; i += W) {
    const int slices = taken >= W ? 1 : W / taken + (i < W % taken), slice = taken >= W ? 0 : w / taken;
    const int4 c = a.copy[i];
    if ((unsigned)c.x >= (unsigned)a.n || (unsigned)c.y >= (unsigned)a.n) continue;
    const int run = c.z * a.row_pieces;   // pieces of a head's tokens, which lie side by side
    const int64_t all = (int64_t)a.H * run, head = (int64_t)a.ps * a.row_pieces, step = (int64_t)slices * kThreads;
    const Divider by_run((uint32_t)run);
    const bool small = all < 0x7fffffff;
    const T* kf = static_cast<const T*>(a.kp) + c.x * a.page_stride;
    const T* vf = static_cast<const T*>(a.vp) + c.x * a.page_stride;
    T* kt = static_cast<T*>(a.kp) + c.y * a.page_stride;
    T* vt = static_cast<T*>(a.vp) + c.y * a.page_stride;
    for (int64_t x0 = slice * kThreads + tid; x0 < all; x0 += 2 * step) {
      T k[2], v[2];
      int64_t at[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t x = x0 + u * step;
        at[u] = -1;
        if (x < all) {
          const int h = small ? by_run.div((int)x) : (int)((uint64_t)x / (uint32_t)run);
          at[u] = h * head + (x - (int64_t)h * run);
          k[u] = kf[at[u]];
          v[u] = vf[at[u]];
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (at[u] >= 0) {
          __builtin_nontemporal_store(k[u], kt + at[u]);
          __builtin_nontemporal_store(v[u], vt + at[u]);
        }
    }
  }
}
template <typename T>
__global__ __launch_bounds__(kThreads) void fork_copy_kernel(const ForkArgs a) { fork_copy<T>(a, blockIdx.x, gridDim.x); }

template <typename T>
__global__ __launch_bounds__(kThreads) void fork_ring_kernel(const ForkArgs a) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= (int)gridDim.x - a.wgs) return fork_copy<T>(a, blockIdx.x - (gridDim.x - a.wgs), a.wgs);
  if (blockIdx.x > 0) {   // tables that are replaced in place
    for (int b = blockIdx.x - 1; b < a.B; b += gridDim.x - a.wgs - 1) {
      const int now = a.src[b] >= 0 ? fork_pages_of(a, a.len[b]) : 0;
      for (int j = tid; j < now; j += kThreads) a.table_out[(size_t)b * a.max_pages + j] = a.staged[(size_t)b * a.max_pages + j];
    }
    return;
  }
  __shared__ int part[kThreads / kWave];
  const int first = a.sums[0], count = a.sums[1], taken = a.sums[2];
  const unsigned end = ((unsigned)first + (unsigned)count) % (unsigned)a.n;
  int before = 0;
  for (int c = 0; c < a.words; c += kThreads) {
    uint32_t free = c + tid < a.words ? a.had[c + tid] & ~a.has[c + tid] : 0;
    int all;
    const int n = __popc(free);
    unsigned at = (unsigned)(before + fork_sum<kThreads>(n, all, part) - n);
    while (free) {
      const int bit = __ffs(free) - 1;
      free &= free - 1;
      a.ring[end + at < (unsigned)a.n ? end + at : end + at - a.n] = 32 * (c + tid) + bit;   // (at < n: each page once)
      ++at;
    }
    before += all;
  }
  for (int b = tid; b < a.B; b += kThreads) a.seq_out[b] = a.len[b];
  if (tid == 0) {
    a.state_out[0] = (int)(((unsigned)first + (unsigned)taken) % (unsigned)a.n);
    a.state_out[1] = (int)min((unsigned)a.n, (unsigned)(count - taken) + (unsigned)before);
  }
}

static size_t fork_words(int32_t n) { return ((size_t)n + 31) / 32; }
size_t fork_workspace_bytes(int32_t B, int32_t max_pages, int32_t n_pages) {
  return 16 * (size_t)B + 4 * (4 + 2 * fork_words(n_pages) + 4 * (size_t)B + (size_t)B * max_pages);
}

template <typename T>
static hipError_t launch_fork_as(const ForkArgs& a, hipStream_t stream) {
  const int entries = a.B * a.max_pages;
  if (a.B <= kForkRows && entries <= kForkSmallEntries && a.words <= kForkSmallWords) {
    hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(kForkRows), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((fork_copy_kernel<T>), dim3((unsigned)a.wgs), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int clear = (int)((2LL * a.words + kForkRows - 1) / kForkRows);
  hipLaunchKernelGGL(fork_rows_kernel, dim3((unsigned)(1 + (clear < 1024 ? clear : 1024))), dim3(kForkRows), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.words <= kForkSmallWords) hipLaunchKernelGGL(fork_flat_kernel, dim3((unsigned)((entries - 1) / a.flat + 1)), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(fork_tables_kernel, dim3((unsigned)(a.B * a.segs)), dim3(kThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int back = a.table_out == a.table ? (a.B < 1024 ? a.B : 1024) : 0;
  hipLaunchKernelGGL((fork_ring_kernel<T>), dim3((unsigned)(1 + back + a.wgs)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_fork(const ForkLaunch& p, hipStream_t stream) {
  ForkArgs a;
  a.from = p.from; a.seq_len = p.seq_len; a.state = p.free_state; a.table = p.page_table;
  a.ring = p.free_pages; a.table_out = p.page_table_out; a.seq_out = p.seq_len_out; a.state_out = p.free_state_out;
  a.kp = p.k_pages; a.vp = p.v_pages;
  a.B = p.B; a.H = p.H; a.max_pages = p.max_pages; a.n = p.n_pages; a.ps = p.page_size;
  a.sinks = p.sinks; a.window = p.window;
  a.words = (int)fork_words(p.n_pages);
  a.flat = a.words > 256 ? 4 * a.words : 1024;   // (several entries for each word that is written)
  a.copy = static_cast<int4*>(p.ws);
  a.sums = static_cast<int32_t*>(p.ws) + 4 * (size_t)p.B;
  a.had = reinterpret_cast<uint32_t*>(a.sums + 4);
  a.has = a.had + a.words;
  a.src = a.sums + 4 + 2 * (size_t)a.words;
  a.len = a.src + p.B; a.take = a.len + p.B; a.keeper = a.take + p.B; a.staged = a.keeper + p.B;
  a.segs = (p.max_pages + kForkEntries - 1) / kForkEntries;
  const int row_bytes = p.D * p.elt;
  const bool wide = row_bytes % 16 == 0;
  a.row_pieces = row_bytes / (wide ? 16 : 4);
  a.page_stride = p.page_stride * p.elt / (wide ? 16 : 4);
  a.by_ps = Divider((uint32_t)p.page_size);
  a.by_segs = Divider((uint32_t)a.segs);
  a.by_max_pages = Divider((uint32_t)p.max_pages);
  // workgroups that copy: as many as 1,024 pieces of the most that there can be make, eight a compute unit
  const double most = (double)p.B * (((double)p.H * p.page_size * a.row_pieces + 1023) / 1024);
  a.wgs = most < 2048 ? (int)most + 1 : 2048;
  return wide ? launch_fork_as<u32x4>(a, stream) : launch_fork_as<uint32_t>(a, stream);
}

}  // namespace ac
