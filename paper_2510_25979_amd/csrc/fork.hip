// Rows of a paged cache that become other rows: beams that change places, answers that begin at one prompt, requests that end, and
// pages that a window has left behind.
//
// Row b becomes what row from[b] was.  Full pages are shared: the new row names the same ones.  The page in which a row ends will be written, so
// one row keeps it (the row itself if it goes on, otherwise the first that takes it) and each other takes a page from the ring and copies its
// tokens.  A page is free when some row had it and no row has it: two bitmaps of the pages, before and after, say so without a count a page.
//
// Three launches, since each needs all of the one before: the rows (who keeps, who copies, which of the ring's pages; one workgroup, which
// looks at 1,024 rows a step, while others clear the bitmaps), tables, bitmaps and tokens (the whole chip), the ring (one workgroup, pages in order
// of their number; others bring tables that are replaced in place into place).
#include "common.hpp"
#include "serve.h"
#include "serve_index.h"

namespace ac {

struct ForkArgs {
  const int32_t *from, *seq_len, *state, *table;
  int32_t *ring, *table_out, *seq_out, *state_out;
  void *kp, *vp;
  // workspace: of each row its source (-1: none), tokens and entry of the ring (-1: no copy), of each source who keeps its last page; rows
  // that copy, their number and the ring's first entry and number; bitmaps; new tables that replace their source
  int32_t *src, *len, *take, *keeper, *list, *sums, *staged;
  uint32_t *had, *has;
  int32_t B, H, D, max_pages, n, ps, sinks, window, words, segs, row_pieces;
  int64_t page_stride;   // pieces
  Divider by_ps, by_segs;
};

constexpr int kForkRows = 1024;   // threads of the workgroup that plans
constexpr int kForkEntries = 4 * kThreads;   // entries of a table that a workgroup deals with

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
  __shared__ int s_taken;
  const int first = ring_first(a.state[0], a.n), count = min(max(a.state[1], 0), a.n);
  for (int b = tid; b < a.B; b += kForkRows) a.keeper[b] = a.B;
  if (tid == 0) s_taken = 0;
  __threadfence();
  __syncthreads();
  for (int b = tid; b < a.B; b += kForkRows) {
    const int f = a.from[b];
    if ((unsigned)f < (unsigned)a.B) atomicMin(&a.keeper[f], f == b ? -1 : b);
  }
  __threadfence();
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
        const int k = __hip_atomic_load(&a.keeper[f], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
      if (copies && served) {
        a.list[upto - 1] = b;
        atomicMax(&s_taken, upto);
      }
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

// T: a piece of a row, 16 bytes, or 4 where rows are no whole number of those.
template <typename T>
__global__ __launch_bounds__(kThreads) void fork_tables_kernel(const ForkArgs a, int table_wgs) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < table_wgs) {
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
        int page = j == now - 1 && take >= 0 ? fork_ring_page(a, a.sums[0], take) : theirs[j];
        if (fork_gone(a, len, j)) page = -1;
        out[j] = page;
        mark(a.has, page);
      }
    }
    return;
  }
  // Tokens: workgroup w of W serves copy w mod (their number), pieces of it in turn with the others that do.
  const int taken = a.sums[2], w = blockIdx.x - table_wgs, W = gridDim.x - table_wgs;
  if (taken == 0) return;
  for (int i = w % taken; i < taken; i += W) {
    const int slices = taken >= W ? 1 : W / taken + (i < W % taken), slice = taken >= W ? 0 : w / taken;
    const int b = a.list[i], len = a.len[b], src = a.src[b], last = fork_pages_of(a, len) - 1;
    const int page = a.table[(size_t)src * a.max_pages + last], fresh = fork_ring_page(a, a.sums[0], i);
    if ((unsigned)page >= (unsigned)a.n || (unsigned)fresh >= (unsigned)a.n) continue;
    const int run = (len - last * a.ps) * a.row_pieces;   // pieces of a head's tokens, which lie side by side
    const int64_t all = (int64_t)a.H * run, head = (int64_t)a.ps * a.row_pieces, step = (int64_t)slices * kThreads;
    const T* kf = static_cast<const T*>(a.kp) + page * a.page_stride;
    const T* vf = static_cast<const T*>(a.vp) + page * a.page_stride;
    T* kt = static_cast<T*>(a.kp) + fresh * a.page_stride;
    T* vt = static_cast<T*>(a.vp) + fresh * a.page_stride;
    for (int64_t x0 = slice * kThreads + tid; x0 < all; x0 += 2 * step) {
      T k[2], v[2];
      int64_t at[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int64_t x = x0 + u * step;
        at[u] = -1;
        if (x < all) {
          const int h = (int)((uint64_t)x / (uint32_t)run);
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

__global__ __launch_bounds__(kForkRows) void fork_ring_kernel(const ForkArgs a) {
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {   // tables that are replaced in place
    for (int b = blockIdx.x - 1; b < a.B; b += gridDim.x - 1) {
      const int now = a.src[b] >= 0 ? fork_pages_of(a, a.len[b]) : 0;
      for (int j = tid; j < now; j += kForkRows) a.table_out[(size_t)b * a.max_pages + j] = a.staged[(size_t)b * a.max_pages + j];
    }
    return;
  }
  __shared__ int part[kForkRows / kWave];
  const int first = a.sums[0], count = a.sums[1], taken = a.sums[2];
  const unsigned end = ((unsigned)first + (unsigned)count) % (unsigned)a.n;
  int before = 0;
  for (int c = 0; c < a.words; c += kForkRows) {
    uint32_t free = c + tid < a.words ? a.had[c + tid] & ~a.has[c + tid] : 0;
    int all;
    const int n = __popc(free);
    unsigned at = (unsigned)(before + fork_sum<kForkRows>(n, all, part) - n);
    while (free) {
      const int bit = __ffs(free) - 1;
      free &= free - 1;
      a.ring[(end + at % (unsigned)a.n) % (unsigned)a.n] = 32 * (c + tid) + bit;
      ++at;
    }
    before += all;
  }
  for (int b = tid; b < a.B; b += kForkRows) a.seq_out[b] = a.len[b];
  if (tid == 0) {
    a.state_out[0] = (int)(((unsigned)first + (unsigned)taken) % (unsigned)a.n);
    a.state_out[1] = (int)min((unsigned)a.n, (unsigned)(count - taken) + (unsigned)before);
  }
}

static size_t fork_words(int32_t n) { return ((size_t)n + 31) / 32; }
size_t fork_workspace_bytes(int32_t B, int32_t max_pages, int32_t n_pages) {
  return 4 * (4 + 2 * fork_words(n_pages) + 5 * (size_t)B + (size_t)B * max_pages);
}

hipError_t launch_fork(const ForkLaunch& p, hipStream_t stream) {
  ForkArgs a;
  a.from = p.from; a.seq_len = p.seq_len; a.state = p.free_state; a.table = p.page_table;
  a.ring = p.free_pages; a.table_out = p.page_table_out; a.seq_out = p.seq_len_out; a.state_out = p.free_state_out;
  a.kp = p.k_pages; a.vp = p.v_pages;
  a.B = p.B; a.H = p.H; a.D = p.D; a.max_pages = p.max_pages; a.n = p.n_pages; a.ps = p.page_size;
  a.sinks = p.sinks; a.window = p.window;
  a.words = (int)fork_words(p.n_pages);
  int32_t* ws = static_cast<int32_t*>(p.ws);
  a.sums = ws;
  a.had = reinterpret_cast<uint32_t*>(ws + 4);
  a.has = a.had + a.words;
  a.src = ws + 4 + 2 * (size_t)a.words;
  a.len = a.src + p.B; a.take = a.len + p.B; a.keeper = a.take + p.B; a.list = a.keeper + p.B; a.staged = a.list + p.B;
  a.segs = (p.max_pages + kForkEntries - 1) / kForkEntries;
  const int row_bytes = p.D * p.elt;
  const bool wide = row_bytes % 16 == 0;
  a.row_pieces = row_bytes / (wide ? 16 : 4);
  a.page_stride = p.page_stride * p.elt / (wide ? 16 : 4);
  a.by_ps = Divider((uint32_t)p.page_size);
  a.by_segs = Divider((uint32_t)a.segs);
  const int clear = (int)((2LL * a.words + kForkRows - 1) / kForkRows);
  hipLaunchKernelGGL(fork_rows_kernel, dim3((unsigned)(1 + (clear < 1024 ? clear : 1024))), dim3(kForkRows), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tables = p.B * a.segs, copies = 2048;
  if (wide)
    hipLaunchKernelGGL((fork_tables_kernel<u32x4>), dim3((unsigned)(tables + copies)), dim3(kThreads), 0, stream, a, tables);
  else
    hipLaunchKernelGGL((fork_tables_kernel<uint32_t>), dim3((unsigned)(tables + copies)), dim3(kThreads), 0, stream, a, tables);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int back = p.page_table_out == p.page_table ? (p.B < 1024 ? p.B : 1024) : 0;
  hipLaunchKernelGGL(fork_ring_kernel, dim3((unsigned)(1 + back)), dim3(kForkRows), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ac
