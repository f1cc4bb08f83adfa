// Bookkeeping of a paged K/V cache: which pages the requests of a step take and give back and where each of their new
// tokens goes (page_plan_kernel), and the copy of K and V rows to those places (page_append_kernel).
//
// The plan.  A request of len tokens holds h = ceil(len / p) pages; n more tokens need d = ceil((len + n) / p) - h new
// ones.  With P the running sum of d over the requests, request b takes entries [P_b - d_b, P_b) of the free pages'
// ring if P_b does not exceed what is there.  Ended requests put their pages behind the ring's last one; these places are
// not among those that are read, so pages go both ways in one launch and without an order among workgroups.
// Bound by latency: dependent loads (lengths -> sums -> ring -> slots), 4.1 us for 64 requests of one token.  From some thousands of requests
// on the workgroup that writes the new state, 256 of them a step, is the longest: 2^20 requests 4.9 ms, 2^22 41.
#include "common.hpp"
#include "serve.h"
#include "serve_index.h"

namespace ac {

struct PlanArgs {
  const int32_t *seq_len, *new_len, *state;
  int32_t *ring, *table, *seq_out, *added, *state_out, *slot;
  int32_t B, S, max_pages, ps, n, rows, seg;   // rows of a workgroup, slots of a row's segment
  Divider by_s, by_ps;
};

struct PlanRequest {
  int len, have, add, need, give;
  bool fits, ended;
};
__device__ __forceinline__ int pages_of(const PlanArgs& a, int tokens) { return tokens ? a.by_ps.div(tokens - 1) + 1 : 0; }
__device__ __forceinline__ PlanRequest plan_request(const PlanArgs& a, int b) {
  const int cap = a.max_pages * a.ps;
  PlanRequest r;
  r.len = min(max(a.seq_len[b], 0), cap);
  const int n = a.new_len[b];
  r.ended = n < 0;
  r.add = min(max(n, 0), a.S);
  r.fits = !r.ended && r.add <= cap - r.len;
  r.have = pages_of(a, r.len);
  r.need = r.fits ? pages_of(a, r.len + r.add) - r.have : 0;
  r.give = r.ended ? r.have : 0;
  return r;
}

// Inclusive sums of x and y over the workgroup's threads, and both totals.
template <int NT>
__device__ __forceinline__ void block_sums(int& x, int& y, int& all_x, int& all_y, int2* part) {
  constexpr int NW = NT / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int px = __shfl_up(x, off), py = __shfl_up(y, off);
    if (lane >= off) {
      x += px;
      y += py;
    }
  }
  if (lane == kWave - 1) part[wave] = make_int2(x, y);
  __syncthreads();
  all_x = all_y = 0;
  int bx = 0, by = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int2 p = part[w];
    if (w < wave) {
      bx += p.x;
      by += p.y;
    }
    all_x += p.x;
    all_y += p.y;
  }
  x += bx;
  y += by;
  __syncthreads();
}

// The last row whose start is not beyond e (rows that take nothing share the start of the next one that does).
__device__ __forceinline__ int row_of(const int* start, int rows, int e) {
  int lo = 0, hi = rows - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= e) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// What workgroups do: kPlanAll one alone does everything (it reads every array that may be written in place before it writes it);
// kPlanRows page table, ring and slots of its rows, summing what lies before them for itself; kPlanState one alone the new lengths
// and the ring's new state; kPlanBoth the last one the state, the others rows, where no output is an input.
// us: 256 prompts of up to 1,024 tokens 10.6 in two launches, 5.3 in one; 64 requests of one token 4.1 in one workgroup of 256
// threads.
enum PlanWork { kPlanAll, kPlanRows, kPlanState, kPlanBoth };
template <int NT, PlanWork WORK>
__global__ __launch_bounds__(NT) void page_plan_kernel(const PlanArgs a) {
  const bool state_too = WORK == kPlanBoth && blockIdx.x == gridDim.x - 1;   // uniform
  const bool rows_too = WORK == kPlanAll || WORK == kPlanRows || (WORK == kPlanBoth && !state_too);
  const bool writes_state = WORK == kPlanAll || WORK == kPlanState || state_too;
  if (state_too && blockIdx.y > 0) return;
  __shared__ int s_len[NT], s_have[NT], s_add[NT], s_new[NT], s_give[NT];
  __shared__ int2 part[NT / kWave];
  __shared__ int s_taken;
  const int tid = threadIdx.x;
  const int r0 = state_too ? 0 : blockIdx.x * a.rows, r1 = state_too ? a.B : min(a.B, r0 + a.rows);
  const int first = ring_first(a.state[0], a.n), count = min(max(a.state[1], 0), a.n);
  int before_new = 0, before_give = 0;   // what the requests before this chunk need and give back
  if (r0 > 0) {
    int x = 0, y = 0, ix, iy;
    for (int b = tid; b < r0; b += NT) {
      const PlanRequest r = plan_request(a, b);
      x += r.need;
      y += r.give;
    }
    ix = x;
    iy = y;
    block_sums<NT>(ix, iy, before_new, before_give, part);
  }
  if (tid == 0) s_taken = 0;   // pages taken by the requests up to here
  for (int c = r0; c < r1; c += NT) {
    const int rows = min(NT, r1 - c), b = c + tid;
    PlanRequest r = {0, 0, 0, 0, 0, false, false};
    if (tid < rows) r = plan_request(a, b);
    int upto = r.need, given = r.give, all_new, all_give;
    block_sums<NT>(upto, given, all_new, all_give, part);
    const bool served = r.fits && (r.need == 0 || upto <= count - before_new);
    const int add = served ? r.add : 0;
    s_len[tid] = r.len;
    s_have[tid] = r.have;
    s_add[tid] = add;
    s_new[tid] = upto - r.need;
    s_give[tid] = given - r.give;
    if (served && r.need > 0) atomicMax(&s_taken, before_new + upto);
    if (writes_state && tid < rows) {
      a.seq_out[b] = r.ended ? 0 : r.len + add;
      a.added[b] = add;
    }
    __syncthreads();
    if (rows_too) {
      // the served requests that need pages come before all others that do: theirs are the ring's next entries
      auto ring_at = [&](int i) {   // entry i < count of the free pages
        const unsigned at = (unsigned)first + (unsigned)i;
        return a.ring[at >= (unsigned)a.n ? at - a.n : at];
      };
      if (blockIdx.y == 0) {
        const int taken = s_taken - before_new;
        for (int e = tid; e < taken; e += NT) {
          const int row = row_of(s_new, rows, e);
          a.table[(size_t)(c + row) * a.max_pages + s_have[row] + e - s_new[row]] = ring_at(before_new + e);
        }
        const unsigned end = ((unsigned)first + (unsigned)count) % (unsigned)a.n;
        for (int e = tid; e < all_give; e += NT) {
          const int row = row_of(s_give, rows, e);
          a.ring[(end + (unsigned)(before_give + e) % (unsigned)a.n) % (unsigned)a.n] =
              a.table[(size_t)(c + row) * a.max_pages + e - s_give[row]];
        }
      }
      const int t0 = blockIdx.y * a.seg, width = min(a.seg, a.S - t0);   // (one row a workgroup where a row has segments)
      const int n_slots = rows * width;
      for (int e = tid; e < n_slots; e += NT) {
        const int row = gridDim.y == 1 ? a.by_s.div(e) : 0, t = t0 + e - row * width;
        int slot = -1;
        if (t < s_add[row]) {
          const int pos = s_len[row] + t, j = a.by_ps.div(pos), have = s_have[row];
          const int page = j < have ? a.table[(size_t)(c + row) * a.max_pages + j] : ring_at(before_new + s_new[row] + j - have);
          if ((unsigned)page < (unsigned)a.n) slot = page * a.ps + pos - j * a.ps;
        }
        a.slot[(size_t)(c + row) * a.S + t] = slot;
      }
      __syncthreads();
    }
    before_new += all_new;
    before_give += all_give;
  }
  if (writes_state && tid == 0) {
    const int taken = s_taken;
    a.state_out[0] = (int)(((unsigned)first + (unsigned)taken) % (unsigned)a.n);
    a.state_out[1] = (int)min((unsigned)a.n, (unsigned)(count - taken) + (unsigned)before_give);
  }
}

constexpr int kPlanSmall = 4096;   // slots that one workgroup writes
hipError_t launch_plan(const PlanLaunch& p, hipStream_t stream) {
  PlanArgs a;
  a.seq_len = p.seq_len; a.new_len = p.new_len; a.state = p.free_state;
  a.ring = p.free_pages; a.table = p.page_table; a.seq_out = p.seq_len_out; a.added = p.added;
  a.state_out = p.free_state_out; a.slot = p.slot;
  a.B = p.B; a.S = p.S; a.max_pages = p.max_pages; a.ps = p.page_size; a.n = p.n_pages;
  a.by_s = Divider((uint32_t)p.S);
  a.by_ps = Divider((uint32_t)p.page_size);
  a.rows = p.B;
  a.seg = p.S;
  if ((int64_t)p.B * p.S <= kThreads) {
    hipLaunchKernelGGL((page_plan_kernel<kThreads, kPlanAll>), dim3(1), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  if ((int64_t)p.B * p.S <= kPlanSmall) {
    hipLaunchKernelGGL((page_plan_kernel<1024, kPlanAll>), dim3(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
  }
  PlanArgs r = a;
  r.rows = plan_rows(p.B, p.S);
  r.seg = r.rows == 1 && p.S > kPlanSlots ? kPlanSlots : p.S;
  const unsigned gx = (unsigned)((p.B + r.rows - 1) / r.rows), gy = (unsigned)((p.S + r.seg - 1) / r.seg);
  if (p.seq_len_out != p.seq_len && p.added != p.new_len && p.free_state_out != p.free_state) {
    hipLaunchKernelGGL((page_plan_kernel<kThreads, kPlanBoth>), dim3(gx + 1, gy), dim3(kThreads), 0, stream, r);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((page_plan_kernel<kThreads, kPlanRows>), dim3(gx, gy), dim3(kThreads), 0, stream, r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((page_plan_kernel<1024, kPlanState>), dim3(1), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

// K and V rows to their pages: row (b, h, t) of the source, [B][H][S][D], to page slot / p, place (h, slot % p).  Nothing is
// computed: bound by memory, each byte read once and written once.  Both sides are whole lines: the rows of one head and
// neighbouring tokens lie side by side in the source and, up to the end of a page, in the cache.  Two pieces a thread and tensor on
// their way at once, streaming stores: 64 prompts of up to 128 tokens, 128 heads of 64 (291 MB) 61 us = 4.8 TB/s (four pieces 60,
// one 66; ordinary stores 65); 1,000 tokens half of which are padding 54 us (four 77, one 55); 128 tokens of 8 heads of 128 2.6 (four 3.3).
struct AppendArgs {
  const void *K, *V;
  const int32_t* slot;
  void *kp, *vp;
  int32_t H, S, ps, n_slots, begin, rows, wg_rows, ppr;   // rows [begin, rows) of this launch; ppr: pieces of a row
  int64_t stride;                                     // of a page, in pieces
  Divider by_s, by_h, by_ps, by_ppr;
};
constexpr int kAppendPieces = 2;

template <typename T>   // a piece: 16 bytes, or 4 where rows are no whole number of those
__global__ __launch_bounds__(kThreads) void page_append_kernel(const AppendArgs a) {
  const int row0 = a.begin + blockIdx.x * a.wg_rows;
  T k[kAppendPieces], v[kAppendPieces];
  int64_t to[kAppendPieces];
#pragma unroll
  for (int n = 0; n < kAppendPieces; ++n) {
    const int i = n * kThreads + threadIdx.x, in = a.by_ppr.div(i), row = row0 + in, piece = i - in * a.ppr;
    to[n] = -1;
    if (in < a.wg_rows && row < a.rows) {
      const int bh = a.by_s.div(row), t = row - bh * a.S, b = a.by_h.div(bh), h = bh - b * a.H;
      const int slot = a.slot[(size_t)b * a.S + t];
      if ((unsigned)slot < (unsigned)a.n_slots) {
        const int page = a.by_ps.div(slot), off = slot - page * a.ps;
        to[n] = page * a.stride + ((int64_t)h * a.ps + off) * a.ppr + piece;
        const size_t from = (size_t)row * a.ppr + piece;
        k[n] = static_cast<const T*>(a.K)[from];
        v[n] = static_cast<const T*>(a.V)[from];
      }
    }
  }
#pragma unroll
  for (int n = 0; n < kAppendPieces; ++n)
    if (to[n] >= 0) {
      __builtin_nontemporal_store(k[n], static_cast<T*>(a.kp) + to[n]);
      __builtin_nontemporal_store(v[n], static_cast<T*>(a.vp) + to[n]);
    }
}

hipError_t launch_append(const AppendLaunch& p, hipStream_t stream) {
  const int row_bytes = p.D * p.elt;
  const bool wide = row_bytes % 16 == 0;
  AppendArgs a;
  a.K = p.K; a.V = p.V; a.slot = p.slot; a.kp = p.k_pages; a.vp = p.v_pages;
  a.H = p.H; a.S = p.S; a.ps = p.page_size; a.n_slots = p.n_pages * p.page_size;
  a.rows = p.B * p.H * p.S;
  a.ppr = row_bytes / (wide ? 16 : 4);
  a.wg_rows = kAppendPieces * kThreads / a.ppr;
  a.stride = p.page_stride * p.elt / (wide ? 16 : 4);
  a.by_s = Divider((uint32_t)p.S);
  a.by_h = Divider((uint32_t)p.H);
  a.by_ps = Divider((uint32_t)p.page_size);
  a.by_ppr = Divider((uint32_t)a.ppr);
  const int most = 1 << 23;   // workgroups of a launch: 2^31 threads
  for (int64_t begin = 0; begin < a.rows; begin += (int64_t)most * a.wg_rows) {
    a.begin = (int)begin;
    const int64_t wgs = (a.rows - begin + a.wg_rows - 1) / a.wg_rows;
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
    if (wide)
      hipLaunchKernelGGL((page_append_kernel<u32x4>), dim3(grid), dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((page_append_kernel<uint32_t>), dim3(grid), dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ac
