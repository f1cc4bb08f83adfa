// Launch descriptors and small helpers of the operators that serve generation: the page plan and K/V rows into their
// pages (page.hip), attention of few rows over pages or an encoder's states (decode.hip) and of many (cross.hip).
// Plain data; validation happens in api.hip before a descriptor is filled.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ac {

// Division of 0 <= n < 2^31 by a positive number that is known when a launch is made (a division by a variable is some
// 30 instructions): n / d = (n + mulhi(n, m)) >> s with m = floor(2^32 (2^s - d) / d) + 1, s = ceil(log2 d).  The sum
// stays below 2^32 because mulhi(n, m) <= n.
struct Divider {
  uint32_t d, m, s;
  Divider() = default;
  __host__ __device__ explicit Divider(uint32_t by) : d(by), s(by > 1 ? 32 - __builtin_clz(by - 1) : 0) {
    m = (uint32_t)((((1ull << s) - d) << 32) / d + 1);
  }
  __device__ __forceinline__ int div(int n) const {
    return (int)(((uint32_t)n + __umulhi((uint32_t)n, m)) >> s);
  }
};

struct PlanLaunch {
  const int32_t *seq_len, *new_len, *free_state;   // device [B], [B], [2]; the outputs may be the same arrays
  int32_t *free_pages, *page_table;                // device [n_pages], [B][max_pages]
  int32_t *seq_len_out, *added, *free_state_out;   // device [B], [B], [2]
  int32_t* slot;                                   // device [B][S]
  int32_t B, S, max_pages, page_size, n_pages;
};
hipError_t launch_plan(const PlanLaunch& p, hipStream_t stream);

struct AppendLaunch {
  const void *K, *V;       // device [B][H][S][D]
  const int32_t* slot;     // device [B][S]
  void *k_pages, *v_pages;
  int32_t B, H, S, D, n_pages, page_size, elt;   // elt: bytes of an element
  int64_t page_stride;     // elements
};
hipError_t launch_append(const AppendLaunch& p, hipStream_t stream);

// A projection's rows to heads (rotate.hip).
struct RotateLaunch {
  const void* X;                       // device [B][S] rows of Hq + 2 Hkv heads
  const float *q_weight, *k_weight;    // device [D] or nullptr
  const int32_t* pos;                  // device [B][S]
  const double* freq;                  // device [rot / 2]
  const int32_t* slot;                 // device [B][S] or nullptr
  void *Q, *K, *V;                     // device [B][Hq][S][D], [B][Hkv][S][D] or nullptr
  void *k_pages, *v_pages;             // with a slot
  int64_t batch_stride, row_stride, page_stride;   // elements
  int32_t B, S, Hq, Hkv, D, rot, n_pages, page_size, is_f32, interleaved;
  float eps, amplitude;
};
hipError_t launch_rotate(const RotateLaunch& p, hipStream_t stream);

// Rows of a paged cache that become other rows (fork.hip); the outputs may be the inputs of the same meaning.
struct ForkLaunch {
  const int32_t *from, *seq_len, *free_state, *page_table;   // device [B], [B], [2], [B][max_pages]
  int32_t *free_pages, *page_table_out, *seq_len_out, *free_state_out;
  void *k_pages, *v_pages;
  int32_t B, H, D, max_pages, n_pages, page_size, sinks, window, elt;
  int64_t page_stride;   // elements
  void* ws;
};
size_t fork_workspace_bytes(int32_t B, int32_t max_pages, int32_t n_pages);
hipError_t launch_fork(const ForkLaunch& p, hipStream_t stream);

// Attention of R rows per (item, K/V head), which lie side by side in Q and O, over the keys of that head.
struct DecodeLaunch {
  const void *Q, *K, *V;    // K, V: pages, or [B][Hkv][Sk][D]
  void* O;
  const int32_t* table;     // device [B][max_pages], nullptr: K and V are not paged
  const int32_t* len;       // device [B] or nullptr (all Sk)
  const int32_t* row_sel;   // device [B] or nullptr
  int32_t B, Hkv, R, D, Sk, is_f32;   // Sk: the most keys an item can have
  int32_t n_pages, page_size, max_pages;
  int64_t page_stride;
  float scale;              // 0: 1 / sqrt(D)
  void* ws;
  int32_t sinks, window;    // launch_window_step: first and last keys that are seen
};
size_t decode_workspace_bytes(int32_t R, int32_t D);
bool decode_fits(int64_t B, int64_t Hkv, int64_t R, int64_t keys);   // the blocks of a call can be counted in 31 bits
hipError_t launch_decode(const DecodeLaunch& p, hipStream_t stream);
hipError_t launch_window_step(const DecodeLaunch& p, hipStream_t stream);   // over pages (window_step.hip)

// Cross attention: the same call, not paged.  Many rows go to a kernel that shares K and V between them and needs no
// workspace (cross_workspace_bytes says 0), few to the one above.
size_t cross_workspace_bytes(int32_t B, int32_t Hkv, int32_t R, int32_t Sk, int32_t D, int32_t is_f32);
hipError_t launch_cross(const DecodeLaunch& p, hipStream_t stream);

// One new token of each request over its pages, where consecutive requests share prefixes (shared.hip).
struct SharedLaunch {
  DecodeLaunch d;                            // as for launch_decode, over pages; R heads a K/V head
  const int32_t *share_first, *share_len;    // device [G + 1], [G]
  int32_t G;
};
size_t shared_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t G);
bool shared_fits(int64_t B, int64_t Hkv, int64_t g, int64_t G, int64_t keys);
hipError_t launch_shared(const SharedLaunch& p, hipStream_t stream);

// Attention of prompts within a window (window.hip).
struct WindowLaunch {
  const void *Q, *K, *V;    // device [B][Hq|Hkv][S][D]
  void* O;
  const int32_t *row_sel, *key_len;   // device [B] or nullptr
  int32_t B, Hq, Hkv, S, D, window, sinks, is_f32;
  float scale;
};
hipError_t launch_window(const WindowLaunch& p, hipStream_t stream);

}  // namespace ac
