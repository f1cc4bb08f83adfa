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
  explicit Divider(uint32_t by) : d(by), s(by > 1 ? 32 - __builtin_clz(by - 1) : 0) {
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
};
size_t decode_workspace_bytes(int32_t R, int32_t D);
bool decode_fits(int64_t B, int64_t Hkv, int64_t R, int64_t keys);   // the blocks of a call can be counted in 31 bits
hipError_t launch_decode(const DecodeLaunch& p, hipStream_t stream);

// Cross attention: the same call, not paged.  Many rows go to a kernel that shares K and V between them and needs no
// workspace (cross_workspace_bytes says 0), few to the one above.
size_t cross_workspace_bytes(int32_t B, int32_t Hkv, int32_t R, int32_t Sk, int32_t D, int32_t is_f32);
hipError_t launch_cross(const DecodeLaunch& p, hipStream_t stream);

}  // namespace ac
