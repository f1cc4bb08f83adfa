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
#include "decode_tile.h"

namespace ac {

template <class Core, DecodeKeys KEYS>
__global__ __launch_bounds__(kThreads, Core::WGS) void decode_run_kernel(const DecodeArgs a) { decode_run<Core, KEYS>(a); }
template <class Core, DecodeKeys KEYS, int NW>
__global__ __launch_bounds__(NW* kWave, Core::OCC) void decode_unit_kernel(const DecodeArgs a) { decode_unit<Core, KEYS, NW>(a); }
template <bool F32, int G, int NW>   // (states and pages alike: a join looks at lengths)
__global__ __launch_bounds__(NW == 1 ? kThreads : NW * kWave) void decode_join_kernel(const DecodeArgs a) { decode_join<F32, kPages, G, NW>(a); }

template <DecodeKeys KEYS>
struct DecodeKernels {
  static constexpr bool kWave = false;
  template <class Core> static constexpr auto run() { return &decode_run_kernel<Core, KEYS>; }
  template <class Core, int NW> static constexpr auto unit() { return &decode_unit_kernel<Core, KEYS, NW>; }
  template <bool F32, int G, int NW> static constexpr auto join() { return &decode_join_kernel<F32, G, NW>; }
};

size_t decode_workspace_bytes(int32_t R, int32_t D) {
  return (size_t)2 * kDecodeWaves * (R < kDecodeRows ? R : kDecodeRows) * (D + 2) * sizeof(float);
}
bool decode_fits(int64_t B, int64_t Hkv, int64_t R, int64_t keys) {
  // blocks of 16 rows and 16 keys (binary32, the smaller ones), and the rows themselves; keys <= 2^30, so their numbers are far from the end
  const double units = (double)B * Hkv * ((R + kDecodeRows - 1) / kDecodeRows);
  return units * ((keys + 15) / 16 + kUnitCost) < 2147483648.0 - 65536 && (double)B * Hkv * R < 2147483648.0 - 65536;
}

hipError_t launch_decode(const DecodeLaunch& p, hipStream_t stream) {
  DecodeArgs a = decode_args(p);
  return p.table ? launch_decode_as<DecodeKernels<kPages>>(p, a, stream) : launch_decode_as<DecodeKernels<kStates>>(p, a, stream);
}

}  // namespace ac
