// Attention of one new token of each request within a window, with a few first tokens that stay visible: of n tokens, j < sinks and
// j >= n - window are seen.  They are numbered one after the other, and the rest is attention over pages (decode.hip): the same units, runs and
// partial results over at most window + sinks keys, whatever the lengths.  Pages in the gap are not looked at, nor their entries.
#include "decode_tile.h"

namespace ac {

template <class Core>
__global__ __launch_bounds__(kThreads, Core::WGS) void window_step_run_kernel(const DecodeArgs a) { decode_run<Core, kWindow>(a); }
template <class Core, int NW>
__global__ __launch_bounds__(NW* kWave, Core::OCC) void window_step_unit_kernel(const DecodeArgs a) { decode_unit<Core, kWindow, NW>(a); }
template <class Core>
__global__ __launch_bounds__(kThreads, Core::OCC) void window_step_wave_kernel(const DecodeArgs a) { decode_wave<Core, kWindow>(a); }
template <bool F32, int G, int NW>
__global__ __launch_bounds__(NW == 1 ? kThreads : NW * kWave) void window_step_join_kernel(const DecodeArgs a) { decode_join<F32, kWindow, G, NW>(a); }

struct WindowStepKernels {
  static constexpr bool kWave = true;
  template <class Core> static constexpr auto run() { return &window_step_run_kernel<Core>; }
  template <class Core, int NW> static constexpr auto unit() { return &window_step_unit_kernel<Core, NW>; }
  template <class Core> static constexpr auto wave() { return &window_step_wave_kernel<Core>; }
  template <bool F32, int G, int NW> static constexpr auto join() { return &window_step_join_kernel<F32, G, NW>; }
};

hipError_t launch_window_step(const DecodeLaunch& p, hipStream_t stream) {
  DecodeArgs a = decode_args(p);
  // all that an item sees is at most what it can have: both numbers add up below 2^31
  a.window = p.window < a.cap ? p.window : a.cap;
  a.sinks = p.sinks < a.cap - a.window ? p.sinks : a.cap - a.window;
  a.Sk = a.window + a.sinks;
  return launch_decode_as<WindowStepKernels>(p, a, stream);
}

}  // namespace ac
