// The index arithmetic of the generation kernels, callable on the host.
#include "../paper_2510_25979_amd/csrc/serve_index.h"

extern "C" int ring_first(int first, int n) { return ac::ring_first(first, n); }
extern "C" int run_length(int total, int waves) { return ac::run_length(total, waves); }
extern "C" int partial_of(int w, int per, int from) { return ac::partial_of(w, per, from); }
extern "C" int rows_of_a_wave(int rows, int most) { return ac::rows_of_a_wave(rows, most); }
extern "C" int plan_rows(int B, int S) { return ac::plan_rows(B, S); }
