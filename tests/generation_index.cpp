// The index arithmetic of the generation kernels, callable on the host.
#include "../paper_2510_25979_amd/csrc/serve_index.h"

extern "C" int ring_first(int first, int n) { return ac::ring_first(first, n); }
