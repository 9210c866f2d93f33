// Arithmetic of the cache's kernels on the host: the same functions, so that a value at which they would go wrong is found without a GPU.
#include "bv_cache.cuh"

extern "C" {
int host_place_of(int len, int m, int t, int width, int page) { return bv::place_of(len, m, t, width, page); }
int host_sum_up_to(int most, int sum, int more) { return bv::sum_up_to(most, sum, more); }
}
