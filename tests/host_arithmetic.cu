// Arithmetic of the cache's kernels on the host: the same functions, so that a value at which they would go wrong is found without a GPU.
#include "bv_cache.cuh"

extern "C" {
int host_place_of(int len, int m, int t, int width, int page) { return bv::place_of(len, m, t, width, page); }
int host_sum_up_to(int most, int sum, int more) { return bv::sum_up_to(most, sum, more); }
// (the quotient as the device forms it: the high half of a product of 32 bits by 32, a sum and a shift)
int host_divide(unsigned by, int n) {
    const bv::Divider d = bv::divider(by);
    return static_cast<int>((static_cast<unsigned>(static_cast<unsigned long long>(n) * d.mul >> 32) + static_cast<unsigned>(n)) >> d.shift);
}
}
