// The cache's attention as bv_cache.cu hands it to its kernels, on the runtime of host_runtime.cu: launches check the memory they are given.
#include "host_runtime.cu"

#define launch_attend_tiles fake_launch_attend_tiles
#define launch_attend_rows fake_launch_attend_rows
#include "bv_cache.cuh"

namespace {
int g_kernel = 0, g_refuse_tiles = 0, g_rows = 0;
cudaError_t attended(const bv::AttendArgs& a, int ctas, cudaStream_t st) {
    ++g_launches;
    g_rows = a.rows;
    if (a.rows < 1 || a.span < 1 || a.per_page < 1 || ctas < 1 || ctas > bv::kCacheCounters) complain("a plan that is none");
    return enqueue(st, [=] {
        inside("status word", a.status, 4);
        zeros("counters of the units", a.counters, bv::kCacheCounters * 4);
        scratch("parts", a.part, 2 * ctas * bv::part_floats(a.rows, a.D) * sizeof(float));
        zeros("counters beside the scratch", a.counters, bv::kCacheCounters * 4);
    });
}
}  // namespace
namespace bv {
cudaError_t fake_launch_attend_tiles(const AttendArgs& a, bool, bool, int ctas, cudaStream_t st, bool* taken) {
    *taken = !g_refuse_tiles;
    if (!*taken) return cudaSuccess;
    g_kernel = 1;
    return attended(a, ctas, st);
}
cudaError_t fake_launch_attend_rows(const AttendArgs& a, int, bool, bool, int ctas, cudaStream_t st) {
    g_kernel = 2;
    return attended(a, ctas, st);
}
}  // namespace bv
#include "bv_cache.cu"

extern "C" {
// an attention call on memory that is never touched: its status; then which kernel it took and the rows of its units
int host_attend(int B, int n, int q_heads, int heads, int D, int page, int dtype, long long offset, void* stream) {
    bv_cache c{};
    const int es = dtype == BV_DTYPE_F32 ? 4 : 2;
    c.k = reinterpret_cast<void*>((1ull << 40) + offset * es);
    c.v = reinterpret_cast<void*>(1ull << 41);
    c.table = c.lens = reinterpret_cast<int32_t*>(1ull << 42);
    const int64_t st[3] = {static_cast<int64_t>(heads) * page * D, static_cast<int64_t>(page) * D, D}, qs[3] = {static_cast<int64_t>(n) * q_heads * D, static_cast<int64_t>(q_heads) * D, D};
    for (int i = 0; i < 3; ++i) c.k_stride[i] = c.v_stride[i] = st[i];
    c.B = B; c.width = 100; c.num_pages = 1000; c.page_size = page; c.heads = heads; c.D = D; c.dtype = dtype;
    g_kernel = 0;
    return bv_cache_attend(&c, reinterpret_cast<void*>(1ull << 43), qs, nullptr, n, q_heads, 1.f, 0, 0, reinterpret_cast<void*>(1ull << 44), qs, stream);
}
int host_attend_kernel() { return g_kernel; }
int host_attend_rows() { return g_rows; }
void host_refuse_tiles(int on) { g_refuse_tiles = on; }
}
