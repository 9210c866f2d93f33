// The paged key-value cache: entry points (contracts in include/bv.h), argument checks, the choice of the attention's kernel, and
// the kernels that only move data (bv_cache_append, bv_pages_copy).
#include <cmath>

#include "bv_cache.cuh"
#include "bv_launch.h"

namespace bv {
namespace {

constexpr double kLog2e = 1.4426950408889634073599246810019;
bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int size_of(int dtype) { return dtype == BV_DTYPE_F32 ? 4 : 2; }
// Are rows of D elements at these strides whole 16-byte vectors on 16-byte boundaries?
bool vectors(const void* p, const int64_t* stride, int D, int es) {
    return on(p, 16) && static_cast<int64_t>(D) * es % 16 == 0 && stride[0] * es % 16 == 0 && stride[1] * es % 16 == 0 && stride[2] * es % 16 == 0;
}
bool none_negative(const int64_t* stride) { return stride[0] >= 0 && stride[1] >= 0 && stride[2] >= 0; }

// The members of a cache that a call uses: `pools` its keys and values, `counts` its pages' counts.
int check_cache(const bv_cache* c, bool pools, bool counts, bool sequences = true) {
    if (!c || c->num_pages < 1 || c->page_size < 1) return BV_ERR_INVALID_ARG;
    if (sequences && (!c->table || !c->lens || !on(c->table, 4) || !on(c->lens, 4) || c->B < 0 || c->width < 1)) return BV_ERR_INVALID_ARG;
    if (counts && (!c->refs || !on(c->refs, 4))) return BV_ERR_INVALID_ARG;
    if (!pools) return BV_OK;
    if (c->dtype != BV_DTYPE_F32 && c->dtype != BV_DTYPE_BF16) return BV_ERR_INVALID_ARG;
    if (!c->k || !c->v || c->heads < 1 || c->D < 1 || !on(c->k, size_of(c->dtype)) || !on(c->v, size_of(c->dtype))) return BV_ERR_INVALID_ARG;
    return none_negative(c->k_stride) && none_negative(c->v_stride) ? BV_OK : BV_ERR_INVALID_ARG;
}
int done(cudaError_t e, int launches) {
    if (e != cudaSuccess) return note_cuda_error(e);
    note_launches(launches);
    return BV_OK;
}

// ---- append ------------------------------------------------------------------------------------------------------------

struct AppendArgs {
    const char* src[2];
    char* dst[2];
    long long ss[2][3];       // bytes between sequences, tokens, heads
    long long ds[2][3];       // bytes between pages, heads, tokens
    const int32_t* table;
    const int32_t* lens;
    const int32_t* n_new;
    int B, n, heads, page, num_pages, width, vecs;
    Divider by_n, by_heads, by_vecs, by_page;
};

// A thread copies the same vector of a row's key and of its value: two loads in flight, then two stores.
template <typename V, typename I>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a, const I total) {
    for (I x = static_cast<I>(blockIdx.x) * 256 + threadIdx.x; x < total; x += static_cast<I>(gridDim.x) * 256) {
        int b, t, h, c;
        if constexpr (sizeof(I) == 4) {
            const int y = a.by_vecs(x), z = a.by_heads(y);
            b = a.by_n(z);
            t = z - b * a.n;
            h = y - z * a.heads;
            c = x - y * a.vecs;
        } else {
            const I y = x / a.vecs, z = y / a.heads;
            b = static_cast<int>(z / a.n);
            t = static_cast<int>(z - static_cast<I>(b) * a.n);
            h = static_cast<int>(y - z * a.heads);
            c = static_cast<int>(x - y * a.vecs);
        }
        const int len = __ldg(a.lens + b);
        const int m = a.n_new ? brought(__ldg(a.n_new + b), a.n) : a.n;
        const int pos = place_of(len, m, t, a.width, a.page);
        if (pos < 0) continue;
        const int j = a.by_page(pos), page = __ldg(a.table + static_cast<long long>(b) * a.width + j);
        if (page < 0 || page >= a.num_pages) continue;
        V val[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) val[w] = *reinterpret_cast<const V*>(a.src[w] + b * a.ss[w][0] + t * a.ss[w][1] + h * a.ss[w][2] + c * sizeof(V));
#pragma unroll
        for (int w = 0; w < 2; ++w) *reinterpret_cast<V*>(a.dst[w] + page * a.ds[w][0] + h * a.ds[w][1] + (pos - j * a.page) * a.ds[w][2] + c * sizeof(V)) = val[w];
    }
}
template <typename V>
cudaError_t launch_append(AppendArgs a, long long row_bytes, cudaStream_t stream) {
    a.vecs = static_cast<int>(row_bytes / static_cast<int>(sizeof(V)));      // (no more than D)
    a.by_n = divider(a.n);
    a.by_heads = divider(a.heads);
    a.by_vecs = divider(a.vecs);
    a.by_page = divider(a.page);
    const long long total = static_cast<long long>(a.B) * a.n * a.heads * a.vecs;
    const long long blocks = (total + 255) / 256;
    const unsigned grid = static_cast<unsigned>(blocks < (1 << 20) ? blocks : (1 << 20));
    if (total + 256LL * grid < (1LL << 31)) append_kernel<V, unsigned><<<grid, 256, 0, stream>>>(a, static_cast<unsigned>(total));
    else append_kernel<V, unsigned long long><<<grid, 256, 0, stream>>>(a, static_cast<unsigned long long>(total));
    return cudaGetLastError();
}

// ---- copies of pages ---------------------------------------------------------------------------------------------------

struct CopyArgs {
    char* pool[2];
    long long ps[2], hs[2], ts[2];    // bytes between pages, heads, tokens
    const int32_t* pairs;     // [n][2] source, destination
    const int32_t* count;     // how many of them count, or null: all
    int n, num_pages;
    bool run[2];              // a page is one run
    int tokens, vecs, all;    // tokens of a head, vectors of a row, of a page
    Divider by_chunks, by_vecs, by_tokens;
};
constexpr int kCopyVecs = 4;

// An item is 16 KB of a pair's page, of its keys or of its values; a thread has four loads in flight.  As many CTAs as items as long as those
// are few: they come and go as memory lets them, which carries 6.0 TB/s for 2048 pages of 64 KB where 8 CTAs an SM that take item after
// item carry 5.4 (6.7 and 5.9 for 16384 pages).  With a count on the device most of the items may be none, so there are at most
// kCopyCtas then, which go on.
constexpr int kCopyCtas = 148 * 64;
template <typename V>
__global__ void __launch_bounds__(256) copy_kernel(const CopyArgs a, const long long most) {
    long long items = most;
    if (a.count) {
        const int n = __ldg(a.count);
        const long long some = 2LL * (n < 0 ? 0 : n < a.n ? n : a.n) * a.by_chunks.by;
        items = some < items ? some : items;
    }
    for (long long x = blockIdx.x; x < items; x += gridDim.x) {
        const long long y = x >> 31 ? x / a.by_chunks.by : a.by_chunks(static_cast<int>(x));
        const int chunk = static_cast<int>(x - y * a.by_chunks.by), w = static_cast<int>(y & 1);
        const int from = __ldg(a.pairs + (y & ~1LL)), into = __ldg(a.pairs + (y | 1));
        if (from < 0 || into < 0 || from >= a.num_pages || into >= a.num_pages || from == into) continue;
        const char* src = a.pool[w] + from * a.ps[w];
        char* dst = a.pool[w] + into * a.ps[w];
        const int first = chunk * kCopyVecs * 256 + threadIdx.x;
        V val[kCopyVecs];
        if (a.run[w]) {
            src += static_cast<long long>(first) * sizeof(V);
            dst += static_cast<long long>(first) * sizeof(V);
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i)
                if (first + i * 256 < a.all) val[i] = *reinterpret_cast<const V*>(src + i * 256 * sizeof(V));
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i)
                if (first + i * 256 < a.all) *reinterpret_cast<V*>(dst + i * 256 * sizeof(V)) = val[i];
        } else {
            long long off[kCopyVecs];
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i) {
                const int z = first + i * 256, row = a.by_vecs(z), h = a.by_tokens(row);
                off[i] = h * a.hs[w] + (row - h * a.tokens) * a.ts[w] + static_cast<long long>(z - row * a.vecs) * sizeof(V);
                if (z < a.all) val[i] = *reinterpret_cast<const V*>(src + off[i]);
            }
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i)
                if (first + i * 256 < a.all) *reinterpret_cast<V*>(dst + off[i]) = val[i];
        }
    }
}
template <typename V>
cudaError_t launch_copy(CopyArgs a, const bv_cache& c, cudaStream_t stream) {
    const int es = size_of(c.dtype);
    for (int w = 0; w < 2; ++w) {
        const int64_t* st = w ? c.v_stride : c.k_stride;
        // a page whose rows lie one after the other, heads or tokens first, is one run
        const bool heads = (st[2] == c.D || c.page_size == 1) && (st[1] == static_cast<int64_t>(c.page_size) * c.D || c.heads == 1);
        const bool tokens = (st[1] == c.D || c.heads == 1) && (st[2] == static_cast<int64_t>(c.heads) * c.D || c.page_size == 1);
        a.run[w] = heads || tokens;
        a.ps[w] = st[0] * es;
        a.hs[w] = st[1] * es;
        a.ts[w] = st[2] * es;
    }
    a.tokens = c.page_size;
    a.vecs = static_cast<int>(static_cast<long long>(c.D) * es / static_cast<int>(sizeof(V)));
    a.all = a.vecs * c.heads * c.page_size;
    a.by_vecs = divider(a.vecs);
    a.by_tokens = divider(a.tokens);
    a.by_chunks = divider((a.all + 256 * kCopyVecs - 1) / (256 * kCopyVecs));
    const long long items = 2LL * a.n * a.by_chunks.by, most = a.count ? kCopyCtas : 0x7fffffff;
    copy_kernel<V><<<static_cast<unsigned>(items < most ? items : most), 256, 0, stream>>>(a, items);
    return cudaGetLastError();
}

// ---- attention ---------------------------------------------------------------------------------------------------------

struct AttendCall {
    AttendArgs a;
    int dtype;
    bool aligned, q_vec, out_vec, tiles;
    cudaStream_t stream;
};
// The kernels for every shape, or the one on the tensor cores.
void plan(AttendCall* c, bool tiles) {
    AttendArgs& a = c->a;
    c->tiles = tiles;
    if (tiles) attend_tiles_plan(&a);
    else attend_rows_plan(&a);
    a.by_group = divider(a.group);
    a.by_page = divider(a.page);
    a.by_span = divider(a.span);
}
int attend_ctas(int sm_count) { return sm_count < kCacheCounters ? sm_count : kCacheCounters; }
size_t attend_scratch(int sm_count, const void* ctx) {
    const AttendCall& c = *static_cast<const AttendCall*>(ctx);
    const int other = attend_rows_most();                                 // (should the first kernel not take the call)
    return attend_ctas(sm_count) * 2 * part_floats(c.a.rows > other ? c.a.rows : other, c.a.D) * sizeof(float);
}
int enqueue_attend(const StreamWork& work, void* ctx) {
    AttendCall& c = *static_cast<AttendCall*>(ctx);
    c.a.part = reinterpret_cast<float*>(work.scratch);
    c.a.counters = work.counters;
    c.a.status = work.status;
    c.a.wait_limit = work.wait_limit;
    c.a.never_signal = work.never_signal;
    const int ctas = attend_ctas(work.sm_count);
    // (a CTA for each part of a unit where there are fewer units than CTAs: of up to 32 sequences, a lane looks at each of them, of three tiles of rows)
    auto few_units = [&] {
        const long long tiles = (c.a.n * c.a.group + c.a.rows - 1) / c.a.rows, units = static_cast<long long>(c.a.B) * c.a.Hkv * tiles;
        if (units >= ctas || c.a.B > 32 || tiles > 3) c.a.slack = -1;
    };
    few_units();
    if (c.tiles) {
        bool taken = false;
        const cudaError_t e = launch_attend_tiles(c.a, c.q_vec, c.out_vec, ctas, c.stream, &taken);
        if (e != cudaSuccess || taken) return done(e, 1);
        plan(&c, false);
        few_units();
    }
    return done(launch_attend_rows(c.a, c.dtype, c.aligned, c.q_vec, ctas, c.stream), 1);
}

}  // namespace
}  // namespace bv

using bv::check_cache;

extern "C" int bv_cache_append(const bv_cache* c, const void* k_new, const int64_t* k_new_stride, const void* v_new,
                               const int64_t* v_new_stride, const int32_t* n_new, int n, void* stream) {
    int rc = check_cache(c, true, false);
    if (rc != BV_OK) return rc;
    const int es = bv::size_of(c->dtype);
    if (!k_new || !v_new || !k_new_stride || !v_new_stride || n < 1 || !bv::on(k_new, es) || !bv::on(v_new, es) || (n_new && !bv::on(n_new, 4)) ||
        !bv::none_negative(k_new_stride) || !bv::none_negative(v_new_stride)) return BV_ERR_INVALID_ARG;
    bv::note_launches(0);
    if (c->B == 0) return BV_OK;
    bv::AppendArgs a{};
    const bool vec = bv::vectors(k_new, k_new_stride, c->D, es) && bv::vectors(v_new, v_new_stride, c->D, es) &&
                     bv::vectors(c->k, c->k_stride, c->D, es) && bv::vectors(c->v, c->v_stride, c->D, es);
    a.src[0] = static_cast<const char*>(k_new); a.src[1] = static_cast<const char*>(v_new);
    a.dst[0] = static_cast<char*>(c->k); a.dst[1] = static_cast<char*>(c->v);
    for (int i = 0; i < 3; ++i) {
        a.ss[0][i] = k_new_stride[i] * es; a.ss[1][i] = v_new_stride[i] * es;
        a.ds[0][i] = c->k_stride[i] * es; a.ds[1][i] = c->v_stride[i] * es;
    }
    a.table = c->table; a.lens = c->lens; a.n_new = n_new;
    a.B = c->B; a.n = n; a.heads = c->heads; a.page = c->page_size; a.num_pages = c->num_pages; a.width = c->width;
    const long long row_bytes = static_cast<long long>(c->D) * es;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return bv::done(vec ? bv::launch_append<uint4>(a, row_bytes, s) : es == 4 ? bv::launch_append<uint32_t>(a, row_bytes, s) : bv::launch_append<uint16_t>(a, row_bytes, s), 1);
}

extern "C" int bv_pages_copy(const bv_cache* c, const int32_t* pairs, int n_pairs, const int32_t* count, void* stream) {
    int rc = check_cache(c, true, false, false);
    if (rc != BV_OK) return rc;
    if (!pairs || n_pairs < 0 || !bv::on(pairs, 4) || (count && !bv::on(count, 4))) return BV_ERR_INVALID_ARG;
    if (static_cast<long long>(c->heads) * c->page_size * c->D > 0x3fffffff) return BV_ERR_UNSUPPORTED;
    bv::note_launches(0);
    if (n_pairs == 0) return BV_OK;
    bv::CopyArgs a{};
    a.pool[0] = static_cast<char*>(c->k); a.pool[1] = static_cast<char*>(c->v);
    a.pairs = pairs; a.count = count; a.n = n_pairs; a.num_pages = c->num_pages;
    const int es = bv::size_of(c->dtype);
    const bool vec = bv::vectors(c->k, c->k_stride, c->D, es) && bv::vectors(c->v, c->v_stride, c->D, es);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return bv::done(vec ? bv::launch_copy<uint4>(a, *c, s) : es == 4 ? bv::launch_copy<uint32_t>(a, *c, s) : bv::launch_copy<uint16_t>(a, *c, s), 1);
}

extern "C" int bv_cache_attend(const bv_cache* c, const void* q, const int64_t* q_stride, const int32_t* n_new, int n, int q_heads,
                               float scale, int window, int sinks, void* out, const int64_t* out_stride, void* stream) {
    int rc = check_cache(c, true, false);
    if (rc != BV_OK) return rc;
    const int es = bv::size_of(c->dtype);
    if (!q || !out || !q_stride || !out_stride || n < 1 || q_heads < 1 || q_heads % c->heads != 0 || window < 0 || sinks < 0 || !std::isfinite(static_cast<float>(scale * bv::kLog2e)) ||
        !bv::on(q, es) || !bv::on(out, es) || (n_new && !bv::on(n_new, 4)) || !bv::none_negative(q_stride) || !bv::none_negative(out_stride)) return BV_ERR_INVALID_ARG;
    const int group = q_heads / c->heads;
    if (c->D > BV_MAX_HEAD_DIM || static_cast<long long>(n) * group > (1 << 30)) return BV_ERR_UNSUPPORTED;
    bv::note_launches(0);
    if (c->B == 0) return BV_OK;
    bv::AttendCall call{};
    bv::AttendArgs& a = call.a;
    a.q = q; a.out = out; a.k = c->k; a.v = c->v;
    a.table = c->table; a.lens = c->lens; a.n_new = n_new;
    for (int i = 0; i < 3; ++i) { a.qs[i] = q_stride[i]; a.os[i] = out_stride[i]; a.ks[i] = c->k_stride[i]; a.vs[i] = c->v_stride[i]; }
    a.B = c->B; a.n = n; a.Hkv = c->heads; a.group = group; a.D = c->D; a.page = c->page_size; a.num_pages = c->num_pages; a.width = c->width;
    a.kf = static_cast<float>(static_cast<double>(scale) * bv::kLog2e);
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    call.dtype = c->dtype;
    call.aligned = bv::vectors(c->k, c->k_stride, c->D, es) && bv::vectors(c->v, c->v_stride, c->D, es);
    call.q_vec = bv::vectors(q, q_stride, c->D, es);
    call.out_vec = bv::vectors(out, out_stride, c->D, es);
    bv::plan(&call, c->dtype == BV_DTYPE_BF16 && call.aligned && bv::attend_tiles_takes(a));
    call.stream = static_cast<cudaStream_t>(stream);
    return bv::with_stream_work(call.stream, bv::attend_scratch, bv::enqueue_attend, &call);
}
