// The pages of a key-value cache: taking, sharing and giving them back, and moving the ones in use together (contracts in
// include/bv.h).  A page is free where its count is 0; the lowest free pages are taken first, by the sequences in order.  So
// nothing but the counts says what is free, giving back is an atomic decrement in any order, and the outcome of every call is the
// same whatever the order in which its threads run.
//
// Taking needs the free pages' ranks: one cluster of up to 8 CTAs reads the counts in as many contiguous regions, the regions' sums
// cross through distributed shared memory, and a second look at the counts (the first 65536 of them kept in registers) hands out the pages.  (One CTA reads some 60 bytes a
// clock: 100000 counts would take it 4 us twice, a cluster has them in one round of loads per CTA.)
#include <cooperative_groups.h>

#include "bv_cache.cuh"
#include "bv_launch.h"

namespace cg = cooperative_groups;

namespace bv {
namespace {

constexpr int kThreads = 512, kEach = 16, kRound = kThreads * kEach;      // counts a thread, a CTA looks at in one go
constexpr int kMaxSequences = 8192;                                       // of bv_pages_extend: their needs lie in shared memory
constexpr int kMost = (1 << 22) - 2;                                      // pages of a cache, entries of a table's row

struct PagesArgs {
    int32_t* table;
    int32_t* lens;
    int32_t* refs;
    const int32_t* n_new;
    int B, n, page, num_pages, width;
};

__device__ __forceinline__ int pages_of(long long tokens, int page) { return static_cast<int>((tokens + page - 1) / page); }
__device__ __forceinline__ bool length_ok(const PagesArgs& a, int len) { return bv::length_ok(len, a.width, a.page); }

// The counts of pages first .. first + 15 of a region that ends at `end`, as bits: which are 0.
__device__ __forceinline__ unsigned zero_bits(const int32_t* refs, int first, int end, bool vec) {
    unsigned bits = 0;
    if (vec && first + kEach <= end) {
        int4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __ldcg(reinterpret_cast<const int4*>(refs + first) + i);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            bits |= (static_cast<unsigned>(x[i].x == 0) | static_cast<unsigned>(x[i].y == 0) << 1 | static_cast<unsigned>(x[i].z == 0) << 2 | static_cast<unsigned>(x[i].w == 0) << 3) << 4 * i;
    } else {
        for (int i = 0; i < kEach; ++i)
            if (first + i < end && __ldcg(refs + first + i) == 0) bits |= 1u << i;
    }
    return bits;
}
static_assert(kThreads / 32 == 16, "a half warp has the warps' sums");
struct ScanSmem {
    int2 warp[kThreads / 32];
};
// Two sums over the CTA at once, and what lies before this thread.
__device__ __forceinline__ int2 scan(ScanSmem& sm, int2 mine, int2* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto.x, o), y = __shfl_up_sync(0xffffffffu, upto.y, o);
        if (lane >= o) {
            upto.x += x;
            upto.y += y;
        }
    }
    __syncthreads();                          // (the last scan's readers)
    if (lane == 31) sm.warp[warp] = upto;
    __syncthreads();
    // (the warps' sums, by a lane each, in every warp)
    int2 sums = sm.warp[lane & 15];
#pragma unroll
    for (int o = 1; o < kThreads / 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, sums.x, o, 16), y = __shfl_up_sync(0xffffffffu, sums.y, o, 16);
        if ((lane & 15) >= o) {
            sums.x += x;
            sums.y += y;
        }
    }
    const int2 all = make_int2(__shfl_sync(0xffffffffu, sums.x, 15), __shfl_sync(0xffffffffu, sums.y, 15));
    int2 before = make_int2(__shfl_sync(0xffffffffu, sums.x, (warp - 1) & 15), __shfl_sync(0xffffffffu, sums.y, (warp - 1) & 15));
    if (warp == 0) before = make_int2(0, 0);
    *total = all;
    return make_int2(before.x + upto.x - mine.x, before.y + upto.y - mine.y);
}
__device__ __forceinline__ int scan(ScanSmem& sm, int mine, int* total) {
    int2 all;
    const int2 before = scan(sm, make_int2(mine, 0), &all);
    *total = all.x;
    return before.x;
}
// All CTAs of the cluster have come here; a number of each, added up: what lies before this CTA, and all.
__device__ __forceinline__ void come_together(cg::cluster_group& cluster, int ctas) {
    if (ctas > 1) cluster.sync(); else __syncthreads();
}
__device__ __forceinline__ int2 across(cg::cluster_group& cluster, int* mine, int rank, int ctas) {
    int x[8], before = 0, all = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) x[r] = r < ctas ? *cluster.map_shared_rank(mine, r) : 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        before += r < rank ? x[r] : 0;
        all += x[r];
    }
    return make_int2(before, all);
}

// A CTA's region of the counts: whole rounds of 16 but for the last.
__device__ __forceinline__ void region(int num_pages, int rank, int ctas, int* begin, int* end) {
    const int each = ((num_pages + ctas - 1) / ctas + kEach - 1) / kEach * kEach;
    const long long b = static_cast<long long>(each) * rank;
    *begin = b < num_pages ? static_cast<int>(b) : num_pages;
    *end = b + each < num_pages ? static_cast<int>(b + each) : num_pages;
}

// ---- extend ------------------------------------------------------------------------------------------------------------

struct ExtendSmem {
    ScanSmem scan;
    int free;                 // free pages of this CTA's region
    int upto[kMaxSequences];  // pages needed by the sequences up to and including this one, at most one more than there are
    int list[kRound];         // the free pages of a round, by rank
    int info[kMaxSequences];  // negative: refused whatever is free; else kReplace, kNeeds, and the first entry of its table row to be filled
};
enum : int { kReplace = 1, kNeeds = 2, kFirst = 4 };

// What a sequence asks for: the number of pages, and its `info`.
__device__ __forceinline__ int need_of(const PagesArgs& a, int b, int* info) {
    const int len = __ldcg(a.lens + b);
    const int m = a.n_new ? __ldg(a.n_new + b) : a.n;
    const long long grown = static_cast<long long>(len) + m;
    *info = -1;
    if (m < 0 || m > a.n || !length_ok(a, len) || grown > static_cast<long long>(a.width) * a.page || grown > kLongest) return 0;
    int first = pages_of(len, a.page), pages = pages_of(grown, a.page) - first, replace = 0;
    if (m > 0 && len % a.page != 0) {
        const int last = __ldcg(a.table + static_cast<long long>(b) * a.width + first - 1);
        if (last < 0 || last >= a.num_pages) return 0;
        if (__ldcg(a.refs + last) > 1) {      // shared and partly filled
            replace = kReplace;
            --first;
            ++pages;
        }
    }
    *info = first * kFirst + (pages > 0 ? kNeeds : 0) + replace;
    return min(pages, a.num_pages + 1);
}

__global__ void __launch_bounds__(kThreads, 1) extend_pages_kernel(const PagesArgs a, int32_t* out_new, int32_t* out_copies, const int vec) {
    extern __shared__ __align__(16) char raw[];
    ExtendSmem& sm = *reinterpret_cast<ExtendSmem*>(raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ctas = static_cast<int>(cluster.num_blocks()), tid = threadIdx.x;
    int begin, end;
    region(a.num_pages, rank, ctas, &begin, &end);

    // The free pages of the region and what the sequences need, in their order (every CTA for itself: the pages it finds may be anybody's).
    // The first round's loads, of counts and of sequences, are under way together; its counts are kept for the second look.
    const int p0 = begin + tid * kEach;
    const unsigned bits0 = p0 < end ? zero_bits(a.refs, p0, end, vec) : 0u;
    int info = -1, want = tid < a.B ? need_of(a, tid, &info) : 0, mine = __popc(bits0);
    for (int p = p0 + kRound; p < end; p += kRound) mine += __popc(zero_bits(a.refs, p, end, vec));
    static_assert(static_cast<long long>(kThreads) * (kMost + 1) <= 0x7fffffff, "a round's numbers stay within 32 bits");
    int2 all;
    int2 ahead = scan(sm.scan, make_int2(mine, want), &all);
    if (tid == 0) sm.free = all.x;
    int sum = 0;
    for (int b = tid, b0 = 0;;) {
        if (b < a.B) {
            sm.upto[b] = sum_up_to(a.num_pages + 1, sum, ahead.y + want);
            sm.info[b] = info;
        }
        sum = sum_up_to(a.num_pages + 1, sum, all.y);
        b0 += kThreads;
        b += kThreads;
        if (b0 >= a.B) break;
        want = b < a.B ? need_of(a, b, &info) : 0;
        ahead = scan(sm.scan, make_int2(0, want), &all);
    }
    come_together(cluster, ctas);             // everything that decides has been read, and nothing changed so far
    const int2 cut = across(cluster, &sm.free, rank, ctas);
    const int free = cut.y;
    // the region's free pages, by rank, to the sequences
    const int wanted = min(sum, free);
    int at = cut.x;
    for (int first = begin; first < end && at < wanted; first += kRound) {
        const int p = first + tid * kEach;
        unsigned bits = first == begin ? bits0 : p < end ? zero_bits(a.refs, p, end, vec) : 0u;
        int some;
        int f = scan(sm.scan, __popc(bits), &some);
        for (; bits && at + f < wanted; bits &= bits - 1, ++f) sm.list[f] = p + __ffs(bits) - 1;
        __syncthreads();
        // a thread a page (each thread with the free ones of its 16 took 13000 clocks for 256 sequences)
        const int n = some < wanted - at ? some : wanted - at;
        for (int x = tid; x < n; x += kThreads) {
            const int page = sm.list[x], rank_of = at + x;
            int lo = 0, hi = a.B - 1;         // the first sequence whose sum is above it
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (sm.upto[mid] > rank_of) hi = mid; else lo = mid + 1;
            }
            if (sm.upto[lo] > free) continue; // it is not served, nor is any after it
            const int slot = rank_of - (lo > 0 ? sm.upto[lo - 1] : 0), asked = sm.info[lo];
            int32_t* entry = a.table + static_cast<long long>(lo) * a.width + asked / kFirst + slot;
            if (slot == 0 && (asked & kReplace)) {
                out_copies[2 * lo] = *entry;
                out_copies[2 * lo + 1] = page;
            }
            *entry = page;
            a.refs[page] = 1;
        }
        at += some;
    }
    __threadfence();
    come_together(cluster, ctas);
    // lengths, what was served, and the counts of the pages that were replaced (only now: one that comes to 0 is free for the next call)
    for (int b = rank * kThreads + tid; b < a.B; b += ctas * kThreads) {
        const int asked = sm.info[b];
        const bool ok = asked >= 0 && (!(asked & kNeeds) || sm.upto[b] <= free);
        const int m = a.n_new ? __ldg(a.n_new + b) : a.n;
        if (ok && (asked & kReplace)) atomicSub(a.refs + __ldcg(out_copies + 2 * b), 1);
        else out_copies[2 * b] = out_copies[2 * b + 1] = -1;
        out_new[b] = ok ? m : -1;
        if (ok) a.lens[b] += m;
    }
}

// ---- truncate ----------------------------------------------------------------------------------------------------------

// One use of a page less.  (A count that is not positive is none of ours to lower: it stays.)
__device__ __forceinline__ void give_back(int32_t* refs, int num_pages, int page) {
    if (page < 0 || page >= num_pages) return;
    if (atomicSub(refs + page, 1) <= 0) atomicAdd(refs + page, 1);
}

// A CTA per sequence.
__global__ void __launch_bounds__(128) truncate_pages_kernel(const PagesArgs a, const int32_t* keep) {
    const int b = blockIdx.x;
    const int len = __ldcg(a.lens + b);
    if (!length_ok(a, len)) return;
    int m = len;
    if (a.n > 0) {
        m = a.n_new ? brought(__ldg(a.n_new + b), a.n) : a.n;
        m = m > len ? len : m;
    }
    int k = __ldg(keep + b);
    k = k < 0 ? 0 : k > m ? m : k;
    const int left = len - m + k;
    int32_t* row = a.table + static_cast<long long>(b) * a.width;
    for (int j = pages_of(left, a.page) + threadIdx.x; j < pages_of(len, a.page); j += 128) {
        give_back(a.refs, a.num_pages, row[j]);
        row[j] = -1;
    }
    __syncthreads();                          // (everybody has read the length)
    if (threadIdx.x == 0) a.lens[b] = left;
}

// ---- fork --------------------------------------------------------------------------------------------------------------

// A CTA per fork.  A fork whose target another one names, or that any one has as its source, is refused: those that are left change
// rows that nobody else reads or changes, so they need no order.
__global__ void __launch_bounds__(128) fork_pages_kernel(const PagesArgs a, const int32_t* src, const int32_t* dst, int forks, int32_t* out_ok) {
    const int f = blockIdx.x;
    const int s = __ldg(src + f), d = __ldg(dst + f);
    bool bad = s < 0 || s >= a.B || d < 0 || d >= a.B;
    for (int g = threadIdx.x; g < forks; g += 128) bad |= (g != f && __ldg(dst + g) == d) || __ldg(src + g) == d;
    if (!__syncthreads_or(bad)) {
        const int len = __ldcg(a.lens + s), old = __ldcg(a.lens + d);
        bad = !length_ok(a, len) || !length_ok(a, old);
        if (!bad) {
            const int32_t* from = a.table + static_cast<long long>(s) * a.width;
            int32_t* to = a.table + static_cast<long long>(d) * a.width;
            const int take = pages_of(len, a.page), give = pages_of(old, a.page);
            for (int j = threadIdx.x; j < a.width; j += 128) {
                const int had = to[j];
                const int page = j < take ? from[j] : -1;
                if (page >= 0 && page < a.num_pages) atomicAdd(a.refs + page, 1);
                if (j < give) give_back(a.refs, a.num_pages, had);
                to[j] = page;
            }
            __syncthreads();
            if (threadIdx.x == 0) a.lens[d] = len;
        }
    } else {
        bad = true;
    }
    if (threadIdx.x == 0) out_ok[f] = bad ? -1 : 0;
}

// ---- compact -----------------------------------------------------------------------------------------------------------

struct CompactSmem {
    ScanSmem scan;
    int used, holes, sources;
};
// The n pages in use are to lie at 0 .. n-1: those beyond move, in order, to the free pages before, in order.  Writes the moves, moves the
// counts, and leaves in `moved` which move takes a page that moves (nothing for the others), and n at moved[num_pages].
__global__ void __launch_bounds__(kThreads, 1) compact_pages_kernel(const PagesArgs a, int32_t* moves, int32_t* out_count, int32_t* moved, const int vec) {
    __shared__ CompactSmem sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = static_cast<int>(cluster.block_rank()), ctas = static_cast<int>(cluster.num_blocks()), tid = threadIdx.x;
    int begin, end;
    region(a.num_pages, rank, ctas, &begin, &end);
    // (the first round's counts are kept)
    const int p0 = begin + tid * kEach;
    const unsigned zero0 = p0 < end ? zero_bits(a.refs, p0, end, vec) : 0u;
    auto zeros = [&](int p) { return p == p0 ? zero0 : zero_bits(a.refs, p, end, vec); };
    int mine = 0, some;
    for (int p = p0; p < end; p += kRound) mine += min(end - p, kEach) - __popc(zeros(p));
    scan(sm.scan, mine, &some);
    if (tid == 0) sm.used = some;
    come_together(cluster, ctas);
    const int live = across(cluster, &sm.used, rank, ctas).y;
    // free pages before `live`, pages in use from there on, as bits
    auto look = [&](int p, unsigned* holes, unsigned* sources) {
        *holes = *sources = 0;
        if (p >= end) return;
        const unsigned zero = zeros(p), there = end - p >= kEach ? 0xffffu : (1u << (end - p)) - 1;
        const unsigned before = live - p >= kEach ? 0xffffu : live <= p ? 0u : (1u << (live - p)) - 1;
        *holes = zero & before;
        *sources = ~zero & there & ~before;
    };
    int2 found{0, 0}, all;
    for (int p = p0; p < end; p += kRound) {
        unsigned hb, sb;
        look(p, &hb, &sb);
        found.x += __popc(hb);
        found.y += __popc(sb);
    }
    scan(sm.scan, found, &all);
    if (tid == 0) {
        sm.holes = all.x;
        sm.sources = all.y;
    }
    come_together(cluster, ctas);
    const int2 holes = across(cluster, &sm.holes, rank, ctas), sources = across(cluster, &sm.sources, rank, ctas);
    int hole_at = holes.x, source_at = sources.x;
    const int count = sources.y;
    for (int first = begin; first < end; first += kRound) {
        const int p = first + tid * kEach;
        unsigned hb, sb;
        look(p, &hb, &sb);
        const int2 ahead = scan(sm.scan, make_int2(__popc(hb), __popc(sb)), &all);
        int f = hole_at + ahead.x, g = source_at + ahead.y;
        hole_at += all.x;
        source_at += all.y;
        for (; hb; hb &= hb - 1) moves[2 * f++ + 1] = p + __ffs(hb) - 1;
        for (; sb; sb &= sb - 1) moves[2 * g++] = p + __ffs(sb) - 1;
    }
    __threadfence();
    come_together(cluster, ctas);
    for (int i = rank * kThreads + tid; i < a.num_pages / 2; i += ctas * kThreads) {
        if (i >= count) {
            moves[2 * i] = moves[2 * i + 1] = -1;
            continue;
        }
        const int from = __ldcg(moves + 2 * i), into = __ldcg(moves + 2 * i + 1);
        a.refs[into] = __ldcg(a.refs + from);
        a.refs[from] = 0;
        moved[from] = i;
    }
    if (rank == 0 && tid == 0) {
        *out_count = count;
        moved[a.num_pages] = live;
    }
    come_together(cluster, ctas);             // (the others' shared memory is read above)
}
// Gives the pages of all tables their new numbers.
__global__ void __launch_bounds__(256) rename_pages_kernel(const PagesArgs a, const int32_t* moves, const int32_t* count, const int32_t* moved) {
    const int live = __ldg(moved + a.num_pages), n = __ldg(count);
    const int len = __ldg(a.lens + blockIdx.y);
    if (!length_ok(a, len)) return;
    int32_t* row = a.table + static_cast<long long>(blockIdx.y) * a.width;
    for (int j = blockIdx.x * 256 + threadIdx.x; j < pages_of(len, a.page); j += gridDim.x * 256) {
        const int page = row[j];
        if (page < live || page >= a.num_pages) continue;
        // (a move that is this page's says so itself: `moved` holds anything for a page that the table names though its count is 0)
        const int i = __ldg(moved + page);
        if (i < 0 || i >= n) continue;
        const int from = __ldg(moves + 2 * i), into = __ldg(moves + 2 * i + 1);
        if (from == page) row[j] = into;
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------

// One cluster, of as many CTAs as have a round of counts to look at.
template <typename... P, typename... A>
cudaError_t one_cluster(void (*kernel)(P...), int num_pages, size_t smem, cudaStream_t stream, A... args) {
    int ctas = 1;
    while (ctas < 8 && num_pages > ctas * kRound) ctas *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = ctas;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int check(const bv_cache* c, PagesArgs* a) {
    if (!c || !c->table || !c->lens || !c->refs || !on(c->table, 4) || !on(c->lens, 4) || !on(c->refs, 4)) return BV_ERR_INVALID_ARG;
    if (c->B < 0 || c->width < 1 || c->num_pages < 1 || c->page_size < 1) return BV_ERR_INVALID_ARG;
    if (c->num_pages > kMost || c->width > kMost || c->B > 0xffff) return BV_ERR_UNSUPPORTED;
    *a = PagesArgs{c->table, c->lens, c->refs, nullptr, c->B, 0, c->page_size, c->num_pages, c->width};
    note_launches(0);
    return BV_OK;
}
int done(cudaError_t e, int launches) {
    if (e != cudaSuccess) return note_cuda_error(e);
    note_launches(launches);
    return BV_OK;
}

struct CompactCall {
    PagesArgs a;
    int32_t* moves;
    int32_t* count;
    cudaStream_t stream;
};
size_t compact_scratch(int, const void* ctx) { return (static_cast<const CompactCall*>(ctx)->a.num_pages + 1) * sizeof(int32_t); }
int enqueue_compact(const StreamWork& work, void* ctx) {
    const CompactCall& c = *static_cast<const CompactCall*>(ctx);
    int32_t* moved = reinterpret_cast<int32_t*>(work.scratch);
    cudaError_t e = one_cluster(compact_pages_kernel, c.a.num_pages, 0, c.stream, c.a, c.moves, c.count, moved, static_cast<int>(on(c.a.refs, 16)));
    if (e == cudaSuccess && c.a.B > 0) {
        const int blocks = (c.a.width + 1023) / 1024;
        rename_pages_kernel<<<dim3(blocks < 64 ? blocks : 64, c.a.B), 256, 0, c.stream>>>(c.a, c.moves, c.count, moved);
        e = cudaGetLastError();
    }
    return done(e, c.a.B > 0 ? 2 : 1);
}

}  // namespace
}  // namespace bv

extern "C" int bv_pages_extend(const bv_cache* c, const int32_t* n_new, int n, int32_t* out_new, int32_t* out_copies, void* stream) {
    bv::PagesArgs a;
    const int rc = bv::check(c, &a);
    if (rc != BV_OK) return rc;
    if (n < 1 || !out_new || !out_copies || !bv::on(out_new, 4) || !bv::on(out_copies, 4) || (n_new && !bv::on(n_new, 4))) return BV_ERR_INVALID_ARG;
    if (a.B > bv::kMaxSequences) return BV_ERR_UNSUPPORTED;
    if (a.B == 0) return BV_OK;
    a.n_new = n_new;
    a.n = n;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = bv::allow_shared(bv::extend_pages_kernel, static_cast<int>(sizeof(bv::ExtendSmem)), asked);
    if (e == cudaSuccess)
        e = bv::one_cluster(bv::extend_pages_kernel, a.num_pages, sizeof(bv::ExtendSmem), static_cast<cudaStream_t>(stream), a, out_new, out_copies,
                            static_cast<int>(bv::on(a.refs, 16)));
    return bv::done(e, 1);
}

extern "C" int bv_pages_truncate(const bv_cache* c, const int32_t* keep, const int32_t* n_new, int n, void* stream) {
    bv::PagesArgs a;
    const int rc = bv::check(c, &a);
    if (rc != BV_OK) return rc;
    if (n < 0 || !keep || !bv::on(keep, 4) || (n_new && !bv::on(n_new, 4))) return BV_ERR_INVALID_ARG;
    if (a.B == 0) return BV_OK;
    a.n_new = n_new;
    a.n = n;
    bv::truncate_pages_kernel<<<a.B, 128, 0, static_cast<cudaStream_t>(stream)>>>(a, keep);
    return bv::done(cudaGetLastError(), 1);
}

extern "C" int bv_pages_fork(const bv_cache* c, const int32_t* src, const int32_t* dst, int forks, int32_t* out_ok, void* stream) {
    bv::PagesArgs a;
    const int rc = bv::check(c, &a);
    if (rc != BV_OK) return rc;
    if (forks < 0 || !src || !dst || !out_ok || !bv::on(src, 4) || !bv::on(dst, 4) || !bv::on(out_ok, 4)) return BV_ERR_INVALID_ARG;
    if (forks == 0) return BV_OK;
    bv::fork_pages_kernel<<<forks, 128, 0, static_cast<cudaStream_t>(stream)>>>(a, src, dst, forks, out_ok);
    return bv::done(cudaGetLastError(), 1);
}

extern "C" int bv_pages_compact(const bv_cache* c, int32_t* out_moves, int32_t* out_count, void* stream) {
    bv::CompactCall call{};
    const int rc = bv::check(c, &call.a);
    if (rc != BV_OK) return rc;
    if (!out_moves || !out_count || !bv::on(out_moves, 4) || !bv::on(out_count, 4)) return BV_ERR_INVALID_ARG;
    call.moves = out_moves;
    call.count = out_count;
    call.stream = static_cast<cudaStream_t>(stream);
    return bv::with_stream_work(call.stream, bv::compact_scratch, bv::enqueue_compact, &call);
}
