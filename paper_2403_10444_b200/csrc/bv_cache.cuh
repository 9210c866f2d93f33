// The paged key-value cache: what its kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/bv.h"
#include "bv_device.cuh"

namespace bv {

// One call of bv_cache_attend.  Work is cut into units (sequence, key-value head, tile of query rows), a unit into tiles of
// keys; all tiles of all units, in that order, are one list that is cut into gridDim.x equal contiguous parts.  A CTA goes
// through its part; what a unit has in several CTAs is left in `part` and joined by the one that finishes last.
// (Lengths lie on the device and change from call to call, so the list is laid out by the kernel itself: equal parts keep
// every SM at work whatever the lengths are, where a grid of (sequence, head, fixed pieces) waits for the longest sequence.)
struct AttendArgs {
    const void* q;
    void* out;
    const void* k;
    const void* v;
    const int32_t* table;     // [B, width]
    const int32_t* lens;      // [B]
    const int32_t* n_new;     // [B] or null: n
    long long qs[3], os[3];   // elements between sequences, tokens, heads
    long long ks[3], vs[3];   // elements between pages, heads, tokens
    int B, n, Hkv, group, D, page, num_pages, width;
    float kf;                 // scale log2(e)
    int window, sinks;
    int rows;                 // query rows of a unit, at most (row = token * group + head of the group)
    int span;                 // keys of a tile; for pages that are several tiles those of a tile but the last of a page
    int per_page;             // tiles of a page, where a page is more than one (else 1)
    float* part;              // [gridDim.x][2] partial results of part_floats(rows, D)
    unsigned* counters;       // [gridDim.x] CTAs that have left their part of the unit that a CTA's last tiles belong to; zero between launches
    int* status;              // set if a bounded wait gave up
    unsigned wait_limit;
    int never_signal;
};

__host__ __device__ __forceinline__ size_t part_floats(int rows, int D) { return static_cast<size_t>(rows) * (D + 2); }

__device__ __forceinline__ int tile_of(const AttendArgs& a, int pos) {
    return a.per_page == 1 ? pos / a.span : pos / a.page * a.per_page + pos % a.page / a.span;
}
__device__ __forceinline__ int tile_start(const AttendArgs& a, int tile) {
    return a.per_page == 1 ? tile * a.span : tile / a.per_page * a.page + tile % a.per_page * a.span;
}

// A sequence of the batch: its length and the tokens it brings.
struct Seq {
    int len;          // 0 where the length is none
    int base;         // position of its first new token (negative where the block is longer than the sequence)
    int rows;         // query rows of a key-value head
    bool bad;         // the length is none: its rows become NaN
};
__device__ __forceinline__ Seq seq_of(const AttendArgs& a, int b) {
    Seq s;
    s.len = __ldg(a.lens + b);
    s.bad = s.len < 0 || s.len > static_cast<long long>(a.width) * a.page;
    if (s.bad) s.len = 0;
    int m = a.n_new ? __ldg(a.n_new + b) : a.n;
    m = m < 0 ? 0 : m > a.n ? a.n : m;
    s.base = s.len - m;
    s.rows = m * a.group;
    return s;
}
// The lowest position that a token at `pos` sees through its window.
__device__ __forceinline__ int low_of(const AttendArgs& a, int pos) {
    if (a.window <= 0) return 0;
    const long long low = static_cast<long long>(pos) - a.window + 1;
    return low > 0 ? static_cast<int>(low) : 0;
}

// The tiles of keys that query rows [r0, r1] of a sequence can see any of: `sink` tiles from the front, then `tiles` - `sink` from
// `first` on.  At least one: rows that see nothing are written too.
struct Span {
    int sink, first, tiles;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, const Seq& s, int r0, int r1) {
    const int p0 = s.base + r0 / a.group, p1 = s.base + r1 / a.group;
    Span u{0, 0, 1};
    if (p1 < 0) return u;
    const int low = low_of(a, p0);
    u.first = tile_of(a, low);
    const int sinks = a.sinks < low ? a.sinks : low;
    if (sinks > 0) {
        const int upto = tile_of(a, sinks - 1) + 1;
        u.sink = upto < u.first ? upto : u.first;
    }
    u.tiles = u.sink + tile_of(a, p1) - u.first + 1;
    return u;
}
// Tiles of one key-value head of a sequence, over its tiles of rows.
__device__ __forceinline__ long long head_tiles(const AttendArgs& a, const Seq& s) {
    long long sum = 0;
    for (int r0 = 0; r0 < s.rows; r0 += a.rows) {
        const int r1 = (r0 + a.rows < s.rows ? r0 + a.rows : s.rows) - 1;
        sum += span_of(a, s, r0, r1).tiles;
    }
    return sum;
}

// Where a CTA's part of the list begins, as found by all its threads together.
struct Share {
    long long total;          // tiles of the list
    int ctas;                 // CTAs that take part: no more than there are tiles, so that each has some
    long long begin, end;     // the CTA's part
    int b;                    // the sequence its first tile belongs to
    long long off;            // ... and how many of that sequence's tiles come before it
};
struct ShareSmem {
    long long sums[33];
    long long off;
    int b;
};
template <int THREADS>
__device__ __forceinline__ Share find_share(const AttendArgs& a, ShareSmem& sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int each = (a.B + THREADS - 1) / THREADS;
    const int b0 = tid * each < a.B ? tid * each : a.B, b1 = b0 + each < a.B ? b0 + each : a.B;
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += a.Hkv * head_tiles(a, seq_of(a, b));
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.sums[warp] = upto;
    if (tid == 0) { sm.b = a.B; sm.off = 0; }
    __syncthreads();
    long long before = 0, total = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += sm.sums[w];
        total += sm.sums[w];
    }
    before += upto - mine;
    Share s;
    s.total = total;
    s.ctas = total < gridDim.x ? static_cast<int>(total) : gridDim.x;
    const int c = blockIdx.x;
    s.begin = c < s.ctas ? total * c / s.ctas : total;
    s.end = c < s.ctas ? total * (c + 1) / s.ctas : total;
    if (s.begin < s.end && before <= s.begin && s.begin < before + mine) {
        long long at = before;
        for (int b = b0; b < b1; ++b) {
            const long long t = a.Hkv * head_tiles(a, seq_of(a, b));
            if (s.begin < at + t) { sm.b = b; sm.off = s.begin - at; break; }
            at += t;
        }
    }
    __syncthreads();
    s.b = sm.b;
    s.off = sm.off;
    return s;
}

// A walk over a CTA's part, unit by unit.
struct Walk {
    long long at, end;        // the list's tile that comes next, the end of the part
    int b, h, r0;             // the unit
    Seq s;
    Span u;
    int i, upto;              // its tiles [i, upto) are the CTA's
    long long unit_at;        // the list's number of its tile 0
    bool more;
};
__device__ __forceinline__ void walk_unit(const AttendArgs& a, Walk& w) {
    const int r1 = (w.r0 + a.rows < w.s.rows ? w.r0 + a.rows : w.s.rows) - 1;
    w.u = span_of(a, w.s, w.r0, r1);
}
__device__ __forceinline__ void walk_cut(Walk& w) {
    w.unit_at = w.at - w.i;
    const long long left = w.end - w.at;
    w.upto = left < w.u.tiles - w.i ? w.i + static_cast<int>(left) : w.u.tiles;
}
__device__ __forceinline__ Walk walk_begin(const AttendArgs& a, const Share& sh) {
    Walk w;
    w.at = sh.begin;
    w.end = sh.end;
    w.more = sh.begin < sh.end;
    if (!w.more) return w;
    w.b = sh.b;
    w.s = seq_of(a, w.b);
    const long long per_head = head_tiles(a, w.s);
    w.h = static_cast<int>(sh.off / per_head);
    long long off = sh.off % per_head;
    for (w.r0 = 0;; w.r0 += a.rows) {
        walk_unit(a, w);
        if (off < w.u.tiles) break;
        off -= w.u.tiles;
    }
    w.i = static_cast<int>(off);
    walk_cut(w);
    return w;
}
__device__ __forceinline__ void walk_next(const AttendArgs& a, Walk& w) {
    w.at += w.upto - w.i;
    if (w.at >= w.end) { w.more = false; return; }
    w.i = 0;
    w.r0 += a.rows;
    if (w.r0 >= w.s.rows) {
        w.r0 = 0;
        if (++w.h >= a.Hkv) {
            w.h = 0;
            do w.s = seq_of(a, ++w.b); while (w.s.rows == 0);     // (the list has tiles left, so there is one)
        }
    }
    walk_unit(a, w);
    walk_cut(w);
}
__device__ __forceinline__ int tile_at(const Span& u, int i) { return i < u.sink ? i : u.first + i - u.sink; }

// Which CTAs hold tiles of the unit, the first and the last of them.
__device__ __forceinline__ int holder_of(const Share& sh, long long tile) {
    return static_cast<int>(((tile + 1) * sh.ctas - 1) / sh.total);
}

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// The unit's rows from the parts that CTAs `first` to `last` left: out = sum_c 2^{m_c - M} O_c / sum_c 2^{m_c - M} l_c, in the order of the
// CTAs, so that the result does not depend on who finishes last.
template <typename T>
__device__ __forceinline__ void join_unit(const AttendArgs& a, const Walk& w, int first, int last, int tid, int threads) {
    const size_t stride = part_floats(a.rows, a.D);
    const int count = (w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0);
    for (int x = tid; x < count * a.D; x += threads) {
        const int row = x / a.D, d = x - row * a.D;
        float M = -INFINITY;
        bool nan = false;
        for (int c = first; c <= last; ++c) {
            const float m = __ldcg(a.part + (2 * static_cast<size_t>(c) + (c == first)) * stride + row);
            nan |= m != m;
            M = fmaxf(M, m);
        }
        float l = 0.f, o = 0.f;
        for (int c = first; c <= last; ++c) {
            const float* p = a.part + (2 * static_cast<size_t>(c) + (c == first)) * stride;
            const float m = __ldcg(p + row);
            if (m == -INFINITY) { l += __ldcg(p + a.rows + row); continue; }       // (nothing visible there: zero; or a page that is none: NaN)
            const float f = exp2f(m - M);
            l += f * __ldcg(p + a.rows + row);
            o += f * __ldcg(p + 2 * a.rows + static_cast<size_t>(row) * a.D + d);
        }
        const int r = w.r0 + row, t = r / a.group, g = r - t * a.group;
        T* dst = static_cast<T*>(a.out) + w.b * a.os[0] + t * a.os[1] + (w.h * a.group + g) * a.os[2] + d;
        *dst = from_float<T>(nan ? NAN : l == 0.f ? 0.f : o / l);
    }
}
// Who holds tiles of the unit: CTAs `first` to `last`; `split`: others than this one too.
struct Leave { int first, last; bool split; };
__device__ __forceinline__ Leave leave_of(const AttendArgs& a, const Share& sh, const Walk& w) {
    Leave l;
    l.split = w.i > 0 || w.upto < w.u.tiles;
    l.first = holder_of(sh, w.unit_at);
    l.last = holder_of(sh, w.unit_at + w.u.tiles - 1);
    return l;
}

// The kernel for every shape (bv_attend_rows.cu): query rows of a unit, keys of a tile.
int attend_rows_tile(int D, int rows);
int attend_rows_keys();
// The kernel on the tensor cores (bv_attend_tiles.cu), for calls that attend_tiles_takes; `taken` is false if no map of the pools could be had.
bool attend_tiles_takes(const AttendArgs& a);
int attend_tiles_rows(int rows);
void attend_tiles_plan(AttendArgs* a);
cudaError_t launch_attend_tiles(const AttendArgs& a, bool q_vec, int ctas, cudaStream_t stream, bool* taken);
cudaError_t launch_attend_rows(const AttendArgs& a, int dtype, bool aligned, int ctas, cudaStream_t stream);

}  // namespace bv
