// The paged key-value cache: what its kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/bv.h"
#include "bv_device.cuh"

namespace bv {

// The longest sequence: a tile that begins in it ends below 2^31.
constexpr int kLongest = 0x7fffffff - 1023;

// Is it the length of a sequence whose row of the table has `width` pages?  Asked before anything is taken from it: -2^31 less one is positive.
__host__ __device__ __forceinline__ bool length_ok(int len, int width, int page) { return len >= 0 && len <= kLongest && len <= static_cast<long long>(width) * page; }
// How many tokens a sequence brings where n_new says m: 0 .. n.
__host__ __device__ __forceinline__ int brought(int m, int n) { return m < 0 ? 0 : m > n ? n : m; }
// The position that row t of the m newest tokens of a sequence is stored at; negative where there is none.
__host__ __device__ __forceinline__ int place_of(int len, int m, int t, int width, int page) { return t < m && length_ok(len, width, page) ? len - m + t : -1; }

// Division of numbers below 2^31 by one that the host knows: (n mul / 2^32 + n) / 2^shift.  (A division of unknown integers is some
// thirty instructions in a row, and the laying out of the work below is a chain of them.)  The method is that of Granlund and Montgomery, "Division by
// Invariant Integers using Multiplication" (1994), section 4: shift = ceil(log2 by), mul = floor(2^32 (2^shift - by) / by) + 1; sums stay below 2^32
// since n is below 2^31, which saves their correction step.
struct Divider {
    unsigned by, mul, shift;
    __device__ __forceinline__ int operator()(int n) const { return static_cast<int>((__umulhi(static_cast<unsigned>(n), mul) + static_cast<unsigned>(n)) >> shift); }
};
inline Divider divider(unsigned by) {
    unsigned shift = 0;
    while ((1ull << shift) < by) ++shift;
    return Divider{by, static_cast<unsigned>(((1ull << 32) * ((1ull << shift) - by)) / by + 1), shift};
}

// A sum that is not let grow beyond `most`; `more` may be a whole round of numbers, which 32 bits hold but not the sum with them.
__host__ __device__ __forceinline__ int sum_up_to(int most, int sum, int more) {
    const long long x = static_cast<long long>(sum) + more;
    return x < most ? static_cast<int>(x) : most;
}

// One call of bv_cache_attend.  Work is cut into units (sequence, key-value head, tile of query rows), a unit into tiles of
// keys; all tiles of all units, in that order, are one list that is cut into gridDim.x equal contiguous parts.  A CTA goes
// through its part; what a unit has in several CTAs is left in `part` and joined by those CTAs together.
// (Lengths lie on the device and change from call to call, so the list is laid out by the kernel itself: equal parts keep
// every SM at work whatever the lengths are, where a grid of (sequence, head, fixed pieces) waits for the longest sequence.  Units of
// different sequences are not equally long, so some CTAs have twelve ends of units where others have three: each counts as `extra` tiles in
// front of its own; so too where the list is cut although units are fewer than CTAs, by which 250 such calls took 0.96 of the time on average, 0.70 to 1.05.)
// With fewer units than CTAs the cuts of equal parts leave CTAs the end of one unit and the beginning of another, which they go through one
// after the other.  There a CTA has a part of one unit instead: a unit of t tiles is one CTA's up to `whole` tiles and else cut into
// ceil(t / T) equal parts, with the least T for which the CTAs suffice, if the longest part is at most `slack` tiles more than an equal one.
// (8 sequences of 2000 tokens, 8 heads on 2, D = 128: 13.4 us against 14.0 for the list; in 32 bits 15.4 against 16.3.  250 tokens: 9.3 against 9.6, 10.9
// against 11.9.)
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
    Divider by_group, by_page, by_span;
    float kf;                 // scale log2(e)
    int window, sinks;
    int rows;                 // query rows of a unit, at most (row = token * group + head of the group)
    int span;                 // keys of a tile; for pages that are several tiles those of a tile but the last of a page
    int box;                  // ... as they are copied: tokens of a page at a time (on the tensor cores)
    int per_page;             // tiles of a page, where a page is more than one (else 1)
    int extra;                // what a unit costs besides its tiles, in tiles: it counts as that many more when the list is cut
    int whole;                // units of up to so many tiles are one CTA's
    int slack;                // of a CTA for each unit's part; negative: the list is cut
    float* part;              // [gridDim.x][2] partial results of part_floats(rows, D)
    unsigned* counters;       // [gridDim.x] by the first CTA of a unit that several have: those that have come, then gone; zero between launches
    int* status;              // set if a bounded wait gave up
    unsigned wait_limit;
    int never_signal;
};

__host__ __device__ __forceinline__ size_t part_floats(int rows, int D) { return static_cast<size_t>(rows) * (D + 2); }

__device__ __forceinline__ int tile_of(const AttendArgs& a, int pos) {
    if (a.per_page == 1) return a.by_span(pos);
    const int page = a.by_page(pos);
    return page * a.per_page + a.by_span(pos - page * a.page);
}
__device__ __forceinline__ int tile_start(const AttendArgs& a, int tile) {
    if (a.per_page == 1) return tile * a.span;
    const int page = tile / a.per_page;
    return page * a.page + (tile - page * a.per_page) * a.span;
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
    s.bad = !length_ok(s.len, a.width, a.page);
    if (s.bad) s.len = 0;
    const int m = a.n_new ? brought(__ldg(a.n_new + b), a.n) : a.n;
    s.base = s.len - m;
    s.rows = m * a.group;
    return s;
}
// What a row with the sum 0 gets: 0 where it sees nothing (its position is below 0), else 0 / 0 as the formula has it (all its scores are -inf).
__device__ __forceinline__ float of_nothing(const AttendArgs& a, const Seq& s, int row) { return s.base + a.by_group(row) < 0 ? 0.f : NAN; }
// The lowest position that a token at `pos` sees through its window.
__device__ __forceinline__ int low_of(const AttendArgs& a, int pos) {
    if (a.window <= 0) return 0;
    const long long low = static_cast<long long>(pos) - a.window + 1;
    return low > 0 ? static_cast<int>(low) : 0;
}

// Does a token at `pos` see any of the positions x0 .. x1?
__device__ __forceinline__ bool sees_any(const AttendArgs& a, int pos, int x0, int x1) {
    if (x1 > pos) x1 = pos;
    return x0 <= x1 && (x1 >= low_of(a, pos) || x0 < a.sinks);
}
// The tiles of keys that query rows [r0, r1] of a sequence can see any of: `sink` tiles from the front, then `tiles` - `sink` from
// `first` on.  At least one: rows that see nothing are written too.
struct Span {
    int sink, first, tiles;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, const Seq& s, int r0, int r1) {
    const int p0 = s.base + a.by_group(r0), p1 = s.base + a.by_group(r1);
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
// What one key-value head of a sequence takes of the list, over its tiles of rows.
__device__ __forceinline__ long long head_cost(const AttendArgs& a, const Seq& s) {
    long long sum = 0;
    for (int r0 = 0; r0 < s.rows; r0 += a.rows) {
        const int r1 = (r0 + a.rows < s.rows ? r0 + a.rows : s.rows) - 1;
        sum += span_of(a, s, r0, r1).tiles + a.extra;
    }
    return sum;
}

// Tiles of rows of a sequence, of up to three where CTAs have parts of units (all of a head's go through the same tiles of keys there: they
// differ in the last ones at most).
__device__ __forceinline__ int row_tiles(const AttendArgs& a, const Seq& s) { return (s.rows > 0) + (s.rows > a.rows) + (s.rows > 2 * a.rows); }

// Where a CTA's part of the list begins, as found by all its threads together.
struct Share {
    bool parts;               // a CTA has a part of one unit, and what is counted in tiles below is counted in parts of units
    long long total;          // length of the list
    int ctas;                 // CTAs that take part: no more than the list is long
    long long begin, end;     // the CTA's part
    int b;                    // the sequence that it begins in
    long long off;            // ... and how much of that sequence comes before it
    long long per_head;       // what one head of it takes (`parts`: a unit of it)
};
struct ShareSmem {
    long long sums[32];
    long long off, per_head;
    int b;
};
// total * c / n, in 32 bits where that is enough
__device__ __forceinline__ long long part_of(long long total, int c, int n) {
    const unsigned long long x = static_cast<unsigned long long>(total) * static_cast<unsigned>(c);
    return x >> 32 ? static_cast<long long>(x / static_cast<unsigned>(n)) : static_cast<long long>(static_cast<unsigned>(x) / static_cast<unsigned>(n));
}
// (At most 352 threads.  It holds the CTA's first barriers: what threads have set up before is there for all behind it.)
__device__ __forceinline__ Share find_share(const AttendArgs& a, ShareSmem& sm, int threads) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int each = a.B <= threads ? 1 : (a.B + threads - 1) / threads;
    const int b0 = tid * each < a.B ? tid * each : a.B, b1 = b0 + each < a.B ? b0 + each : a.B;
    Share s;
    s.parts = false;
    const unsigned c = blockIdx.x;
    auto cut = [&](long long total) {
        s.total = total;
        s.ctas = total < gridDim.x ? static_cast<int>(total) : gridDim.x;
        s.begin = c < static_cast<unsigned>(s.ctas) ? part_of(total, c, s.ctas) : total;
        s.end = c < static_cast<unsigned>(s.ctas) ? part_of(total, c + 1, s.ctas) : total;
    };
    if (a.B <= 32) {
        // a lane a sequence, every warp for itself
        const Seq q = lane < a.B ? seq_of(a, lane) : Seq{0, 0, 0, false};
        if (a.slack >= 0) {
            // (what is too long for 32 bits is for the list)
            const unsigned units = a.Hkv * row_tiles(a, q), t = units > 0 ? span_of(a, q, 0, q.rows - 1).tiles : 0;
            const bool fits = __all_sync(0xffffffffu, t <= 1u << 18);
            const unsigned tiles = fits ? __reduce_add_sync(0xffffffffu, units * t) : 0u;
            unsigned T = (tiles + gridDim.x - 1) / gridDim.x;
            for (int x = 0; fits && x <= a.slack; ++x, ++T) {
                const unsigned parts = t <= static_cast<unsigned>(a.whole) ? 1u : (t + T - 1) / T, mine = units * parts;
                const unsigned all = __reduce_add_sync(0xffffffffu, mine);
                if (all > gridDim.x) continue;
                unsigned upto = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const unsigned y = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += y;
                }
                const unsigned here = __ballot_sync(0xffffffffu, upto - mine <= c && c < upto);
                s.parts = true;
                s.total = s.ctas = static_cast<int>(all);
                s.begin = c;
                s.end = c + (c < all);
                s.b = here ? __ffs(here) - 1 : 0;
                s.off = c - __shfl_sync(0xffffffffu, upto - mine, s.b);
                s.per_head = __shfl_sync(0xffffffffu, parts, s.b);
                __syncthreads();
                return s;
            }
        }
        const long long ph = head_cost(a, q), mine = a.Hkv * ph;
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        cut(__shfl_sync(0xffffffffu, upto, 31));
        const unsigned here = __ballot_sync(0xffffffffu, upto - mine <= s.begin && s.begin < upto);
        s.b = here ? __ffs(here) - 1 : 0;
        s.off = s.begin - __shfl_sync(0xffffffffu, upto - mine, s.b);
        s.per_head = __shfl_sync(0xffffffffu, ph, s.b);
        __syncthreads();
        return s;
    }
    long long mine = 0, per_head = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) mine += a.Hkv * (per_head = head_cost(a, seq_of(a, b)));
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sm.sums[warp] = upto;
    __syncthreads();
    long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 11; ++w) {
        const long long x = w < threads / 32 ? sm.sums[w] : 0;
        before += w < warp ? x : 0;
        total += x;
    }
    before += upto - mine;
    cut(total);
    if (s.begin < s.end && before <= s.begin && s.begin < before + mine) {
        int b = b0;
        if (each > 1) {
            for (;; ++b) {
                per_head = head_cost(a, seq_of(a, b));
                if (s.begin < before + a.Hkv * per_head) break;
                before += a.Hkv * per_head;
            }
        }
        sm.b = b;
        sm.off = s.begin - before;
        sm.per_head = per_head;
    }
    __syncthreads();
    s.b = sm.b;
    s.off = sm.off;
    s.per_head = sm.per_head;
    return s;
}

// A walk over a CTA's part, unit by unit (those that it has tiles of).
struct Walk {
    long long at, end;        // the list's place of the tile that comes next, the end of the part
    int b, h, r0;             // the unit
    Seq s;
    Span u;
    int i, upto;              // its tiles [i, upto) are the CTA's
    int first, parts;         // where each CTA has a part of one unit: the unit's first CTA and how many they are
    long long unit_at;        // the list's place of its tile 0
    bool more;
};
__device__ __forceinline__ void walk_unit(const AttendArgs& a, Walk& w) {
    const int r1 = (w.r0 + a.rows < w.s.rows ? w.r0 + a.rows : w.s.rows) - 1;
    w.u = span_of(a, w.s, w.r0, r1);
}
// (A cut through a unit of up to `whole` tiles gives it to the CTA that has the larger part, the first one of two halves.)
__device__ __forceinline__ void walk_cut(const AttendArgs& a, Walk& w) {
    w.more = w.at < w.end;
    w.unit_at = w.at - w.i;
    w.upto = w.u.tiles;
    if (w.end - w.at < w.u.tiles - w.i) {
        const int cut = w.i + static_cast<int>(w.end - w.at);
        if (w.u.tiles > a.whole) w.upto = cut;
        else if (2 * cut < w.u.tiles) w.more = false;
    }
}
__device__ __forceinline__ void walk_next(const AttendArgs& a, Walk& w) {
    w.at += w.upto - w.i + a.extra;
    if (w.at >= w.end) { w.more = false; return; }
    w.i = 0;
    const int b = w.b, r0 = w.r0;
    w.r0 += a.rows;
    if (w.r0 >= w.s.rows) {
        w.r0 = 0;
        if (++w.h >= a.Hkv) {
            w.h = 0;
            do w.s = seq_of(a, ++w.b); while (w.s.rows == 0);     // (the list goes on, so there is one)
        }
    }
    if (w.b != b || w.r0 != r0) walk_unit(a, w);                  // (the same rows of the next head see the same)
    walk_cut(a, w);
}
__device__ __forceinline__ Walk walk_begin(const AttendArgs& a, const Share& sh) {
    Walk w;
    w.end = sh.end;
    w.parts = 0;
    w.more = sh.begin < sh.end;
    if (!w.more) return w;
    w.b = sh.b;
    w.s = seq_of(a, w.b);
    if (sh.parts) {
        const unsigned off = static_cast<unsigned>(sh.off), parts = static_cast<unsigned>(sh.per_head), unit = off / parts, k = off - unit * parts;
        const int per_head = row_tiles(a, w.s);
        w.h = per_head == 1 ? unit : unit / per_head;
        w.r0 = (unit - w.h * per_head) * a.rows;
        w.u = span_of(a, w.s, 0, w.s.rows - 1);
        w.parts = parts;
        w.first = blockIdx.x - k;
        w.i = static_cast<unsigned>(w.u.tiles) * k / parts;
        w.upto = static_cast<unsigned>(w.u.tiles) * (k + 1) / parts;
        w.at = w.end;                          // (nothing comes after it)
        return w;
    }
    long long off;
    if ((sh.off | sh.per_head) >> 31) {
        w.h = static_cast<int>(sh.off / sh.per_head);
        off = sh.off % sh.per_head;
    } else {
        w.h = static_cast<unsigned>(sh.off) / static_cast<unsigned>(sh.per_head);
        off = static_cast<unsigned>(sh.off) % static_cast<unsigned>(sh.per_head);
    }
    for (w.r0 = 0;; w.r0 += a.rows) {
        walk_unit(a, w);
        if (off < w.u.tiles + a.extra) break;
        off -= w.u.tiles + a.extra;
    }
    w.i = off > a.extra ? static_cast<int>(off) - a.extra : 0;
    w.at = sh.begin + (off < a.extra ? a.extra - off : 0);
    if (w.i > 0 && w.u.tiles <= a.whole) {
        if (2 * w.i >= w.u.tiles) {            // the CTA's before
            w.upto = w.u.tiles;
            walk_next(a, w);
            return w;
        }
        w.at -= w.i;
        w.i = 0;
    }
    walk_cut(a, w);
    return w;
}
__device__ __forceinline__ int tile_at(const Span& u, int i) { return i < u.sink ? i : u.first + i - u.sink; }

// Keys of a tile, its first position.
__device__ __forceinline__ int tile_keys(const AttendArgs& a, int tile, int* start) {
    *start = tile_start(a, tile);
    if (a.per_page == 1) return a.span;
    const int left = a.page - tile % a.per_page * a.span;
    return left < a.span ? left : a.span;
}

// Is a row of a faulty unit lost: is its sequence's length none, or does it see a page that is none in the tiles that the CTA has of the unit?  (Looked up
// when the unit ends, so that it costs nothing where all pages are some; a row that sees none of the faulty ones is as if they were, since what
// a row does not see does not count.)
__device__ __forceinline__ bool loses_row(const AttendArgs& a, const Walk& w, int row) {
    if (w.s.bad) return true;
    const int pos = w.s.base + a.by_group(w.r0 + row);
#pragma unroll 1
    for (int i = w.i; i < w.upto; ++i) {
        int start;
        const int end = tile_keys(a, tile_at(w.u, i), &start) + start;
#pragma unroll 1
        for (int x = start; x < end && x <= pos;) {
            const int j = a.by_page(x), left = a.page - (x - j * a.page), upto = end - x < left ? end : x + left;       // positions x .. upto - 1 on page j
            if (sees_any(a, pos, x, upto - 1)) {
                const int page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
                if (page < 0 || page >= a.num_pages) return true;
            }
            x = upto;
        }
    }
    return false;
}

// The CTA that holds a place of the list.
__device__ __forceinline__ int holder_of(const Share& sh, long long place) {
    const unsigned long long x = static_cast<unsigned long long>(place + 1) * static_cast<unsigned>(sh.ctas) - 1;
    return (x | sh.total) >> 32 ? static_cast<int>(x / sh.total) : static_cast<unsigned>(x) / static_cast<unsigned>(sh.total);
}

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// ---- units that several CTAs hold tiles of -----------------------------------------------------------------------------

// Each CTA leaves what it has of such a unit (at most two: its first and its last) in `part`: per row the reference m and the sum l, then
// O.  At its end it reports, waits until the unit's other CTAs have (their parts of the list are equal, so they end at about the same time;
// the launch is cooperative, so they all run), and forms its share of the unit's elements from all parts:
//   out = sum_c 2^{m_c - M} O_c / sum_c 2^{m_c - M} l_c,   M = max_c m_c,
// in an order that does not depend on who came when.  (Joined by the last CTA alone, 148 parts of 36 rows took 2.5 ms, and the
// two or three parts that most units of a batch are cut into 0.3 ms in all: one SM has too few loads under way.)
struct Joint {
    int b, h, r0, count;      // the unit
    int first, last;          // the CTAs that have tiles of it
};
struct JointSmem {
    Joint unit[2];
    int n;                    // units left so far; zero at the start
    int ok[2];
};
// Is the unit one of several CTAs?  Then where this one's part goes, and a note of it (by one thread, whose `tid` is 0; visible to the CTA behind its next barrier).
__device__ __forceinline__ float* leave_unit(const AttendArgs& a, const Share& sh, const Walk& w, int count, JointSmem& js, int tid) {
    if (w.i == 0 && w.upto == w.u.tiles) return nullptr;
    const int c = blockIdx.x;
    const int first = w.parts > 0 ? w.first : w.i == 0 ? c : holder_of(sh, w.unit_at);
    const int last = w.parts > 0 ? w.first + w.parts - 1 : w.upto == w.u.tiles ? c : holder_of(sh, w.unit_at + w.u.tiles - 1);
    if (tid == 0) js.unit[atomicAdd(&js.n, 1)] = Joint{w.b, w.h, w.r0, count, first, last};
    return a.part + (2 * static_cast<size_t>(c) + (c == first)) * part_floats(a.rows, a.D);
}

template <typename T, int W>
__device__ __forceinline__ void join_share(const AttendArgs& a, const Joint& u, int tid, int threads) {
    const int parts = u.last - u.first + 1, k = blockIdx.x - u.first, per_row = a.D / W;
    const int all = u.count * per_row;
    const int e0 = static_cast<int>(static_cast<long long>(all) * k / parts), e1 = static_cast<int>(static_cast<long long>(all) * (k + 1) / parts);
    // few elements and many parts: several lanes share an element, each with some of the parts
    int lanes = 1;
    while (lanes < 32 && 2 * lanes * (e1 - e0) <= threads && lanes < parts) lanes *= 2;
    const int sub = tid & (lanes - 1);
    const size_t stride = part_floats(a.rows, a.D);
    const float* const base = a.part + 2 * static_cast<size_t>(u.first) * stride;      // part c lies at 2 c, but that of the first CTA at 2 c + 1
    for (int x = e0; x < e1; x += threads / lanes) {
        const int e = x + tid / lanes;
        const bool mine = e < e1;
        const int row = mine ? e / per_row : 0, d = mine ? (e - row * per_row) * W : 0;
        float M = -INFINITY, l = 0.f, o[W];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < W; ++i) o[i] = 0.f;
        // four parts at a time, all of their numbers under way together; what has been summed up is scaled where a larger m comes
        for (int c0 = sub; c0 < parts; c0 += 4 * lanes) {
            float m[4], pl[4], v[4][W];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int c = c0 + y * lanes;
                const bool there = c < parts;
                const float* p = base + (there ? (2 * c + (c == 0)) * stride : 0);
                m[y] = there ? __ldcg(p + row) : -INFINITY;
                pl[y] = there ? __ldcg(p + a.rows + row) : 0.f;
                const float* const at = p + 2 * a.rows + static_cast<size_t>(row) * a.D + d;
                if constexpr (W == 4) {
                    const float4 x4 = there ? __ldcg(reinterpret_cast<const float4*>(at)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    v[y][0] = x4.x; v[y][1] = x4.y; v[y][2] = x4.z; v[y][3] = x4.w;
                } else {
                    v[y][0] = there ? __ldcg(at) : 0.f;
                }
            }
            float top = M;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                nan |= m[y] != m[y];
                top = fmaxf(top, m[y]);
            }
            const float scale = M == -INFINITY ? 0.f : exp2f(M - top);
            l = M == -INFINITY ? l : l * scale;               // (a sum of nothing: zero; of a page that is none: NaN)
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] *= scale;
            M = top;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float f = m[y] == -INFINITY ? 0.f : exp2f(m[y] - M);
                l += m[y] == -INFINITY ? pl[y] : f * pl[y];
#pragma unroll
                for (int i = 0; i < W; ++i) o[i] += f * v[y][i];
            }
        }
        // the lanes' sums, on one m
        float top = M;
        for (int s = 1; s < lanes; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        if (M != -INFINITY) {
            const float scale = exp2f(M - top);
            l *= scale;
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] *= scale;
        }
        if (nan) l = NAN;
        for (int s = 1; s < lanes; s <<= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, s);
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] += __shfl_xor_sync(0xffffffffu, o[i], s);
        }
        if (mine && sub == 0) {
            const int r = u.r0 + row, t = a.by_group(r);
            T* dst = static_cast<T*>(a.out) + u.b * a.os[0] + t * a.os[1] + (u.h * a.group + r - t * a.group) * a.os[2] + d;
            const float none = l == 0.f ? of_nothing(a, seq_of(a, u.b), r) : 0.f, inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int i = 0; i < W; ++i) dst[i] = from_float<T>(l == 0.f ? none : o[i] * inv);
        }
    }
}
// The end of a CTA: all its threads, its parts written.
template <typename T>
__device__ __forceinline__ void join_units(const AttendArgs& a, JointSmem& js, int tid, int threads) {
    __syncthreads();
    const int n = js.n;
    if (n == 0) return;
    unsigned* counter = nullptr;
    unsigned parts = 0;
    if (tid < n) {
        counter = a.counters + js.unit[tid].first;
        parts = js.unit[tid].last - js.unit[tid].first + 1;
        // (`parts` come, as many go: back to zero with the last one)
        const unsigned limit = a.wait_limit ? a.wait_limit : 1u << 22;
        unsigned v;
        if (a.never_signal == 3 && static_cast<int>(blockIdx.x) == js.unit[tid].last) {
            // (a test: the last CTA of a unit comes when another has given up, or after as many polls as anybody makes)
            int gave_up = 0;
            for (unsigned i = 0; !gave_up && i <= 1u << 22; ++i) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(gave_up) : "l"(a.status) : "memory");
        }
        asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(v) : "l"(counter), "r"(2 * parts - 1) : "memory");
        ++v;
        for (unsigned i = 0; v < parts && i <= limit; ++i) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
        js.ok[tid] = v >= parts;
        if (v < parts) atomicExch(a.status, 1);
    }
    __syncthreads();
    for (int j = 0; j < n; ++j) {
        if (!js.ok[j]) continue;              // (the status says so: the outputs are not to be used)
        if (a.D % 4 == 0) join_share<T, 4>(a, js.unit[j], tid, threads);
        else join_share<T, 1>(a, js.unit[j], tid, threads);
    }
    __syncthreads();
    if (tid < n) atomicInc(counter, 2 * parts - 1);
}

// Lets a kernel have `bytes` of shared memory: asked once per kernel and device (a call takes 1 us of host time).
template <typename K>
cudaError_t allow_shared(K* kernel, int bytes, std::atomic<unsigned long long>& devices) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (devices.load(std::memory_order_acquire) >> (dev & 63) & 1)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) devices.fetch_or(1ull << (dev & 63), std::memory_order_release);
    return e;
}
// A cooperative launch of as many of `ctas` CTAs as can run at once (a process that is given a part of the GPU has fewer).
template <typename... P, typename... A>
cudaError_t launch_together(void (*kernel)(P...), int ctas, int threads, size_t smem, cudaStream_t stream, A... args) {
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeCooperative;
    at.val.cooperative = 1;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    for (;; ctas /= 2) {
        cfg.gridDim = dim3(ctas);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
        if (e != cudaErrorCooperativeLaunchTooLarge || ctas == 1) return e;
        cudaGetLastError();
    }
}

// The kernels for every shape (bv_attend_rows.cu): rows of a unit, keys of a tile; the most rows of a unit.
void attend_rows_plan(AttendArgs* a);
int attend_rows_most();
// The kernel on the tensor cores (bv_attend_tiles.cu), for calls that attend_tiles_takes; `taken` is false if no map of the pools could be had.
bool attend_tiles_takes(const AttendArgs& a);
void attend_tiles_plan(AttendArgs* a);
cudaError_t launch_attend_tiles(const AttendArgs& a, bool q_vec, bool out_vec, int ctas, cudaStream_t stream, bool* taken);
cudaError_t launch_attend_rows(const AttendArgs& a, int dtype, bool aligned, bool q_vec, int ctas, cudaStream_t stream);

}  // namespace bv
