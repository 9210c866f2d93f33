// Attention over a paged cache, for every shape, type, alignment and stride: bv_cache_attend where bv_attend_tiles.cu does not take
// the call (32-bit caches above all: their products are 32-bit FMAs, since a tensor core would round the inputs to 10 bits of mantissa).
//
// One pass over the keys with a running reference m and sum l per row:  p = 2^{k q.k - m},  l += p,  O += p v,  and where a score
// exceeds m by more than 8 (first of all where m is still -inf)  m <- that score, l and O scaled by 2^{m_old - m}.  A reference
// that lags by up to 8 costs nothing in 32 bits (terms of up to 256 instead of 1) and saves nearly all of the scaling.
// A weight of zero takes no value, whatever that is.
//
// (18 sequences of up to 8563 tokens, blocks of 6 tokens, 14 heads on 2, D = 128: 186 us, 3.8 times the FMAs' floor; single tokens, 32 heads on 8, 16
// sequences of up to 4096: 66 us, 4.7 TB/s, 64 of up to 8192: 387 us, 5.9 TB/s.)
// Two kernels.  Few query rows (a token of a group of up to 4 heads): the call is a matter of reading the cache.  Eight lanes share
// a key, each with every 8th group of four of its D elements, of 4 query rows at a time, in registers; a warp has 4 keys of each tile
// of 32, and every thread copies what it will read itself into a ring of cells of its own, several tiles ahead, so no thread
// waits for another until the unit ends.  More rows: reading shared memory and the FMAs
// bound (a 16-byte read takes a warp four clocks, wherever it goes).  A tile of 64 keys lies there, and both products are tiled in
// registers: S by 4 rows x 8 keys a thread with a fourth of D each, O by 8 rows x 8 columns with every 4th or 8th key (2 x 4 and 8 x 4 with no
// such splits: 206 us against 182, when they were built, for 18 sequences of up to 8563 keys, 42 rows on 2 heads, D = 128).
#include "bv_cache.cuh"
#include "bv_launch.h"

namespace bv {
namespace {

constexpr int kThreads = 256, kWarps = 8;
constexpr float kLag = 8.f;

__device__ __forceinline__ void widen(const float* p, float (&x)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void widen(const __nv_bfloat16* p, float (&x)[4]) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void copy4(float* to, const float* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(__nv_bfloat16* to, const __nv_bfloat16* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

// What the unit's rows see: positions p0 to p1 are theirs, low0 and low1 the first positions of the first and the last row's windows.
struct Sight {
    int count, p0, p1, low0, low1;
};
__device__ __forceinline__ Sight sight_of(const AttendArgs& a, const Walk& w) {
    Sight s;
    s.count = w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0;
    s.p0 = w.s.base + a.by_group(w.r0);
    s.p1 = w.s.base + a.by_group(w.r0 + s.count - 1);
    s.low0 = low_of(a, s.p0);
    s.low1 = low_of(a, s.p1);
    return s;
}
// Where a key's row lies in the pools: false if nobody sees it, `bad` if its page is none.
__device__ __forceinline__ bool key_row(const AttendArgs& a, const Walk& w, const Sight& s, int p, long long* k, long long* v, bool* bad) {
    if (p > s.p1 || !(p >= s.low0 || p < a.sinks)) return false;
    const int j = a.by_page(p), page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
    if (page < 0 || page >= a.num_pages) {
        *bad = true;
        return false;
    }
    const int row = p - j * a.page;
    *k = page * a.ks[0] + w.h * a.ks[1] + row * a.ks[2];
    *v = page * a.vs[0] + w.h * a.vs[1] + row * a.vs[2];
    return true;
}
__device__ __forceinline__ bool whole_tile(const AttendArgs& a, const Sight& s, int start, int keys) {
    return start + keys - 1 <= s.p0 && (start >= s.low1 || start + keys <= a.sinks);
}
// (A function that is called, for a fault's sake alone, leaves the loops their registers: 16 sequences of single tokens, D = 256, 58.9 us against 74.5 with
// it inlined, 18 sequences of 42 rows 186 against 189.)
__device__ __noinline__ bool row_lost(const AttendArgs a, const Walk w, int row) { return loses_row(a, w, row); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float factor_of(float m, float M) { return m == -INFINITY ? 0.f : ex2(m - M); }

// Elements d .. d + 3 of the unit's row `row` from their sums, to `out` or to the CTA's part of the unit.
template <typename T>
__device__ __forceinline__ void put(const AttendArgs& a, const Walk& w, float* part, int row, int d, float m, float l, const float (&o)[4]) {
    if (part) {
        float* const to = part + 2 * a.rows + row * a.D + d;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < a.D) to[e] = o[e];
        if (d == 0) {
            part[row] = m;
            part[a.rows + row] = l;
        }
    } else {
        const int r = w.r0 + row, t = a.by_group(r);
        T* const to = static_cast<T*>(a.out) + w.b * a.os[0] + t * a.os[1] + (w.h * a.group + r - t * a.group) * a.os[2] + d;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < a.D) to[e] = from_float<T>(l == 0.f ? of_nothing(a, w.s, r) : o[e] / l);
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------------

constexpr int kFewKeys = 32;

template <typename T, int NJ, int R>
struct FewSmem {
    static constexpr int kDepth = NJ <= 4 ? 5 : 3;                 // tiles ahead
    T ring[kDepth][2 * NJ][kThreads][4];
    float part[kWarps][R][NJ * 32 + 2];
    ShareSmem share;
    JointSmem joint;
};

template <typename T, int NJ, int R>
__global__ void __launch_bounds__(kThreads, 1) attend_few_kernel(const AttendArgs a, const int aligned, const int q_vec) {
    extern __shared__ __align__(16) char raw[];
    using Smem = FewSmem<T, NJ, R>;
    Smem& sm = *reinterpret_cast<Smem*>(raw);
    constexpr int kRow = NJ * 32, kDepth = Smem::kDepth;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int group8 = lane >> 3, l8 = lane & 7, mine = warp * 4 + group8;             // its key of a tile
    if (a.D < kRow) {                          // (a thread's cells beyond D are never copied to: they stay zero)
        for (int x = 0; x < kDepth * 2 * NJ; ++x)
            for (int e = 0; e < 4; ++e) sm.ring[x / (2 * NJ)][x % (2 * NJ)][tid][e] = from_float<T>(0.f);
    }
    if (tid == 0) sm.joint.n = 0;
    const Share sh = find_share(a, sm.share, kThreads);
    Walk w = walk_begin(a, sh);
#pragma unroll 1
    while (w.more) {
        const Sight v = sight_of(a, w);
        const int nt = w.upto - w.i;
        bool bad = w.s.bad;
        // the page of the key that is fetched next, asked for a tile before that
        int page = 0, row = 0;
        bool seen = false;
        auto find = [&](int i) {
            const int p = i < nt ? tile_at(w.u, w.i + i) * kFewKeys + mine : 0, j = a.by_page(p);
            seen = i < nt && p <= v.p1 && (p >= v.low0 || p < a.sinks);
            row = p - j * a.page;
            if (seen) page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
        };
        auto fetch = [&](int i) {
            const bool there = seen && page >= 0 && page < a.num_pages;
            bad |= seen && !there;
            if (there) {
                T(*cell)[kThreads][4] = sm.ring[i % kDepth];
                const T* k = static_cast<const T*>(a.k) + page * a.ks[0] + w.h * a.ks[1] + row * a.ks[2] + l8 * 4;
                const T* vv = static_cast<const T*>(a.v) + page * a.vs[0] + w.h * a.vs[1] + row * a.vs[2] + l8 * 4;
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    if (aligned) {
                        if (j * 32 + l8 * 4 < a.D) {
                            copy4(cell[2 * j][tid], k + j * 32);
                            copy4(cell[2 * j + 1][tid], vv + j * 32);
                        }
                    } else {
                        for (int e = 0; e < 4; ++e) {
                            if (j * 32 + l8 * 4 + e < a.D) {
                                cell[2 * j][tid][e] = k[j * 32 + e];
                                cell[2 * j + 1][tid][e] = vv[j * 32 + e];
                            }
                        }
                    }
                }
            }
            cp_async_commit();
        };
        {
            // (the first tiles' pages are asked for all at once)
            int pages[kDepth - 1];
            unsigned sees = 0;
#pragma unroll
            for (int i = 0; i < kDepth - 1; ++i) {
                find(i);
                pages[i] = page;
                sees |= static_cast<unsigned>(seen) << i;
            }
#pragma unroll 1
            for (int i = 0; i < kDepth - 1; ++i) {
                const int p = i < nt ? tile_at(w.u, w.i + i) * kFewKeys + mine : 0;
                row = p - a.by_page(p) * a.page;
                seen = sees >> i & 1;
                page = pages[0];
#pragma unroll
                for (int x = 0; x + 1 < kDepth - 1; ++x) pages[x] = pages[x + 1];
                fetch(i);
            }
            find(kDepth - 1);
        }
        float q[R][NJ * 4];
        int pos[R], low[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool valid = r < v.count;
            const int row = w.r0 + r, t = valid ? a.by_group(row) : 0;
            pos[r] = valid ? w.s.base + t : -1;
            low[r] = valid ? low_of(a, pos[r]) : 0;
            const T* src = static_cast<const T*>(a.q) + w.b * a.qs[0] + t * a.qs[1] + (w.h * a.group + (valid ? row - t * a.group : 0)) * a.qs[2] + l8 * 4;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                if (valid && j * 32 + l8 * 4 < a.D) {
                    if (q_vec) {
                        widen(src + j * 32, x);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j * 32 + l8 * 4 + e < a.D) x[e] = to_float(src[j * 32 + e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) q[r][j * 4 + e] = x[e] * a.kf;
            }
        }
        float m[R], l[R], acc[R][NJ * 4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int x = 0; x < NJ * 4; ++x) acc[r][x] = 0.f;
        }
#pragma unroll 1
        for (int i = 0; i < nt; ++i) {
            fetch(i + kDepth - 1);
            find(i + kDepth);
            cp_async_wait<kDepth - 1>();
            T(*cell)[kThreads][4] = sm.ring[i % kDepth];
            float s[R];
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float x[4];
                widen(cell[2 * j][tid], x);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r] = fmaf(q[r][j * 4 + e], x[e], s[r]);
            }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1)
#pragma unroll
                for (int r = 0; r < R; ++r) s[r] += __shfl_xor_sync(0xffffffffu, s[r], o);
            const int p = tile_at(w.u, w.i + i) * kFewKeys + mine;
            bool some[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                some[r] = p <= pos[r] && (p >= low[r] || p < a.sinks) && s[r] != -INFINITY;
                if (some[r] && s[r] > m[r] + kLag) {
                    const float f = ex2(m[r] - s[r]);
                    m[r] = s[r];
                    l[r] *= f;
#pragma unroll
                    for (int x = 0; x < NJ * 4; ++x) acc[r][x] *= f;
                }
                s[r] = some[r] ? ex2(s[r] - m[r]) : 0.f;
                l[r] += s[r];
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float x[4];
                widen(cell[2 * j + 1][tid], x);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (some[r]) acc[r][j * 4 + e] = fmaf(s[r], x[e], acc[r][j * 4 + e]);
            }
        }
        // a warp's keys, then the warps'
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int o = 8; o <= 16; o <<= 1) {
                const float om = __shfl_xor_sync(0xffffffffu, m[r], o), ol = __shfl_xor_sync(0xffffffffu, l[r], o);
                const float M = fmaxf(m[r], om), f = factor_of(m[r], M), of = factor_of(om, M);
                l[r] = l[r] * f + ol * of;
                m[r] = M;
#pragma unroll
                for (int x = 0; x < NJ * 4; ++x) acc[r][x] = acc[r][x] * f + __shfl_xor_sync(0xffffffffu, acc[r][x], o) * of;
            }
            if (group8 == 0) {
                float* const to = sm.part[warp][r];
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) to[j * 32 + l8 * 4 + e] = acc[r][j * 4 + e];
                if (l8 == 0) {
                    to[kRow] = m[r];
                    to[kRow + 1] = l[r];
                }
            }
        }
        bad = __syncthreads_or(bad);
        float* const part = leave_unit(a, sh, w, v.count, sm.joint, tid);
        static_assert(R * NJ * 8 <= kThreads, "a thread for every four elements");
        const int at = tid / (NJ * 8), d = tid % (NJ * 8) * 4;
        if (at < v.count && at < R && d < a.D) {
            float M = -INFINITY, sl = 0.f, so[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < kWarps; ++s) M = fmaxf(M, sm.part[s][at][kRow]);
#pragma unroll
            for (int s = 0; s < kWarps; ++s) {
                const float f = factor_of(sm.part[s][at][kRow], M);
                sl += sm.part[s][at][kRow + 1] * f;
#pragma unroll
                for (int e = 0; e < 4; ++e) so[e] += sm.part[s][at][d + e] * f;
            }
            put<T>(a, w, part, at, d, M, bad && row_lost(a, w, at) ? NAN : sl, so);
        }
        cp_async_wait<0>();
        __syncthreads();
        walk_next(a, w);
    }
    join_units<T>(a, sm.joint, tid, kThreads);
}

// ---- more rows ---------------------------------------------------------------------------------------------------------

template <int NJ>
struct ManyShape {
    static constexpr int kRows = 32, kKeys = NJ <= 4 ? 64 : 32, kRow = NJ * 32;
    static constexpr int kPitch = kRow + 16;                           // of a key: two keys' groups of four quads lie in different banks
    static constexpr int kVecs = NJ <= 2 ? 16 : NJ <= 4 ? 32 : 64;     // groups of four of a row, to a power of two
    static constexpr int kLanes = kVecs / 2;                           // threads that share a row of O, two groups each
};
template <int NJ>
struct ManySmem {
    using Sh = ManyShape<NJ>;
    float kv[2 * Sh::kKeys * (Sh::kPitch + Sh::kRow)];                 // two tiles of keys, two of values; at the end of a unit the splits of O
    float q[Sh::kRows][Sh::kRow + 4];
    float p[Sh::kKeys][Sh::kRows + 4];
    float m[Sh::kRows], l[4][Sh::kRows], factor[Sh::kRows], top[4][Sh::kRows];     // sums and maxima by the parts of the keys
    long long row[3][2][Sh::kKeys];            // where the keys' rows lie, of tiles i .. i + 2 (negative: nowhere)
    ShareSmem share;
    JointSmem joint;
};

// PARTS: 32 / PARTS rows at most, whose keys are shared out to as many warps (8 rows of all keys would leave six of eight warps idle in either product:
// 76.8 us against 59.8 for 16 sequences of up to 4096 tokens, 4 key-value heads, 8 rows, D = 128; 16 rows 80.2 against 72.5).
template <typename T, int NJ, int PARTS>
__global__ void __launch_bounds__(kThreads, 1) attend_many_kernel(const AttendArgs a, const int aligned, const int q_vec) {
    extern __shared__ __align__(16) char raw[];
    using Sh = ManyShape<NJ>;
    ManySmem<NJ>& sm = *reinterpret_cast<ManySmem<NJ>*>(raw);
    constexpr int KT = Sh::kKeys, kI = KT / 8 / PARTS, kBlocks = 8 / PARTS, kGroups = 4 / PARTS, kHeld = 32 / PARTS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // S: a warp has 4 rows and its part of the keys, a thread keys 8 (PARTS i + part) + kg and every fourth group of four of D, from `dq` on; added
    // up, row `mine`.
    // O: rows of `rows8`, columns of `col`, every `kSplit`-th key
    const int dq = lane & 3, kg = lane >> 2, mine = warp % kBlocks * 4 + dq, part_of_keys = warp / kBlocks;
    constexpr int kSplit = 8 / kGroups * (32 / Sh::kLanes);
    float* const keys = sm.kv;
    float* const vals = sm.kv + 2 * KT * Sh::kPitch;
    const int rows8 = warp % kGroups * 8, col = lane % Sh::kLanes, split = warp / kGroups + 8 / kGroups * (lane / Sh::kLanes);
    const int quads = (a.D + 3) / 4;

    if (a.D % 4 != 0)                          // (columns D to the next multiple of four stay zero)
        for (int x = tid; x < 2 * KT * Sh::kPitch; x += kThreads) keys[x] = 0.f;
    if (tid == 0) sm.joint.n = 0;
    const Share sh = find_share(a, sm.share, kThreads);
    Walk w = walk_begin(a, sh);
#pragma unroll 1
    while (w.more) {
        const Sight v = sight_of(a, w);
        const int nt = w.upto - w.i;
        bool bad = w.s.bad;
        auto find = [&](int i) {
            if (tid < KT) {
                long long ko = -1, vo = -1;
                if (i < nt && !key_row(a, w, v, tile_at(w.u, w.i + i) * KT + tid, &ko, &vo, &bad)) ko = vo = -1;
                sm.row[i % 3][0][tid] = ko;
                sm.row[i % 3][1][tid] = vo;
            }
        };
        auto fetch = [&](int i) {
            if (i < nt) {
                // (a thread has one group of four of every kStep-th key; eight rows are looked up at a time)
                constexpr int kStep = kThreads / Sh::kVecs, kRound = KT / kStep < 8 ? KT / kStep : 8;
                const int c = tid % Sh::kVecs, key0 = tid / Sh::kVecs;
                if (c < quads) {
#pragma unroll 1
                    for (int y = 0; y < 2 * KT; y += kRound * kStep) {
                        const int which = y >= KT, at = key0 + y - which * KT;
                        const T* const pool = static_cast<const T*>(which ? a.v : a.k) + c * 4;
                        float* const to = which ? vals + ((i & 1) * KT + at) * Sh::kRow + c * 4 : keys + ((i & 1) * KT + at) * Sh::kPitch + c * 4;
                        const int pitch = (which ? Sh::kRow : Sh::kPitch) * kStep;
                        long long off[kRound];
#pragma unroll
                        for (int x = 0; x < kRound; ++x) off[x] = sm.row[i % 3][which][at + x * kStep];
                        if (sizeof(T) == 4 && aligned) {
#pragma unroll
                            for (int x = 0; x < kRound; ++x)
                                if (off[x] >= 0) copy4(to + x * pitch, reinterpret_cast<const float*>(pool + off[x]));
                        } else if (aligned) {
                            float z[kRound][4];
#pragma unroll
                            for (int x = 0; x < kRound; ++x)
                                if (off[x] >= 0) widen(pool + off[x], z[x]);
#pragma unroll
                            for (int x = 0; x < kRound; ++x)
                                if (off[x] >= 0) *reinterpret_cast<float4*>(to + x * pitch) = make_float4(z[x][0], z[x][1], z[x][2], z[x][3]);
                        } else {
#pragma unroll 1
                            for (int x = 0; x < kRound; ++x) {
                                const long long o = sm.row[i % 3][which][at + x * kStep];
                                for (int e = 0; e < 4; ++e)
                                    if (o >= 0 && c * 4 + e < a.D) to[x * pitch + e] = to_float(pool[o + e]);
                            }
                        }
                    }
                }
            }
            cp_async_commit();
        };
        find(0);
        find(1);
#pragma unroll
        for (int x0 = 0; x0 < Sh::kRows * Sh::kVecs; x0 += kThreads) {
            const int row = (x0 + tid) / Sh::kVecs, c = (x0 + tid) % Sh::kVecs;
            if (c < quads) {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                if (row < v.count) {
                    const int r = w.r0 + row, t = a.by_group(r);
                    const T* src = static_cast<const T*>(a.q) + w.b * a.qs[0] + t * a.qs[1] + (w.h * a.group + r - t * a.group) * a.qs[2] + c * 4;
                    if (q_vec) {
                        widen(src, y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c * 4 + e < a.D) y[e] = to_float(src[e]);
                    }
                }
                *reinterpret_cast<float4*>(&sm.q[row][c * 4]) = make_float4(y[0] * a.kf, y[1] * a.kf, y[2] * a.kf, y[3] * a.kf);
            }
        }
        if (tid < Sh::kRows) {
            sm.m[tid] = -INFINITY;
        }
        float m = -INFINITY, l = 0.f;
        const int pos = mine < v.count ? w.s.base + a.by_group(w.r0 + mine) : -1, low = mine < v.count ? low_of(a, pos) : 0;
        float acc[8][8];
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[r][x] = 0.f;
        __syncthreads();
        fetch(0);
#pragma unroll 1
        for (int i = 0; i < nt; ++i) {
            fetch(i + 1);
            find(i + 2);
            cp_async_wait<1>();
            __syncthreads();
            const int start = tile_at(w.u, w.i + i) * KT;
            const bool whole = whole_tile(a, v, start, KT);
            bool raised = false;
            const bool active = warp % kBlocks * 4 < v.count;
            float y[kI], top = -INFINITY;
            if (active) {
                float s[4][kI];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int x = 0; x < kI; ++x) s[r][x] = 0.f;
                const float* const kr = keys + ((i & 1) * KT + 8 * part_of_keys + kg) * Sh::kPitch;
                const float* const qr = &sm.q[warp % kBlocks * 4][0];
#pragma unroll 2
                for (int d = dq * 4; d < quads * 4; d += 16) {
                    float4 q[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) q[r] = *reinterpret_cast<const float4*>(qr + r * (Sh::kRow + 4) + d);
#pragma unroll
                    for (int x = 0; x < kI; ++x) {
                        const float4 k = *reinterpret_cast<const float4*>(kr + x * 8 * PARTS * Sh::kPitch + d);
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[r][x] = fmaf(q[r].x, k.x, fmaf(q[r].y, k.y, fmaf(q[r].z, k.z, fmaf(q[r].w, k.w, s[r][x]))));
                    }
                }
                __syncwarp();
                // the four parts of D: a thread keeps one row of four
#pragma unroll
                for (int x = 0; x < kI; ++x) {
                    const bool up = dq & 2, odd = dq & 1;
                    const float a0 = (up ? s[2][x] : s[0][x]) + __shfl_xor_sync(0xffffffffu, up ? s[0][x] : s[2][x], 2);
                    const float a1 = (up ? s[3][x] : s[1][x]) + __shfl_xor_sync(0xffffffffu, up ? s[1][x] : s[3][x], 2);
                    y[x] = (odd ? a1 : a0) + __shfl_xor_sync(0xffffffffu, odd ? a0 : a1, 1);
                }
#pragma unroll
                for (int x = 0; x < kI; ++x) {
                    const int p = start + kg + 8 * (PARTS * x + part_of_keys);
                    if (!whole && !(p <= pos && (p >= low || p < a.sinks))) y[x] = -INFINITY;
                    top = fmaxf(top, y[x]);
                }
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (PARTS > 1 && kg == 0) sm.top[part_of_keys][mine] = top;
            }
            if constexpr (PARTS > 1) __syncthreads();
            if (active) {
                if constexpr (PARTS > 1) {
#pragma unroll
                    for (int x = 0; x < PARTS; ++x) top = fmaxf(top, sm.top[x][mine]);
                }
                float f = 1.f;
                if (top > m + kLag) {
                    f = ex2(m - top);
                    m = top;
                    l *= f;
                    raised = true;
                }
                if (kg == 0 && part_of_keys == 0) sm.factor[mine] = f;
#pragma unroll
                for (int x = 0; x < kI; ++x) {
                    const float p = y[x] == -INFINITY ? 0.f : ex2(y[x] - m);
                    l += p;
                    sm.p[kg + 8 * (PARTS * x + part_of_keys)][mine] = p;
                }
            }
            raised = __syncthreads_or(raised);
            if (rows8 < v.count) {
                if (raised) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const float f = rows8 + r < v.count ? sm.factor[rows8 + r] : 1.f;
#pragma unroll
                        for (int x = 0; x < 8; ++x) acc[r][x] *= f;
                    }
                }
                auto add = [&](int key, bool guard) {
                    const float4 pa = *reinterpret_cast<const float4*>(&sm.p[key][rows8]), pb = *reinterpret_cast<const float4*>(&sm.p[key][rows8 + 4]);
                    const float p[8] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 val = *reinterpret_cast<const float4*>(vals + ((i & 1) * KT + key) * Sh::kRow + ((col + c * Sh::kLanes) * 4 < Sh::kRow ? (col + c * Sh::kLanes) * 4 : 0));
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            if (guard && p[r] == 0.f) continue;
                            acc[r][4 * c] = fmaf(p[r], val.x, acc[r][4 * c]);
                            acc[r][4 * c + 1] = fmaf(p[r], val.y, acc[r][4 * c + 1]);
                            acc[r][4 * c + 2] = fmaf(p[r], val.z, acc[r][4 * c + 2]);
                            acc[r][4 * c + 3] = fmaf(p[r], val.w, acc[r][4 * c + 3]);
                        }
                    }
                };
                if (whole) {
#pragma unroll 4
                    for (int key = split; key < KT; key += kSplit) add(key, false);
                } else {
#pragma unroll 1
                    for (int key = split; key < KT; key += kSplit) add(key, true);
                }
            }
            __syncthreads();
        }
        // the sums of the rows, and the splits of O, which lie in the place of keys and values
        cp_async_wait<0>();
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (kg == 0) {
            if (part_of_keys == 0) sm.m[mine] = m;
            sm.l[part_of_keys][mine] = l;
        }
        float* const o_at = sm.kv;             // [kSplit][kHeld][kRow]
        static_assert(kSplit * kHeld * Sh::kRow <= static_cast<int>(sizeof(sm.kv) / sizeof(float)), "fits");
        if (rows8 < v.count) {
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if ((col + c * Sh::kLanes) * 4 < Sh::kRow)
                        *reinterpret_cast<float4*>(o_at + (split * kHeld + rows8 + r) * Sh::kRow + (col + c * Sh::kLanes) * 4) =
                            make_float4(acc[r][4 * c], acc[r][4 * c + 1], acc[r][4 * c + 2], acc[r][4 * c + 3]);
        }
        bad = __syncthreads_or(bad);
        float* const part = leave_unit(a, sh, w, v.count, sm.joint, tid);
#pragma unroll 2
        for (int x = tid; x < v.count * Sh::kVecs; x += kThreads) {
            const int row = x / Sh::kVecs, c = x % Sh::kVecs;
            if (c >= quads) continue;
            float so[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int s = 0; s < kSplit; ++s) {
                const float4 y = *reinterpret_cast<const float4*>(o_at + (s * kHeld + row) * Sh::kRow + c * 4);
                so[0] += y.x; so[1] += y.y; so[2] += y.z; so[3] += y.w;
            }
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < PARTS; ++x) sum += sm.l[x][row];
            put<T>(a, w, part, row, c * 4, sm.m[row], bad && row_lost(a, w, row) ? NAN : sum, so);
        }
        __syncthreads();
        if (a.D % 4 != 0) {                    // (the keys' columns beyond D are zero again)
            for (int x = tid; x < 2 * KT * Sh::kPitch; x += kThreads)
                if (x % Sh::kPitch >= a.D) keys[x] = 0.f;
        }
        walk_next(a, w);
    }
    join_units<T>(a, sm.joint, tid, kThreads);
}

// ---- launches ----------------------------------------------------------------------------------------------------------

template <typename T, int NJ, int R>
cudaError_t launch_few(const AttendArgs& a, bool aligned, bool q_vec, int ctas, cudaStream_t stream) {
    constexpr int bytes = static_cast<int>(sizeof(FewSmem<T, NJ, R>));
    static_assert(bytes <= 227 * 1024, "fits an SM");
    static std::atomic<unsigned long long> asked{0};
    const cudaError_t e = allow_shared(attend_few_kernel<T, NJ, R>, bytes, asked);
    if (e != cudaSuccess) return e;
    return launch_together(attend_few_kernel<T, NJ, R>, ctas, kThreads, bytes, stream, a, static_cast<int>(aligned), static_cast<int>(q_vec));
}
template <typename T, int NJ, int PARTS>
cudaError_t launch_many(const AttendArgs& a, bool aligned, bool q_vec, int ctas, cudaStream_t stream) {
    constexpr int bytes = static_cast<int>(sizeof(ManySmem<NJ>));
    static_assert(bytes <= 227 * 1024, "fits an SM");
    static std::atomic<unsigned long long> asked{0};
    const cudaError_t e = allow_shared(attend_many_kernel<T, NJ, PARTS>, bytes, asked);
    if (e != cudaSuccess) return e;
    return launch_together(attend_many_kernel<T, NJ, PARTS>, ctas, kThreads, bytes, stream, a, static_cast<int>(aligned), static_cast<int>(q_vec));
}
template <typename T, int NJ>
cudaError_t pick_many(const AttendArgs& a, bool aligned, bool q_vec, int ctas, cudaStream_t stream) {
    if constexpr (sizeof(T) == 4) {            // (16-bit shapes that the tensor cores do not take are too rare for kernels of their own)
        if (a.rows <= 8) return launch_many<T, NJ, 4>(a, aligned, q_vec, ctas, stream);
        if (a.rows <= 16) return launch_many<T, NJ, 2>(a, aligned, q_vec, ctas, stream);
    }
    return launch_many<T, NJ, 1>(a, aligned, q_vec, ctas, stream);
}
// Up to 4 rows (2 where D is beyond 128), which the kernel that reads takes in one pass, are its; the others the one's that multiplies.  16 sequences
// of up to 4096 tokens, 4 key-value heads: 4 rows 41.2 and 55.2 us (D = 128), 32.6 and 43.0 (64), 8 rows 67.0 and 59.8, 50.9 and 45.4; D = 256:
// 2 rows 59.3 and 93.6, 4 rows 89.6 and 93.5 (64 sequences: 352.7 and 312.5).
constexpr int few_each(int D) { return D <= 128 ? 4 : 2; }
bool few(int D, int rows) { return rows <= few_each(D); }
template <typename T>
cudaError_t pick(const AttendArgs& a, bool aligned, bool q_vec, int ctas, cudaStream_t stream) {
    const int nj = (a.D + 31) / 32;
    if (a.rows <= 4) {
        if (nj <= 2) return launch_few<T, 2, 4>(a, aligned, q_vec, ctas, stream);
        if (nj <= 3) return launch_few<T, 3, 4>(a, aligned, q_vec, ctas, stream);
        if (nj <= 4) return launch_few<T, 4, 4>(a, aligned, q_vec, ctas, stream);
        return launch_few<T, 8, 2>(a, aligned, q_vec, ctas, stream);
    }
    if (nj <= 2) return pick_many<T, 2>(a, aligned, q_vec, ctas, stream);
    if (nj <= 3) return pick_many<T, 3>(a, aligned, q_vec, ctas, stream);
    if (nj <= 4) return pick_many<T, 4>(a, aligned, q_vec, ctas, stream);
    return pick_many<T, 8>(a, aligned, q_vec, ctas, stream);
}

}  // namespace

void attend_rows_plan(AttendArgs* a) {
    const int rows = a->n * a->group;
    if (few(a->D, rows)) {
        a->rows = few_each(a->D);
        a->span = kFewKeys;
        a->extra = 6;                          // a unit's beginning and end, 8000 clocks, where a tile takes 1300
        a->whole = 6;                          // 4 tiles: 7.5 us by one CTA, 9.2 by four; 8 tiles: 9.8 (D = 64) and 12.5 (128) against 9.5 and 10.9 by eight
    } else {
        const int tiles = (rows + 31) / 32;
        a->rows = ((rows + tiles - 1) / tiles + 7) / 8 * 8;
        a->span = a->D <= 128 ? 64 : 32;
        a->extra = 1;
        a->whole = 1;                          // (a tile takes longer than the join)
    }
    a->slack = a->extra;
    a->per_page = 1;
}
int attend_rows_most() { return 32; }

cudaError_t launch_attend_rows(const AttendArgs& a, int dtype, bool aligned, bool q_vec, int ctas, cudaStream_t stream) {
    return dtype == BV_DTYPE_F32 ? pick<float>(a, aligned, q_vec, ctas, stream) : pick<__nv_bfloat16>(a, aligned, q_vec, ctas, stream);
}

}  // namespace bv
