// Attention over a paged cache, for every shape, type, alignment and stride: bv_cache_attend where bv_attend_tiles.cu does not take
// the call (32-bit caches above all: their products are 32-bit FMAs, since a tensor core would round the inputs to 10 bits of mantissa).
//
// One pass over the keys with a running reference m and sum l per row:  p = 2^{k q.k - m},  l += p,  O += p v,  and where a score
// exceeds m by more than 8 (first of all where m is still -inf)  m <- that score, l and O scaled by 2^{m_old - m}.  A reference
// that lags by up to 8 costs nothing in 32 bits (terms of up to 256 instead of 1) and saves nearly all of the scaling.
//
// A CTA stages tiles of 32 keys and their values in shared memory, three deep, with 16-byte asynchronous copies (element by
// element where rows are not whole aligned vectors).  Eight lanes share a key: each holds every 8th group of four of the row's D elements, of R query
// rows at a time, in registers, so a key costs 2 R D / 8 FMAs and 3 R shuffles a lane.  The eight warps take different query rows
// (RG groups of R) and, where there are fewer rows than that, different keys of the tile.
#include "bv_cache.cuh"
#include "bv_launch.h"

namespace bv {
namespace {

constexpr int kThreads = 256, kWarps = 8, kKeys = 32, kStages = 3;

template <typename T> __device__ __forceinline__ void load4(const T* p, float (&x)[4]);
template <> __device__ __forceinline__ void load4<float>(const float* p, float (&x)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
template <> __device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, float (&x)[4]) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}

template <typename T, int NJ, int R>
struct RowsSmem {
    T tile[kStages][2][kKeys * NJ * 32];
    long long row[4][2][kKeys];            // element offsets of the keys' rows, of tiles i .. i+3 (negative: no page)
    float part[kWarps][R][NJ * 32 + 2];
    ShareSmem share;
    JointSmem joint;
    int bad;
};

template <typename T, int NJ, int R>
__global__ void __launch_bounds__(kThreads, 1) attend_rows_kernel(const AttendArgs a, const int aligned) {
    extern __shared__ char smem_raw[];
    using Smem = RowsSmem<T, NJ, R>;
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    constexpr int kRow = NJ * 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int group8 = lane >> 3, l8 = lane & 7;
    const int row_groups = a.rows / R;                     // 1, 2, 4 or 8
    const int key_slices = kWarps / row_groups;
    const int rg = warp % row_groups, ks = warp / row_groups;

    // (columns D .. kRow of the staged rows are never copied to: they stay zero)
    for (int x = tid; x < static_cast<int>(sizeof(sm.tile) / 16); x += kThreads) reinterpret_cast<uint4*>(&sm.tile[0][0][0])[x] = make_uint4(0, 0, 0, 0);
    if (tid == 0) sm.bad = sm.joint.n = 0;
    const Share sh = find_share(a, sm.share, kThreads);
    Walk w = walk_begin(a, sh);

    while (w.more) {
        const int count = w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0;
        const int nt = w.upto - w.i;
        // a row's position, and the positions it sees: low .. pos, and those below `sinks`
        float q[R][NJ * 4];
        int pos[R], low[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = w.r0 + rg * R + r;
            const bool valid = rg * R + r < count;
            const int t = valid ? a.by_group(row) : 0, g = valid ? row - t * a.group : 0;
            pos[r] = valid ? w.s.base + t : -1;
            low[r] = valid ? low_of(a, pos[r]) : 0;
            const T* src = static_cast<const T*>(a.q) + w.b * a.qs[0] + t * a.qs[1] + (w.h * a.group + g) * a.qs[2];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = j * 32 + l8 * 4 + e;
                    q[r][j * 4 + e] = valid && d < a.D ? to_float(src[d]) * a.kf : 0.f;
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
        // what all of the unit's rows see, and what none of them does
        const int p0 = w.s.base + a.by_group(w.r0), p1 = w.s.base + a.by_group(w.r0 + count - 1);
        const int low0 = low_of(a, p0), low1 = low_of(a, p1);

        // the rows of tile i's keys (one warp; -1: beyond what anybody sees, -2: a page that is none)
        auto find_rows = [&](int i, long long& ko, long long& vo) {
            ko = vo = -1;
            if (i >= nt) return;
            const int p = tile_at(w.u, w.i + i) * kKeys + lane;
            if (p > p1 || !(p >= low0 || p < a.sinks)) return;
            const int j = a.by_page(p);
            const int page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
            if (page < 0 || page >= a.num_pages) { ko = -2; return; }
            ko = page * a.ks[0] + w.h * a.ks[1] + (p - j * a.page) * a.ks[2];
            vo = page * a.vs[0] + w.h * a.vs[1] + (p - j * a.page) * a.vs[2];
        };
        auto put_rows = [&](int i, long long ko, long long vo) {
            sm.row[i & 3][0][lane] = ko;
            sm.row[i & 3][1][lane] = vo;
            if (ko == -2) sm.bad = 1;
        };
        auto fetch = [&](int i) {
            if (i < nt) {
                T* dst = sm.tile[i % kStages][0];
                if (aligned) {
                    const int vecs = a.D * static_cast<int>(sizeof(T)) / 16;
                    for (int x = tid; x < 2 * kKeys * vecs; x += kThreads) {
                        const int which = x / (kKeys * vecs), y = x - which * kKeys * vecs, key = y / vecs, c = y - key * vecs;
                        const long long off = sm.row[i & 3][which][key];
                        if (off >= 0) {
                            const T* src = static_cast<const T*>(which ? a.v : a.k) + off + c * (16 / sizeof(T));
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst + (which * kKeys + key) * kRow + c * (16 / sizeof(T)))), "l"(src) : "memory");
                        }
                    }
                } else {
                    for (int x = tid; x < 2 * kKeys * a.D; x += kThreads) {
                        const int which = x / (kKeys * a.D), y = x - which * kKeys * a.D, key = y / a.D, c = y - key * a.D;
                        const long long off = sm.row[i & 3][which][key];
                        if (off >= 0) dst[(which * kKeys + key) * kRow + c] = (static_cast<const T*>(which ? a.v : a.k) + off)[c];
                    }
                }
            }
            cp_async_commit();
        };
        if (warp == 0) {
            long long ko, vo;
            for (int i = 0; i < 3; ++i) { find_rows(i, ko, vo); put_rows(i, ko, vo); }
        }
        __syncthreads();
        fetch(0);
        fetch(1);
        for (int i = 0; i < nt; ++i) {
            fetch(i + 2);
            long long ko = 0, vo = 0;
            if (warp == 0) find_rows(i + 3, ko, vo);
            cp_async_wait<2>();
            __syncthreads();
            const int start = tile_at(w.u, w.i + i) * kKeys;
            const bool whole = start + kKeys - 1 <= p0 && (start >= low1 || start + kKeys <= a.sinks);
            const T* kt = sm.tile[i % kStages][0];
            const T* vt = sm.tile[i % kStages][1];
            for (int key = ks * 4 + group8; key < kKeys; key += key_slices * 4) {
                float s[R];
#pragma unroll
                for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    float x[4];
                    load4<T>(kt + key * kRow + j * 32 + l8 * 4, x);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[r] = fmaf(q[r][j * 4 + e], x[e], s[r]);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    s[r] += __shfl_xor_sync(0xffffffffu, s[r], 4);
                    s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
                    s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
                }
                const int p = start + key;
                const bool there = sm.row[i & 3][0][key] >= 0;
                bool some[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const bool see = there && (whole ? rg * R + r < count : p <= pos[r] && (p >= low[r] || p < a.sinks));
                    some[r] = see && s[r] != -INFINITY;               // (a weight of zero takes no value, whatever that is)
                    if (some[r] && s[r] > m[r] + 8.f) {
                        const float f = exp2f(m[r] - s[r]);
                        m[r] = s[r];
                        l[r] *= f;
#pragma unroll
                        for (int x = 0; x < NJ * 4; ++x) acc[r][x] *= f;
                    }
                    s[r] = some[r] ? exp2f(s[r] - m[r]) : 0.f;
                    l[r] += s[r];
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    float x[4];
                    load4<T>(vt + key * kRow + j * 32 + l8 * 4, x);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (some[r]) acc[r][j * 4 + e] = fmaf(s[r], x[e], acc[r][j * 4 + e]);
                }
            }
            if (warp == 0) put_rows(i + 3, ko, vo);        // (tile i - 1's place: its readers are past the barrier above)
            __syncthreads();
        }
        // lanes of one row, then warps of one row group
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int o = 8; o <= 16; o <<= 1) {
                const float om = __shfl_xor_sync(0xffffffffu, m[r], o), ol = __shfl_xor_sync(0xffffffffu, l[r], o);
                const float M = fmaxf(m[r], om);
                const float f = m[r] == -INFINITY ? 0.f : exp2f(m[r] - M), of = om == -INFINITY ? 0.f : exp2f(om - M);
                l[r] = l[r] * f + ol * of;
                m[r] = M;
#pragma unroll
                for (int x = 0; x < NJ * 4; ++x) {
                    const float oa = __shfl_xor_sync(0xffffffffu, acc[r][x], o);
                    acc[r][x] = acc[r][x] * f + oa * of;
                }
            }
            if (group8 == 0) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sm.part[warp][r][j * 32 + l8 * 4 + e] = acc[r][j * 4 + e];
                if (l8 == 0) { sm.part[warp][r][kRow] = m[r]; sm.part[warp][r][kRow + 1] = l[r]; }
            }
        }
        __syncthreads();
        const bool bad = w.s.bad || sm.bad;
        float* part = leave_unit(a, sh, w, count, sm.joint, tid);
        for (int x = tid; x < count * a.D; x += kThreads) {
            const int row = x / a.D, d = x - row * a.D;
            const int g = row / R, r = row - g * R;
            float M = -INFINITY, sl = 0.f, so = 0.f;
            for (int s = 0; s < key_slices; ++s) M = fmaxf(M, sm.part[g + s * row_groups][r][kRow]);
            for (int s = 0; s < key_slices; ++s) {
                const float* p = sm.part[g + s * row_groups][r];
                const float f = p[kRow] == -INFINITY ? 0.f : exp2f(p[kRow] - M);
                sl += p[kRow + 1] * f;
                so += p[d] * f;
            }
            if (bad) sl = NAN;
            if (part) {
                part[2 * a.rows + static_cast<size_t>(row) * a.D + d] = so;
                if (d == 0) { part[row] = M; part[a.rows + row] = sl; }
            } else {
                const int at = w.r0 + row, t = a.by_group(at);
                T* dst = static_cast<T*>(a.out) + w.b * a.os[0] + t * a.os[1] + (w.h * a.group + at - t * a.group) * a.os[2] + d;
                *dst = from_float<T>(sl == 0.f ? 0.f : so / sl);
            }
        }
        __syncthreads();
        if (warp == 0) {
            if (lane == 0) sm.bad = 0;
            __syncwarp();                              // (this warp is the one that sets it)
        }
        walk_next(a, w);
    }
    join_units<T>(a, sm.joint, tid, kThreads);
}

template <typename T, int NJ, int R>
cudaError_t launch(const AttendArgs& a, bool aligned, int ctas, cudaStream_t stream) {
    constexpr int bytes = static_cast<int>(sizeof(RowsSmem<T, NJ, R>));
    static_assert(bytes <= 227 * 1024, "fits an SM");
    static std::atomic<unsigned long long> asked{0};
    const cudaError_t e = allow_shared(attend_rows_kernel<T, NJ, R>, bytes, asked);
    if (e != cudaSuccess) return e;
    return launch_together(attend_rows_kernel<T, NJ, R>, ctas, kThreads, bytes, stream, a, static_cast<int>(aligned));
}
template <typename T>
cudaError_t pick(const AttendArgs& a, bool aligned, int ctas, cudaStream_t stream) {
    const int nj = (a.D + 31) / 32;
    if (nj <= 2) return launch<T, 2, 4>(a, aligned, ctas, stream);
    if (nj <= 3) return launch<T, 3, 4>(a, aligned, ctas, stream);
    if (nj <= 4) return launch<T, 4, 4>(a, aligned, ctas, stream);
    return launch<T, 8, 2>(a, aligned, ctas, stream);
}

}  // namespace

// Query rows of a unit: R a warp, times as many groups of warps as the call's rows fill.
int attend_rows_tile(int D, int rows) {
    const int R = D <= 128 ? 4 : 2;
    int groups = 1;
    while (groups < kWarps && groups * R < rows) groups *= 2;
    return groups * R;
}
int attend_rows_keys() { return kKeys; }

cudaError_t launch_attend_rows(const AttendArgs& a, int dtype, bool aligned, int ctas, cudaStream_t stream) {
    return dtype == BV_DTYPE_F32 ? pick<float>(a, aligned, ctas, stream) : pick<__nv_bfloat16>(a, aligned, ctas, stream);
}

}  // namespace bv
