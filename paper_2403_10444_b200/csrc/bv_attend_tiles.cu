// Attention over a paged cache in 16 bits on the tensor cores: bv_cache_attend for bf16, D a multiple of 8 up to 128, pages of a
// multiple of 8 tokens, rows at 16-byte strides.
//
// A unit is one key-value head of a sequence with N query rows (the heads of its group times the block's tokens: 1 to some 100), a tile
// 128 keys.  Keys are the large side, so they take the M side of the matrix instructions and nothing is padded but N to 16:
//   S^T [128 keys, N] = K Q^T            K as it lies in its pages, K-major
//   O^T [D, N]       += V^T P            V as it lies in its pages, M-major; P [128 keys, N] from shared memory
// One warp loads (TMA, a box per page and 64 columns, 128-byte swizzle, a ring of slots that hold a tile's keys or its values), one thread
// issues the matrix instructions, four warps turn S into P: a thread has one key and goes over the N rows, so the mask, the
// exponential and the rounding need no other lane.  What softmax usually needs across lanes is avoided: each row has an integer
// reference m in shared memory, weights are 2^{k s - m}, and only where some score exceeds its reference by more than 8 (a vote
// per tile) the new maxima are formed, and O and the sums scaled by the power of two between the old and the new reference.
// Sums stay per thread until a unit ends.  Weights are rounded to 16 bits for the second product, and the sums are taken of
// the rounded weights: a row of one key is that key's value exactly, and the error of a row, 2^-9 of its terms at most, is that
// of an output rounded once more.
//
// Bound: HBM.  A tile of D = 128 is 64 KB, 2850 clocks of an SM's share of the copy bandwidth; the two products take 8 instructions
// each (S: 128 x N x 128), the four warps some 5 N instructions.  The ring holds up to 192 KB, three tiles.
//
// What a row may not see is taken out twice: its weight is 0 whatever the score is, and rows of V that no row of the unit sees (or that were never
// loaded) are set to 0 in shared memory, since 0 times an infinity is not 0.  Rows of V that some see and others do not keep their finite
// elements there; the others are added where they belong when the unit ends, from global memory.
#include <cuda.h>

#include "bv_cache.cuh"
#include "bv_launch.h"

namespace bv {
namespace {

constexpr int kThreads = 192, kSoft = 128, kTile = 128;
constexpr int kProducer = 4, kIssuer = 5;                       // warps; 0 .. 3 are the softmax's
constexpr float kNone = -3.0e38f;                               // the reference of a row that has seen no score
constexpr float kLag = 8.f;                                     // how far a score may exceed its reference

// ---- instructions ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int token, int head, int page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(token), "r"(head), "r"(page), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void ld16(uint32_t addr, float* x) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
// (the values are not there before this; the operands keep the compiler from using them earlier)
__device__ __forceinline__ void wait_ld(float* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]),
                   "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15])::"memory");
}
__device__ __forceinline__ void st16(uint32_t addr, const float* x) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
                 "r"(__float_as_uint(x[0])), "r"(__float_as_uint(x[1])), "r"(__float_as_uint(x[2])), "r"(__float_as_uint(x[3])), "r"(__float_as_uint(x[4])),
                 "r"(__float_as_uint(x[5])), "r"(__float_as_uint(x[6])), "r"(__float_as_uint(x[7])), "r"(__float_as_uint(x[8])), "r"(__float_as_uint(x[9])),
                 "r"(__float_as_uint(x[10])), "r"(__float_as_uint(x[11])), "r"(__float_as_uint(x[12])), "r"(__float_as_uint(x[13])), "r"(__float_as_uint(x[14])),
                 "r"(__float_as_uint(x[15]))
                 : "memory");
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// (a warp's lanes come together before what all of them have to execute at once)
__device__ __forceinline__ void soft_sync() { __syncwarp(); asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool soft_any(bool x) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(static_cast<uint32_t>(x)) : "memory");
    return r != 0;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Shared-memory descriptors: start address, leading and stride byte offsets in units of 16 bytes, version 1, layout (2: 128-byte swizzle,
// 0: none).
__device__ __forceinline__ uint64_t describe(uint32_t addr, uint32_t lead, uint32_t stride, uint64_t layout) {
    return static_cast<uint64_t>((addr & 0x3ffff) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 | static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | layout << 61;
}
// Instruction descriptor: 32-bit sums, bf16 operands; which operands are M / N-major; the sizes.
__host__ __device__ constexpr uint32_t instruction(int M, int N, bool a_m, bool b_n) {
    return 1u << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(a_m) << 15 | static_cast<uint32_t>(b_n) << 16 | static_cast<uint32_t>(N >> 3) << 17 |
           static_cast<uint32_t>(M >> 4) << 24;
}

// ---- layout ------------------------------------------------------------------------------------------------------------

template <int NP, int N>
struct Shape {
    static constexpr int kSlot = kTile * 128 * NP;                       // bytes of a slot: NP panels of 128 rows of 64 columns
    static constexpr int kPanel = kTile * 128;
    static constexpr int kQ = NP * N * 128, kP = N * kTile * 2;
    static constexpr int kRest = N > 64 ? 4096 : 3072;
    static constexpr int kFit = (227 * 1024 - kRest - kQ - kP) / kSlot;
    static constexpr int kSlots = kFit < 8 ? kFit : 8;
    static constexpr int kColumns = 3 * N <= 64 ? 64 : 3 * N <= 128 ? 128 : 3 * N <= 256 ? 256 : 512;      // of tensor memory: S twice, O
    static constexpr int kBytes = kSlots * kSlot + kQ + kP + kRest;
    static_assert(kSlots >= 4, "two tiles in flight");
};
template <int NP, int N>
struct __align__(1024) Smem {
    using Sh = Shape<NP, N>;
    char ring[Sh::kSlots][Sh::kSlot];
    char q[Sh::kQ];
    char p[Sh::kP];
    float nref[N], factor[N];                  // minus the references; what the last move of the references scales by
    float part[4][N];                          // maxima, at the end sums, by warp
    int pos[N], low[N];                        // the rows' positions, and the first positions of their windows
    unsigned long long full[8], empty[8], s_full[2], p_full, p_done, q_full, drain;
    ShareSmem share;
    uint32_t tmem;
    int abort, fix;
    JointSmem joint;
};

struct Geometry {      // of a tile
    int start, keys;   // its first position, its keys
};
__device__ __forceinline__ Geometry geometry(const AttendArgs& a, int tile) {
    Geometry g;
    g.start = tile_start(a, tile);
    g.keys = a.span;
    if (a.per_page > 1) {
        const int left = a.page - tile % a.per_page * a.span;
        if (left < g.keys) g.keys = left;
    }
    return g;
}
// Is page j of a sequence one that the unit's rows see some of?
__device__ __forceinline__ bool page_seen(const AttendArgs& a, int j, int p1, int low0) {
    const long long begin = static_cast<long long>(j) * a.page;
    return begin <= p1 && (begin + a.page > low0 || begin < a.sinks);
}

// Sums over the lanes of 16 or 32 values each: lane x ends up with the sum of value x (of x % 16).
template <int W> __device__ __forceinline__ float across(float* v, int lane) {
    if (W == 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 16);
    }
#pragma unroll
    for (int w = W / 2; w > 0; w >>= 1) {
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const bool up = lane & w;
            const float send = up ? v[i] : v[i + w], keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
        }
    }
    return v[0];
}
// The largest of the lanes' values (as integers that are in the order of the values).
__device__ __forceinline__ float warp_max(float x) {
    int i = __float_as_int(x);
    i ^= (i >> 31) & 0x7fffffff;
    i = __reduce_max_sync(0xffffffffu, i);
    i ^= (i >> 31) & 0x7fffffff;
    return __int_as_float(i);
}

template <int NP, int N>
__global__ void __launch_bounds__(kThreads, 1) attend_tiles_kernel(const AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const int q_vec) {
    extern __shared__ __align__(1024) char raw[];
    using Sh = Shape<NP, N>;
    Smem<NP, N>& sm = *reinterpret_cast<Smem<NP, N>*>(raw);
    static_assert(sizeof(Smem<NP, N>) <= Sh::kBytes, "the rest fits");
    constexpr int kSlots = Sh::kSlots;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t limit = a.wait_limit ? a.wait_limit : 1u << 24;

    // (rows of a slot that no page reaches are never written: they stay zero)
    for (int x = tid; x < kSlots * Sh::kSlot / 16; x += kThreads)
        if (x * 16 % Sh::kPanel / 128 >= a.span) reinterpret_cast<uint4*>(sm.ring)[x] = make_uint4(0, 0, 0, 0);
    fence_async();
    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_u32(&sm.full[i]), 1);
            mbar_init(smem_u32(&sm.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sm.s_full[i]), 1);
        mbar_init(smem_u32(&sm.p_full), kSoft);
        mbar_init(smem_u32(&sm.p_done), 1);
        mbar_init(smem_u32(&sm.q_full), kSoft);
        mbar_init(smem_u32(&sm.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.abort = sm.fix = sm.joint.n = 0;
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "n"(Sh::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    const Share sh = find_share<kThreads>(a, sm.share);
    fence_after();
    const uint32_t tmem = sm.tmem;
    auto s_at = [&](int g) { return tmem + (g & 1) * N; };
    const uint32_t o_at = tmem + 2 * N;
    Walk w = walk_begin(a, sh);

    if (warp == kProducer) {
        // ---- loads
        int x = 0;                             // slots filled
        bool ok = true;
        const int rows = a.page < kTile ? a.page : kTile;                // of a box
        for (; w.more && ok; walk_next(a, w)) {
            const int count = w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0;
            const int p1 = w.s.base + (w.r0 + count - 1) / a.group, low0 = low_of(a, w.s.base + w.r0 / a.group);
            const int per = a.per_page > 1 ? 1 : a.span / a.page;        // pages of a tile
            auto entry = [&](int i) {          // the page of this lane in tile i, or -1
                if (i >= w.upto || lane >= per) return -1;
                const int tile = tile_at(w.u, i);
                const int j = a.per_page > 1 ? tile / a.per_page : tile * per + lane;
                if (!page_seen(a, j, p1, low0)) return -1;
                const int page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
                return page < 0 || page >= a.num_pages ? -1 : page;
            };
            int next = entry(w.i);
            for (int i = w.i; i < w.upto && ok; ++i) {
                const int page = next;
                next = entry(i + 1);
                const int token = a.per_page > 1 ? tile_at(w.u, i) % a.per_page * a.span : 0;
                const unsigned there = __ballot_sync(0xffffffffu, page >= 0);
#pragma unroll
                for (int which = 0; which < 2; ++which, ++x) {
                    const int slot = x % kSlots;
                    ok = ok && mbar_wait_now(smem_u32(&sm.empty[slot]), (x / kSlots & 1) ^ 1, a.status, limit);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&sm.full[slot]);
                    if (lane == 0) mbar_arrive_expect(bar, __popc(there) * rows * 128 * NP);
                    __syncwarp();
                    if (page >= 0) {
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            tma_load(smem_u32(sm.ring[slot]) + p * Sh::kPanel + lane * rows * 128, which ? &v_map : &k_map, p * 64, token, w.h, page, bar);
                    }
                }
            }
        }
        // (a launch that gave up leaves when its copies are in)
        if (!ok)
            for (int y = x < kSlots ? 0 : x - kSlots; y < x; ++y) mbar_wait_now(smem_u32(&sm.full[y % kSlots]), y / kSlots & 1, a.status, limit);
    } else if (warp == kIssuer) {
        // ---- products
        if (lane == 0) {
            constexpr uint32_t qk = instruction(kTile, N, false, false), pv = instruction(64 * NP, N, true, true);
            int g = 0, units = 0;              // tiles, units gone through
            bool ok = true;
            auto wait = [&](unsigned long long& bar, int phase) { ok = ok && mbar_wait_now(smem_u32(&bar), phase & 1, a.status, limit); };
            auto scores = [&](int t) {
                const int x = 2 * t;
                wait(sm.full[x % kSlots], x / kSlots);
                if (!ok) return;
                fence_after();
                const uint32_t k = smem_u32(sm.ring[x % kSlots]), q = smem_u32(sm.q);
#pragma unroll
                for (int i = 0; i < 4 * NP; ++i)
                    mma(s_at(t), describe(k + i / 4 * Sh::kPanel + i % 4 * 32, 16, 1024, 2), describe(q + i / 4 * N * 128 + i % 4 * 32, 16, 1024, 2), qk, i > 0);
                commit(smem_u32(&sm.empty[x % kSlots]));
                if (a.never_signal != 1) commit(smem_u32(&sm.s_full[t & 1]));
            };
            for (; w.more && ok; walk_next(a, w), ++units) {
                const int nt = w.upto - w.i;
                wait(sm.q_full, units);
                if (ok) scores(g);
                for (int i = 0; i < nt && ok; ++i, ++g) {
                    if (i + 1 < nt) scores(g + 1);
                    const int x = 2 * g + 1;
                    wait(sm.full[x % kSlots], x / kSlots);
                    wait(sm.p_full, g);
                    if (!ok) break;
                    fence_after();
                    const uint32_t v = smem_u32(sm.ring[x % kSlots]), p = smem_u32(sm.p);
#pragma unroll
                    for (int j = 0; j < kTile / 16; ++j)
                        mma(o_at, describe(v + j * 2048, Sh::kPanel, 1024, 2), describe(p + j * 256, 128, 2048, 0), pv, i > 0 || j > 0);
                    commit(smem_u32(&sm.empty[x % kSlots]));
                    commit(smem_u32(&sm.p_done));
                }
            }
            if (!ok) {
                commit(smem_u32(&sm.drain));
                mbar_wait_now(smem_u32(&sm.drain), 0, a.status, limit);
            }
        }
        __syncwarp();
    } else {
        // ---- weights
        const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
        const int key = tid;                   // of a tile
        // the element of O that this thread has: with 64 of them a warp has 16, in its lower lanes
        const int dim = NP == 2 ? tid : warp * 16 + lane;
        const bool has_dim = dim < a.D && (NP == 2 || lane < 16);
        char* const p_row = sm.p + key / 8 * 128 + key % 8 * 16;
        int g = 0;
        // A wait that gives up: this thread asks for a vote from then on, and behind the vote all of them leave together (sm.abort is
        // set before a vote or after the barrier that follows the look at it, never between).
        bool failed = false, gone = false;
        auto wait = [&](unsigned long long& bar, int phase) {
            if (!mbar_wait_now(smem_u32(&bar), phase & 1, a.status, limit)) {
                failed = true;
                atomicExch(&sm.abort, 1);
            }
        };
        for (; w.more; walk_next(a, w)) {
            const int count = w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0;
            const int p0 = w.s.base + w.r0 / a.group, p1 = w.s.base + (w.r0 + count - 1) / a.group;
            const int low0 = low_of(a, p0), low1 = low_of(a, p1);
            // the query rows, swizzled like the keys; zero beyond the unit's rows and beyond D
            for (int y = tid; y < N * NP * 8; y += kSoft) {
                const int row = y / (NP * 8), c = y - row * (NP * 8);
                uint4 val = make_uint4(0, 0, 0, 0);
                if (row < count && c * 8 < a.D) {
                    const int r = w.r0 + row, t = r / a.group;
                    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + w.b * a.qs[0] + t * a.qs[1] + (w.h * a.group + r - t * a.group) * a.qs[2] + c * 8;
                    if (q_vec) {
                        val = *reinterpret_cast<const uint4*>(src);
                    } else {
                        const uint16_t* e = reinterpret_cast<const uint16_t*>(src);
                        val = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                    }
                }
                *reinterpret_cast<uint4*>(sm.q + c / 8 * N * 128 + row * 128 + ((c % 8) ^ (row & 7)) * 16) = val;
            }
            if (tid < N) {
                const int t = (w.r0 + (tid < count ? tid : 0)) / a.group;
                sm.pos[tid] = w.s.base + t;
                sm.low[tid] = low_of(a, w.s.base + t);
                sm.nref[tid] = -kNone;
            }
            fence_async();
            mbar_arrive(smem_u32(&sm.q_full));
            // (does the CTA's part of the unit read pages that are none?)
            bool bad = w.s.bad;
            {
                const int t0 = tile_at(w.u, w.i), t1 = tile_at(w.u, w.upto - 1);
                const int j0 = tile_start(a, t0) / a.page, j1 = min(tile_start(a, t1) + a.span - 1, p1) / a.page;
                for (int j = j0 + tid; p1 >= 0 && j <= j1; j += kSoft) {
                    if (!page_seen(a, j, p1, low0)) continue;
                    const int page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
                    bad |= page < 0 || page >= a.num_pages;
                }
            }
            float l[N];
#pragma unroll
            for (int c = 0; c < N; ++c) l[c] = 0.f;
            soft_sync();                       // pos, low, nref
            const int nt = w.upto - w.i;
            for (int i = 0; i < nt && !gone; ++i, ++g) {
                const Geometry ge = geometry(a, tile_at(w.u, w.i + i));
                const bool whole = ge.start + ge.keys - 1 <= p0 && (ge.start >= low1 || ge.start + ge.keys <= a.sinks) && ge.keys == kTile;
                unsigned see[(N + 31) / 32];
                wait(sm.s_full[g & 1], g >> 1);
                __syncwarp();
                fence_after();
                float s[N];
#pragma unroll
                for (int c = 0; c < N; c += 16) ld16(s_at(g) + lanes + c, s + c);
                if (!whole) {
                    const int p = ge.start + key;
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        if (c % 32 == 0) see[c / 32] = 0;
                        const bool x = key < ge.keys && p <= sm.pos[c] && (p >= sm.low[c] || p < a.sinks);
                        see[c / 32] |= static_cast<unsigned>(x) << (c % 32);
                    }
                    // the value's row: zero where nobody sees it, its finite elements where some do not
                    const bool any = key < ge.keys && p <= p1 && (p >= low0 || p < a.sinks), all = any && p <= p0 && (p >= low1 || p < a.sinks);
                    const int xv = 2 * g + 1;
                    if (!all) wait(sm.full[xv % kSlots], xv / kSlots);
                    char* row = sm.ring[xv % kSlots] + key * 128;
                    if (!any) {
#pragma unroll
                        for (int e = 0; e < 8 * NP; ++e) *reinterpret_cast<uint4*>(row + e / 8 * Sh::kPanel + ((e + lane) % 8) * 16) = make_uint4(0, 0, 0, 0);
                    } else if (!all) {
                        for (int e = 0; e < 32 * NP; ++e) {
                            uint32_t* at = reinterpret_cast<uint32_t*>(row + e / 32 * Sh::kPanel) + (e + lane) % 32;
                            uint32_t v = *at;
                            const uint32_t was = v;
                            if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
                            if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
                            if (v != was) {
                                *at = v;
                                sm.fix = 1;
                            }
                        }
                    }
                }
                __syncwarp();
#pragma unroll
                for (int c = 0; c < N; c += 16) wait_ld(s + c);
                // k s - m, and whether any of them is too large
                float most = -INFINITY;
#pragma unroll
                for (int c = 0; c < N; c += 4) {
                    const float4 nr = *reinterpret_cast<const float4*>(sm.nref + c);
                    s[c] = fmaf(s[c], a.kf, nr.x);
                    s[c + 1] = fmaf(s[c + 1], a.kf, nr.y);
                    s[c + 2] = fmaf(s[c + 2], a.kf, nr.z);
                    s[c + 3] = fmaf(s[c + 3], a.kf, nr.w);
                }
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < N; ++c) s[c] = see[c / 32] >> (c % 32) & 1 ? s[c] : -INFINITY;
                }
#pragma unroll
                for (int c = 0; c < N; ++c) most = fmaxf(most, s[c]);
                if (soft_any(most > kLag || failed)) {
                    // (the scores once more: what is left of them next to a reference that is none is not exact)
#pragma unroll
                    for (int c = 0; c < N; c += 16) ld16(s_at(g) + lanes + c, s + c);
#pragma unroll
                    for (int c = 0; c < N; c += 16) wait_ld(s + c);
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        s[c] *= a.kf;
                        if (!whole && !(see[c / 32] >> (c % 32) & 1)) s[c] = -INFINITY;
                        const float x = warp_max(s[c]);
                        if (lane == c % 32) sm.part[warp][c] = x;
                    }
                    soft_sync();
                    if (tid < N) {
                        const float top = fmaxf(fmaxf(sm.part[0][tid], sm.part[1][tid]), fmaxf(sm.part[2][tid], sm.part[3][tid]));
                        const float old = -sm.nref[tid];
                        const float now = top - old > kLag ? rintf(top) : old;
                        sm.factor[tid] = now == old ? 1.f : exp2f(old - now);
                        sm.nref[tid] = -now;
                    }
                    gone = *static_cast<volatile int*>(&sm.abort) != 0;
                    soft_sync();
                    if (gone) break;
                    if (i > 0) {
                        wait(sm.p_done, g - 1);
                        __syncwarp();
                        fence_after();
#pragma unroll
                        for (int c = 0; c < N; c += 16) {
                            float o[16];
                            ld16(o_at + lanes + c, o);
                            wait_ld(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= sm.factor[c + e];
                            st16(o_at + lanes + c, o);
                        }
                        wait_st();
                    }
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        l[c] *= sm.factor[c];
                        s[c] += sm.nref[c];
                    }
                }
                if (i > 0) wait(sm.p_done, g - 1);                       // (the last tile's weights have been read)
#pragma unroll
                for (int c = 0; c < N; c += 8) {
                    uint32_t pk[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(ex2(s[c + 2 * e]), ex2(s[c + 2 * e + 1]));
                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                        l[c + 2 * e] += __uint_as_float(pk[e] << 16);
                        l[c + 2 * e + 1] += __uint_as_float(pk[e] & 0xffff0000u);
                    }
                    *reinterpret_cast<uint4*>(p_row + c / 8 * (kTile * 16)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                }
                fence_async();
                fence_before();
                mbar_arrive(smem_u32(&sm.p_full));
            }
            if (!gone) wait(sm.p_done, g - 1);
            __syncwarp();
            fence_after();
            // the sums
#pragma unroll
            for (int c = 0; c < N; c += 32) {
                if (c + 32 <= N) {
                    const float x = across<32>(l + c, lane);
                    sm.part[warp][c + lane] = x;
                } else {
                    const float x = across<16>(l + c, lane);
                    if (lane < 16) sm.part[warp][c + lane] = x;
                }
            }
            bad = soft_any(bad || failed || gone);
            const bool fix = *static_cast<volatile int*>(&sm.fix) != 0;
            float* part = leave_unit(a, sh, w, count, sm.joint, tid);
            if (part && tid < count) {
                part[tid] = -sm.nref[tid];
                part[a.rows + tid] = bad ? NAN : sm.part[0][tid] + sm.part[1][tid] + sm.part[2][tid] + sm.part[3][tid];
            }
#pragma unroll 1
            for (int c0 = 0; c0 < count; c0 += 16) {
                float o[16];
                __syncwarp();
                ld16(o_at + lanes + c0, o);
                wait_ld(o);
                if (fix && has_dim) {
                    // what is not finite among the values that some rows see and others do not
#pragma unroll 1
                    for (int i = w.i; i < w.upto; ++i) {
                        const Geometry ge = geometry(a, tile_at(w.u, i));
                        if (ge.start + ge.keys - 1 <= p0 && (ge.start >= low1 || ge.start + ge.keys <= a.sinks)) continue;
                        for (int x = 0; x < ge.keys; ++x) {
                            const int p = ge.start + x;
                            const bool any = p <= p1 && (p >= low0 || p < a.sinks), all = p <= p0 && (p >= low1 || p < a.sinks);
                            if (!any || all) continue;
                            const int page = __ldg(a.table + static_cast<long long>(w.b) * a.width + p / a.page);
                            if (page < 0 || page >= a.num_pages) continue;
                            const float v = to_float((static_cast<const __nv_bfloat16*>(a.v) + page * a.vs[0] + w.h * a.vs[1] + p % a.page * a.vs[2])[dim]);
                            if (isfinite(v)) continue;
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (c0 + e < count && p <= sm.pos[c0 + e] && (p >= sm.low[c0 + e] || p < a.sinks)) o[e] += v;
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = c0 + e;
                    if (row < count && has_dim) {
                        if (part) {
                            part[2 * a.rows + static_cast<size_t>(row) * a.D + dim] = o[e];
                        } else {
                            const float sum = sm.part[0][row] + sm.part[1][row] + sm.part[2][row] + sm.part[3][row];
                            const int r = w.r0 + row, t = r / a.group;
                            __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out) + w.b * a.os[0] + t * a.os[1] + (w.h * a.group + r - t * a.group) * a.os[2] + dim;
                            *dst = __float2bfloat16_rn(bad ? NAN : sum == 0.f ? 0.f : o[e] / sum);
                        }
                    }
                }
            }
            fence_before();
            soft_sync();
            if (tid == 0) sm.fix = 0;
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Sh::kColumns) : "memory");
    join_units<__nv_bfloat16>(a, sm.joint, tid, kThreads);
}

// ---- launch ------------------------------------------------------------------------------------------------------------

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                            CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encode_fn() {
    static const Encode fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    return fn;
}
// The map of a pool: columns, tokens of a page, heads, pages; a box is 64 columns (128 bytes) of a page's tokens, at most 128.
bool encode(const AttendArgs& a, const void* pool, const long long* stride, CUtensorMap* map) {
    const Encode fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(a.D), static_cast<cuuint64_t>(a.page), static_cast<cuuint64_t>(a.Hkv), static_cast<cuuint64_t>(a.num_pages)};
    // (the stride of an axis of one is nobody's concern, but has to be one that the map takes)
    cuuint64_t st[3] = {static_cast<cuuint64_t>(stride[2]) * 2, static_cast<cuuint64_t>(a.Hkv > 1 ? stride[1] : a.D) * 2, static_cast<cuuint64_t>(a.num_pages > 1 ? stride[0] : a.D) * 2};
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(a.page < kTile ? a.page : kTile), 1, 1}, ones[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, st, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NP, int N>
cudaError_t launch(const AttendArgs& a, const CUtensorMap& k, const CUtensorMap& v, bool q_vec, int ctas, cudaStream_t stream) {
    const cudaError_t e = cudaFuncSetAttribute(attend_tiles_kernel<NP, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<NP, N>::kBytes);
    if (e != cudaSuccess) return e;
    return launch_together(attend_tiles_kernel<NP, N>, ctas, kThreads, Shape<NP, N>::kBytes, stream, a, k, v, static_cast<int>(q_vec));
}
template <int NP>
cudaError_t pick(const AttendArgs& a, const CUtensorMap& k, const CUtensorMap& v, bool q_vec, int ctas, cudaStream_t stream) {
    switch (a.rows) {
        case 16: return launch<NP, 16>(a, k, v, q_vec, ctas, stream);
        case 32: return launch<NP, 32>(a, k, v, q_vec, ctas, stream);
        case 48: return launch<NP, 48>(a, k, v, q_vec, ctas, stream);
        case 64: return launch<NP, 64>(a, k, v, q_vec, ctas, stream);
        default: return launch<NP, 80>(a, k, v, q_vec, ctas, stream);
    }
}

}  // namespace

bool attend_tiles_takes(const AttendArgs& a) { return a.D >= 16 && a.D <= 128 && a.D % 8 == 0 && a.page % 8 == 0 && a.page <= (1 << 20); }
// The fewest tiles of rows, of sizes as even as multiples of 16 are.
int attend_tiles_rows(int rows) {
    const int tiles = (rows + 79) / 80;
    return ((rows + tiles - 1) / tiles + 15) / 16 * 16;
}
void attend_tiles_plan(AttendArgs* a) {
    a->span = a->page <= kTile ? kTile / a->page * a->page : kTile;
    a->per_page = a->page <= kTile ? 1 : (a->page + kTile - 1) / kTile;
}
cudaError_t launch_attend_tiles(const AttendArgs& a, bool q_vec, int ctas, cudaStream_t stream, bool* taken) {
    CUtensorMap k, v;
    *taken = encode(a, a.k, a.ks, &k) && encode(a, a.v, a.vs, &v);
    if (!*taken) return cudaSuccess;
    return a.D <= 64 ? pick<1>(a, k, v, q_vec, ctas, stream) : pick<2>(a, k, v, q_vec, ctas, stream);
}

}  // namespace bv
