// Attention over a paged cache in 16 bits on the tensor cores: bv_cache_attend for bf16, D a multiple of 8 up to 128, pages of a
// multiple of 8 tokens, rows at 16-byte strides.
//
// Bound by the cache's bytes: 64 sequences of up to 8192 tokens, 32 heads on 8, D = 128: 195 us, 5.9 TB/s (0.90 of the copy bandwidth); one of
// 131072: 94 us, 5.7 TB/s; blocks of 9 tokens, 64 heads on 8, 64 sequences of up to 16384: 402 to 411 us, 5.7 TB/s, a few calls after a pause; called
// in a loop the GPU reaches its 1000 W and 1560 MHz, and a call takes 449 to 483 (box by box).  Small
// calls by the chain of steps: 7.2 us for a tile of one unit, 11 with a join.  Prompts by the products, of which a tile's keys feed 80 rows: 4 of 2048
// tokens, 32 heads on 8, D = 128: 434 us, 320 TFLOP/s; of 8192: 4.4 ms, 500.
//
// A unit is one key-value head of a sequence with up to N query rows (the heads of its group times the block's tokens), a tile
// 128 keys.  Keys are the large side, so they take the M side of the matrix instructions and nothing is padded but N, to 16:
//   S^T [128 keys, N] = K Q^T            K as it lies in its pages, K-major
//   O^T [D, N]       += V^T P            V as it lies in its pages, M-major; P [128 keys, N] from shared memory
// Two warps load (TMA, a box per page and 64 columns, 128-byte swizzle, a ring of slots that hold a tile's keys or its values), one
// thread issues the matrix instructions, eight warps turn S into P, four of them a tile's 128 keys: a thread has one key and goes over
// the rows, so the mask, the exponential and the rounding need no other lane.  Up to 32 rows the two fours are two teams that take
// units in turn, so that one unit's end and the next one's beginning overlap; from 48 rows on, where the exponentials bound (80 x 128 of
// them are 640 clocks of an SM), each four has half of the rows.  What softmax usually needs across lanes is avoided: each row has an
// integer reference m in shared memory, weights are 2^{k s - m}, and only where some score exceeds its reference by more than 16
// (a vote per tile; 32-bit sums and bf16 weights have the range) maxima are formed, and O and the sums scaled by the power of two between the
// old and the new reference.  A unit's first references are the scores of one key, which are there without any look at the others.  Sums stay per
// thread until a unit ends.  Weights are rounded to 16 bits for the second product, and the sums are taken of the rounded weights: a row of one key is
// that key's value exactly, and the error of a row, 2^-8 of its terms at most, is that of an output rounded once more (0.0022 against 0.0017
// on random values).
//
// What a row may not see is taken out twice: its weight is 0 whatever the score is, and rows of V that no row of the unit sees (or that were never
// loaded) are set to 0 in shared memory, since 0 times an infinity is not 0.  Rows of V that some see and others do not keep their finite
// elements there; the others are added where they belong when the unit ends, from global memory.
//
// What a unit takes besides its tiles is instructions that run once, at some four clocks each, since they are fetched for it: 65000 clocks with
// everything unrolled, 13000 with loops of 16 rows, 8000 now (80 rows) that the first references are one key's, that values are cleared by all threads
// a vector each, that results go out as whole vectors and that the next unit is looked up by one warp beside the first product.
#include <numeric>

#include "bv_cache.cuh"
#include "bv_launch.h"
#include "bv_tensor.cuh"

namespace bv {
namespace {

constexpr int kTile = 128;
constexpr float kNone = -3.0e38f;                               // the reference of a row that has seen no score
constexpr float kLag = 16.f;                                    // how far a score may exceed its reference (values up to 2^128 / 2^16 then stay finite)

// ---- instructions ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int token, int head, int page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(token), "r"(head), "r"(page), "r"(bar)
                 : "memory");
}
// (a warp's lanes come together before what all of them have to execute at once)
template <int T> __device__ __forceinline__ void team_sync(int bar) { __syncwarp(); asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(T) : "memory"); }
template <int T> __device__ __forceinline__ bool team_any(int bar, bool x) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(static_cast<uint32_t>(x)), "r"(bar), "n"(T) : "memory");
    return r != 0;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- layout ------------------------------------------------------------------------------------------------------------

template <int NP, int N>
struct Shape {
    // the softmax's eight warps: teams that take units in turn, of halves that share a unit's rows
    static constexpr int kHalves = N >= 48 ? 2 : 1, kTeams = 2 / kHalves, kColumnsEach = N / kHalves;
    static constexpr int kTeam = 128 * kHalves, kSoft = kTeam * kTeams, kThreads = kSoft + 96;
    static constexpr int kKeys = 8, kValues = 9, kIssuer = 10;           // warps: loads of keys, of values, products
    static constexpr int kPanel = kTile * 128, kSlot = NP * kPanel;      // a slot: NP panels of 128 rows of 64 columns
    static constexpr int kQ = NP * N * 128, kP = N * kTile * 2;
    static constexpr int kRest = (N > 64 ? 4 : 3) * 1024;
    // two buffers for the weights (the next tile's are formed while the last one's are multiplied) where that leaves five slots
    static constexpr int kTwo = (227 * 1024 - kRest - kTeams * kQ - 2 * kP) / kSlot;
    static constexpr int kBuffers = kTwo >= 5 ? 2 : 1;
    static constexpr int kFit = (227 * 1024 - kRest - kTeams * kQ - kBuffers * kP) / kSlot;
    static constexpr int kSlots = kFit < 8 ? kFit : 8;
    static constexpr int kUsed = (2 + kTeams) * N, kColumns = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : 256;      // of tensor memory: S twice, O for each team
    static constexpr int kBytes = kSlots * kSlot + kTeams * kQ + kBuffers * kP + kRest;
    static_assert(kSlots >= 4, "two tiles in flight");
};
// Marks of units (Smem::bad).  While a team has not yet read unit u's, the products may be at the scores of u + 3 (with two teams: each hands in the rows
// of its next unit before it ends one, and scores go a tile ahead), so the keys' warp, which marks a unit when a slot is free for it, at u + 3 + half
// of the slots.
constexpr int kUnits = 8;
// Sees of a unit: positions p0 to p1 are its rows', low0 and low1 the first positions of the first and the last row's windows.
struct View {
    int count, p0, p1, low0, low1;
    int j0, j1, js;            // pages j0 .. j1, and those before js, hold what its rows see
};
template <int NP, int N>
struct __align__(1024) Smem {
    using Sh = Shape<NP, N>;
    char ring[Sh::kSlots][Sh::kSlot];
    char q[Sh::kTeams][Sh::kQ];
    char p[Sh::kBuffers][Sh::kP];
    struct __align__(16) {
        float nref[N], mref[N];                // minus the references (read four at a time): for the first look, and as they are
        float part[4][N];                      // maxima by warp; then in part[0] what the move of the references scales by
        long long off[N];                      // where the rows' results go
        int abort, fix, far;                   // (far: some row's reference is)
        Walk next;                             // the team's next unit, the tiles of the other team's one before it
        View next_view;
        int skipped;
    } team[Sh::kTeams];
    unsigned long long full[8], empty[8], s_full[2], p_full[2], p_done[2], q_full[2], u_start[2], u_done[2], drain;
    ShareSmem share;
    JointSmem joint;
    uint32_t tmem;
    int bad[kUnits];                           // units that name a page that is none
};

__device__ __forceinline__ View view_of(const AttendArgs& a, const Walk& w) {
    View v;
    v.count = w.r0 + a.rows < w.s.rows ? a.rows : w.s.rows - w.r0;
    v.p0 = w.s.base + a.by_group(w.r0);
    v.p1 = w.s.base + a.by_group(w.r0 + v.count - 1);
    v.low0 = low_of(a, v.p0);
    v.low1 = low_of(a, v.p1);
    v.j0 = a.by_page(v.low0);
    v.j1 = v.p1 < 0 ? -1 : a.by_page(v.p1);
    v.js = a.sinks > 0 ? a.by_page(a.sinks - 1) + 1 : 0;
    return v;
}
__device__ __forceinline__ bool any_sees(const AttendArgs& a, const View& v, int p) { return p <= v.p1 && (p >= v.low0 || p < a.sinks); }
__device__ __forceinline__ bool all_see(const AttendArgs& a, const View& v, int p) { return p <= v.p0 && (p >= v.low1 || p < a.sinks); }
__device__ __forceinline__ bool whole_tile(const AttendArgs& a, const View& v, int start, int keys) {
    return start + keys - 1 <= v.p0 && (start >= v.low1 || start + keys <= a.sinks);
}

// The largest of the lanes' values (as integers that are in the order of the values).
__device__ __forceinline__ float warp_max(float x) {
    int i = __float_as_int(x);
    i ^= (i >> 31) & 0x7fffffff;
    i = __reduce_max_sync(0xffffffffu, i);
    i ^= (i >> 31) & 0x7fffffff;
    return __int_as_float(i);
}

// Sums over the lanes of W = 8, 16 or 32 values each: lane x ends up with the sum of value x % W.
template <int W> __device__ __forceinline__ float across(float* v, int lane) {
#pragma unroll
    for (int w = 16; w >= W; w >>= 1) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], w);
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

// ---- the parts of a CTA ------------------------------------------------------------------------------------------------

// Loads: the keys' warp fills the even slots of the ring's order, the values' warp the odd ones.
template <int NP, int N>
__device__ __forceinline__ void load_tiles(const AttendArgs& a, Smem<NP, N>& sm, Walk w, const CUtensorMap* map, int which, uint32_t limit) {
    using Sh = Shape<NP, N>;
    const int lane = threadIdx.x & 31;
    const int boxes = a.per_page > 1 ? 1 : a.span / a.box;               // of a tile
    int x = which, unit = 0;                   // the slot's number in the ring's order
    bool ok = true;
#pragma unroll 1
    for (; w.more && ok; walk_next(a, w), ++unit) {
        const View v = view_of(a, w);
        const int32_t* row = a.table + static_cast<long long>(w.b) * a.width;
        int token = 0;                         // where in its page the lane's box begins
        auto entry = [&](int i) {              // this lane's page of tile i: -1 none to be seen, -2 none at all
            if (i >= w.upto || lane >= boxes) return -1;
            const int p = tile_start(a, tile_at(w.u, i)) + lane * a.box, j = a.by_page(p);
            token = p - j * a.page;
            if (j > v.j1 || (j < v.j0 && j >= v.js)) return -1;
            const int page = __ldg(row + j);
            return page < 0 || page >= a.num_pages ? -2 : page;
        };
        int next = entry(w.i);
#pragma unroll 1
        for (int i = w.i; i < w.upto && ok; ++i, x += 2) {
            const int page = next, at = token;
            next = entry(i + 1);
            const unsigned there = __ballot_sync(0xffffffffu, page >= 0);
            const bool none = __any_sync(0xffffffffu, page == -2);
            const int slot = x % Sh::kSlots;
            ok = __all_sync(0xffffffffu, mbar_wait_now(smem_u32(&sm.empty[slot]), (x / Sh::kSlots & 1) ^ 1, a.status, limit));
            if (!ok) break;
            if (none && lane == 0) sm.bad[unit % kUnits] = 1;        // (behind the wait: see kUnits)
            const uint32_t bar = smem_u32(&sm.full[slot]);
            if (lane == 0) mbar_arrive_expect(bar, __popc(there) * a.box * 128 * NP);
            __syncwarp();
            if (page >= 0) {
#pragma unroll
                for (int p = 0; p < NP; ++p) tma_load(smem_u32(sm.ring[slot]) + p * Sh::kPanel + lane * a.box * 128, map, p * 64, at, w.h, page, bar);
            }
        }
    }
    // (a launch that gave up leaves when its copies are in)
    if (!ok)
        for (int y = x >= Sh::kSlots ? x - Sh::kSlots : which; y < x; ++y)
            if ((y & 1) == which) mbar_wait_now(smem_u32(&sm.full[y % Sh::kSlots]), y / Sh::kSlots & 1, a.status, limit);
}

// The products, by one thread: S of a tile before O of the one before it.
template <int NP, int N>
__device__ __forceinline__ void issue_products(const AttendArgs& a, Smem<NP, N>& sm, Walk w, uint32_t tmem, uint32_t limit) {
    using Sh = Shape<NP, N>;
    constexpr uint32_t qk = instruction(kTile, N, false, false), pv = instruction(64 * NP, N, true, true);
    const uint32_t ring = smem_u32(sm.ring), o_at = tmem + 2 * N;
    bool ok = true;
    auto wait = [&](unsigned long long& bar, int phase) { ok = ok && mbar_wait_now(smem_u32(&bar), phase & 1, a.status, limit); };
    int unit = 0, left = w.more ? w.upto - w.i : 0;      // of the tile whose scores come next
    unsigned starts = 0, ends = 0, teams = 0;  // bit t & 1: tile t is its unit's first, its last, its unit's team
    auto scores = [&](int t) {                 // false: there is no such tile
        const bool first = t == 0 || left == 0;
        if (left == 0) {
            walk_next(a, w);
            if (!w.more) return false;
            left = w.upto - w.i;
            ++unit;
        }
        --left;
        const int team = unit % Sh::kTeams, bit = t & 1;
        if (first) wait(sm.q_full[team], unit / Sh::kTeams);
        auto note = [&](unsigned& bits, bool x) { bits = (bits & ~(1u << bit)) | static_cast<unsigned>(x) << bit; };
        note(starts, first);
        note(ends, left == 0);
        note(teams, team != 0);
        const int slot = 2 * t % Sh::kSlots;
        wait(sm.full[slot], 2 * t / Sh::kSlots);
        if (!ok) return false;
        fence_after();
        const uint32_t k_low = desc_low(ring + slot * Sh::kSlot, 16), q_low = desc_low(smem_u32(sm.q[team]), 16), s_at = tmem + bit * N;
#pragma unroll
        for (int i = 0; i < 4 * NP; ++i)
            mma(s_at, desc(k_low + (i / 4 * Sh::kPanel + i % 4 * 32) / 16, desc_high(1024, 2)), desc(q_low + (i / 4 * N * 128 + i % 4 * 32) / 16, desc_high(1024, 2)), qk, i > 0);
        commit(smem_u32(&sm.empty[slot]));
        if (a.never_signal != 1) {
            // (a team that waits for its turn may be many tiles early, too early to tell by a phase's parity: a unit's first scores are
            // announced by a barrier of the team's own)
            if (first) commit(smem_u32(&sm.u_start[team]));
            commit(smem_u32(&sm.s_full[bit]));
        }
        return true;
    };
    bool have = w.more && scores(0);
#pragma unroll 1
    for (int g = 0; have && ok; ++g) {
        // (with one team the next unit's rows take the place of this one's when its last scores are there: its end does not wait for them)
        const bool later = Sh::kTeams == 1 && left == 0;
        if (!later) have = scores(g + 1);
        const int x = 2 * g + 1, slot = x % Sh::kSlots, buffer = g % Sh::kBuffers, bit = g & 1, team = teams >> bit & 1;
        wait(sm.full[slot], x / Sh::kSlots);
        wait(sm.p_full[buffer], g / Sh::kBuffers);
        if (!ok) break;
        fence_after();
        const uint32_t p_low = desc_low(smem_u32(sm.p[buffer]), 128);
        const uint32_t v_low = desc_low(ring + slot * Sh::kSlot, Sh::kPanel);
        const uint32_t add = !(starts >> bit & 1);
#pragma unroll
        for (int j = 0; j < kTile / 16; ++j) mma(o_at + team * N, desc(v_low + j * 128, desc_high(1024, 2)), desc(p_low + j * 16, desc_high(2048, 0)), pv, add || j > 0);
        commit(smem_u32(&sm.empty[slot]));
        commit(smem_u32(&sm.p_done[buffer]));
        if (ends >> bit & 1) commit(smem_u32(&sm.u_done[team]));
        if (later) have = scores(g + 1);
    }
    if (!ok) {
        commit(smem_u32(&sm.drain));
        mbar_wait_now(smem_u32(&sm.drain), 0, a.status, limit);
    }
}

// A unit's query rows, swizzled like the keys; zero beyond its rows and beyond D.  They are there when the copies are (fetched_queries).
template <int NP, int N, int T>
__device__ __forceinline__ void fetch_queries(const AttendArgs& a, char* to, const Walk& w, int count, int q_vec, int tid) {
    constexpr int per_row = NP * 8, step = T / per_row;
    const int c = tid % per_row;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + w.b * a.qs[0] + w.h * a.group * a.qs[2] + c * 8;
    if (q_vec) {
        const uint32_t dst = smem_u32(to) + c / 8 * (N * 128) + tid / per_row * 128 + ((c % 8) ^ (tid / per_row & 7)) * 16;
        static_assert(step % 8 == 0, "the swizzle of a thread's rows is one");
#pragma unroll
        for (int x = 0; x < N; x += step) {
            const int row = x + tid / per_row, r = w.r0 + row, t = a.by_group(r);
            if (N % step != 0 && row >= N) break;
            if (row < count && c * 8 < a.D)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + x * 128), "l"(src + t * a.qs[1] + (r - t * a.group) * a.qs[2]) : "memory");
            else
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + x * 128), "r"(0) : "memory");
        }
        cp_async_commit();
        return;
    }
#pragma unroll 1
    for (int row = tid / per_row; row < N; row += step) {
        const uint32_t dst = smem_u32(to) + c / 8 * (N * 128) + row * 128 + ((c % 8) ^ (row & 7)) * 16;
        const int r = w.r0 + row, t = a.by_group(r);
        uint4 val = make_uint4(0, 0, 0, 0);
        if (row < count && c * 8 < a.D) {
            const uint16_t* e = reinterpret_cast<const uint16_t*>(src + t * a.qs[1] + (r - t * a.group) * a.qs[2]);
            val = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(val.x), "r"(val.y), "r"(val.z), "r"(val.w) : "memory");
    }
    cp_async_commit();
}
__device__ __forceinline__ void fetched_queries(unsigned long long& bar) {
    cp_async_wait<0>();
    fence_async();
    mbar_arrive(smem_u32(&bar));
}

// A reference differs from the exact product of its score by half of the product's last bit, which from 2^31 on is a hundred and more: the fused product less
// the reference would overflow as a weight's exponent.  So rows of such references (from 2^20 on) are weighed by products that are rounded as the
// reference was.  For the first look they count as rows without one, so that it always finds them.
constexpr float kFar = 1048576.f;
__device__ __forceinline__ bool far(float m) { return fabsf(m) >= kFar && fabsf(m) != -kNone; }

// C columns of k s - m, those outside [lo, hi) at -inf.
template <int C, bool FAR = false> __device__ __forceinline__ void weigh(float* s, const float* nref, float kf, bool masked, int lo, int hi) {
    auto one = [&](float x, float nr) { return FAR && far(nr) ? __fadd_rn(__fmul_rn(x, kf), nr) : fmaf(x, kf, nr); };
#pragma unroll
    for (int c = 0; c < C; c += 4) {
        const float4 nr = *reinterpret_cast<const float4*>(nref + c);
        s[c] = one(s[c], nr.x);
        s[c + 1] = one(s[c + 1], nr.y);
        s[c + 2] = one(s[c + 2], nr.z);
        s[c + 3] = one(s[c + 3], nr.w);
    }
    if (masked) {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c] = c >= lo && c < hi ? s[c] : -INFINITY;
    }
}

template <int NP, int N>
__global__ void __launch_bounds__((Shape<NP, N>::kThreads), 1) attend_tiles_kernel(const AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const int vec) {
    extern __shared__ __align__(1024) char raw[];
    using Sh = Shape<NP, N>;
    Smem<NP, N>& sm = *reinterpret_cast<Smem<NP, N>*>(raw);
    static_assert(sizeof(Smem<NP, N>) <= Sh::kBytes, "the rest fits");
    static_assert(3 + Sh::kSlots / 2 < kUnits, "no two units with one mark");
    constexpr int kSlots = Sh::kSlots, kSoft = Sh::kSoft, C = Sh::kColumnsEach;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t limit = a.wait_limit ? a.wait_limit : 1u << 24;

    if (warp == Sh::kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "n"(Sh::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    } else if (warp == Sh::kKeys && lane == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_u32(&sm.full[i]), 1);
            mbar_init(smem_u32(&sm.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.s_full[i]), 1);
            mbar_init(smem_u32(&sm.p_full[i]), Sh::kTeam);
            mbar_init(smem_u32(&sm.p_done[i]), 1);
            mbar_init(smem_u32(&sm.q_full[i]), Sh::kTeam);
            mbar_init(smem_u32(&sm.u_start[i]), 1);
            mbar_init(smem_u32(&sm.u_done[i]), 1);
        }
        mbar_init(smem_u32(&sm.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < kUnits; ++i) sm.bad[i] = 0;
        for (int i = 0; i < Sh::kTeams; ++i) sm.team[i].abort = sm.team[i].fix = sm.team[i].far = 0;
        sm.joint.n = 0;
    } else if (warp < Sh::kKeys) {
        // (rows of a slot that no page reaches are never written: they stay zero)
        if (a.span < kTile) {
            const int vecs = (kTile - a.span) * 8;
            for (int x = tid; x < kSlots * NP * vecs; x += kSoft) {
                const int panel = x / vecs;
                reinterpret_cast<uint4*>(sm.ring[0] + panel * Sh::kPanel + a.span * 128)[x - panel * vecs] = make_uint4(0, 0, 0, 0);
            }
        }
        fence_async();
    }
    const Share sh = find_share(a, sm.share, Sh::kThreads);
    fence_after();
    const uint32_t tmem = sm.tmem;
    Walk w = walk_begin(a, sh);

    if (warp == Sh::kKeys || warp == Sh::kValues) {
        load_tiles<NP, N>(a, sm, w, warp == Sh::kKeys ? &k_map : &v_map, warp == Sh::kValues, limit);
    } else if (warp == Sh::kIssuer) {
        // (the lane is elected, not chosen by its number, so that the compiler knows that it is one: a fourth less time an instruction)
        uint32_t one;
        asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
        if (one) issue_products<NP, N>(a, sm, w, tmem, limit);
        __syncwarp();
    } else {
        // ---- weights
        // the thread's key, its four warps' rows c0 .. c0 + C - 1
        constexpr int kTeam = Sh::kTeam;
        const int key = tid & (kTile - 1), quarter = warp & 3, team = tid / kTeam, member = tid % kTeam, half = member >> 7, c0 = half * C;
        auto& ts = sm.team[team];
        const int bar = 1 + team;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16, o_at = tmem + lanes + (2 + team) * N + c0;
        // the element of O that this thread has: with 64 of them a warp has 16, in its lower lanes
        const int dim = NP == 2 ? key : quarter * 16 + lane;
        const bool has_dim = dim < a.D && (NP == 2 || lane < 16);
        char* const p_row = sm.p[0] + c0 / 8 * (kTile * 16) + key / 8 * 128 + key % 8 * 16;
        int g = 0, unit = 0;
        // A wait that gives up: this thread asks for a vote from then on, and behind the vote all of them leave together (ts.abort is
        // set before a vote or after the barrier that follows the look at it, never between).
        bool failed = false, gone = false;
        auto wait = [&](unsigned long long& bar, int phase) {            // (by whole warps)
            if (!mbar_wait_now(smem_u32(&bar), phase & 1, a.status, limit)) {
                failed = true;
                atomicExch(&ts.abort, 1);
            }
            __syncwarp();
        };
        auto products = [&](int t) { wait(sm.p_done[t % Sh::kBuffers], t / Sh::kBuffers); };      // until tile t's are done
        // the team's first unit
        View v{};
        for (; unit < team && w.more; ++unit) {
            g += w.upto - w.i;
            walk_next(a, w);
        }
        if (w.more) {
            v = view_of(a, w);
            fetch_queries<NP, N, kTeam>(a, sm.q[team], w, v.count, vec & 1, member);
            fetched_queries(sm.q_full[team]);
        }
#pragma unroll 1
        while (w.more) {
            float l[C];
#pragma unroll
            for (int c = 0; c < C; ++c) l[c] = 0.f;
            if (member < N) {
                const int r = w.r0 + member, t = a.by_group(r);
                ts.off[member] = t * a.os[1] + (r - t * a.group) * a.os[2];
            }
            // one warp looks ahead while the first scores are under way (here it costs nothing, and nobody has to keep the next unit in registers)
            if (member < 32) {
                Walk next = w;
                int skipped = 0;
                walk_next(a, next);
                if (Sh::kTeams > 1 && next.more) {
                    skipped = next.upto - next.i;
                    walk_next(a, next);
                }
                if (lane == 0) {
                    ts.next = next;
                    if (next.more) ts.next_view = next.b == w.b && next.r0 == w.r0 ? v : view_of(a, next);
                    ts.skipped = skipped;
                }
            }
            const int nt = w.upto - w.i;
#pragma unroll 1
            for (int i = 0; i < nt && !gone; ++i, ++g) {
                int start;
                const int keys = tile_keys(a, tile_at(w.u, w.i + i), &start);
                const bool masked = keys < kTile || !whole_tile(a, v, start, keys);
                int lo = 0, hi = N;            // the rows that see this thread's key, from the first of its four warps on
                if (i == 0) wait(sm.u_start[team], unit / Sh::kTeams);
                else wait(sm.s_full[g & 1], g >> 1);
                fence_after();
                const uint32_t s_at = tmem + lanes + (g & 1) * N + c0;
                float s[C];
                if (masked) {
                    const int p = start + key;
                    const bool any = key < keys && any_sees(a, v, p), all = any && all_see(a, v, p);
                    if (!any) {
                        hi = 0;
                    } else if (!all) {
                        // rows are in the order of their positions: from the first token at or beyond p, to the last whose window reaches p
                        const long long first = static_cast<long long>(p - w.s.base) * a.group - w.r0, last = first + static_cast<long long>(a.window) * a.group;
                        lo = first > 0 ? static_cast<int>(first) : 0;
                        if (a.window > 0 && p >= a.sinks && last < N) hi = static_cast<int>(last);
                    }
                    lo -= c0;
                    hi -= c0;
                    // Values: zero where nobody sees them, their finite elements where some do not; the keys before `pre` and from `post` on, by all
                    // threads, a vector at a time.
                    const int pre = a.window > 0 && v.low1 > start ? (v.low1 - start < a.span ? v.low1 - start : a.span) : 0;
                    const int sure = v.p0 + 1 - start < a.span ? v.p0 + 1 - start : a.span, post = sure > pre ? sure : pre;
                    const int items = (pre + a.span - post) * (8 * NP);
                    if (items > 0) wait(sm.full[(2 * g + 1) % kSlots], (2 * g + 1) / kSlots);
                    bool odd = false;
#pragma unroll 1
                    for (int x = member; x < items; x += kTeam) {
                        const int e = x % (8 * NP), y = x / (8 * NP), z = y < pre ? y : y - pre + post, pz = start + z;
                        const bool seen = z < keys && any_sees(a, v, pz);
                        if (seen && all_see(a, v, pz)) continue;
                        uint4* const at = reinterpret_cast<uint4*>(sm.ring[(2 * g + 1) % kSlots] + e / 8 * Sh::kPanel + z * 128 + e % 8 * 16);
                        uint4 val = make_uint4(0, 0, 0, 0);
                        if (seen) {
                            val = *at;
                            auto finite = [&](uint32_t& x) {
                                const uint32_t low = (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, high = (x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                                x &= ~(low | high);
                                odd |= (low | high) != 0;
                            };
                            finite(val.x); finite(val.y); finite(val.z); finite(val.w);
                        }
                        *at = val;
                    }
                    if (odd) ts.fix = 1;
                    __syncwarp();
                }
                load_columns<C>(s_at, s);
#pragma unroll
                for (int c = 0; c < C; c += 8) wait_ld8(s + c);
                if (i == 0) {
                    // a unit's first references are the scores of a key that all its rows see, if one of the tile's two ends is such a key
                    const int ref = all_see(a, v, start) ? 0 : all_see(a, v, start + keys - 1) ? keys - 1 : -1;
                    if (key == ref) {
#pragma unroll
                        for (int c = 0; c < C; c += 4) *reinterpret_cast<float4*>(ts.part[0] + c0 + c) = make_float4(s[c], s[c + 1], s[c + 2], s[c + 3]);
                    }
                    team_sync<kTeam>(bar);
                    if (member < N) {
                        const float m = rintf(ts.part[0][member] * a.kf);
                        ts.nref[member] = ts.mref[member] = ref >= 0 && fabsf(m) < kFar ? -m : -kNone;
                    }
                    team_sync<kTeam>(bar);
                }
                // k s - m, and whether any of them is too large
                weigh<C>(s, ts.nref + c0, a.kf, masked, lo, hi);
                float most = -INFINITY;
#pragma unroll
                for (int c = 0; c < C; ++c) most = fmaxf(most, s[c]);
                if (team_any<kTeam>(bar, most > kLag || failed)) {
#pragma unroll 1
                    for (int c = 0; c < C; c += 8) {
                        float y[8];
                        ld8(s_at + c, y);
                        wait_ld8(y);
                        float mine = -INFINITY;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float x = warp_max(c + e >= lo && c + e < hi ? y[e] * a.kf : -INFINITY);
                            if (lane == e) mine = x;
                        }
                        if (lane < 8) ts.part[quarter][c0 + c + lane] = mine;
                    }
                    team_sync<kTeam>(bar);
                    if (member < N) {
                        const float top = fmaxf(fmaxf(ts.part[0][member], ts.part[1][member]), fmaxf(ts.part[2][member], ts.part[3][member]));
                        const float old = -ts.mref[member];
                        const float now = top - old > kLag ? rintf(top) : old;
                        ts.part[0][member] = now == old ? 1.f : exp2f(old - now);
                        ts.mref[member] = -now;
                        ts.nref[member] = fabsf(now) < kFar ? -now : -kNone;
                        if (far(now)) ts.far = 1;
                    }
                    gone = *static_cast<volatile int*>(&ts.abort) != 0;
                    team_sync<kTeam>(bar);
                    if (gone) break;
                    if (i > 0) {
                        products(g - 1);
                        fence_after();
#pragma unroll 1
                        for (int c = 0; c < C; c += 8) {
                            float o[8];
                            ld8(o_at + c, o);
                            wait_ld8(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] *= ts.part[0][c0 + c + e];
                            st8(o_at + c, o);
                        }
                        wait_st();
#pragma unroll
                        for (int c = 0; c < C; ++c) l[c] *= ts.part[0][c0 + c];
                    }
                    load_columns<C>(s_at, s);
#pragma unroll
                    for (int c = 0; c < C; c += 8) wait_ld8(s + c);
                    if (*static_cast<volatile int*>(&ts.far)) weigh<C, true>(s, ts.mref + c0, a.kf, masked, lo, hi);
                    else weigh<C>(s, ts.mref + c0, a.kf, masked, lo, hi);
                }
                if (g >= Sh::kBuffers) products(g - Sh::kBuffers);       // (the weights that lie there have been multiplied)
                char* const to = p_row + g % Sh::kBuffers * Sh::kP;
#pragma unroll
                for (int c = 0; c < C; c += 8) {
                    uint32_t pk[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(ex2(s[c + 2 * e]), ex2(s[c + 2 * e + 1]));
                        pk[e] = *reinterpret_cast<const uint32_t*>(&h);
                        l[c + 2 * e] += __uint_as_float(pk[e] << 16);
                        l[c + 2 * e + 1] += __uint_as_float(pk[e] & 0xffff0000u);
                    }
                    *reinterpret_cast<uint4*>(to + c / 8 * (kTile * 16)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                }
                fence_async();
                fence_before();
                mbar_arrive(smem_u32(&sm.p_full[g % Sh::kBuffers]));
            }
            // the next unit's rows, now that this one's have their scores
            if (gone) team_sync<kTeam>(bar);   // (no tile was looked at, so nothing lies between ts.next and its readers)
            const Walk next = ts.next;
            const View nv = ts.next_view;
            if (!gone) {
                if (next.more) fetch_queries<NP, N, kTeam>(a, sm.q[team], next, nv.count, vec & 1, member);
                wait(sm.u_done[team], unit / Sh::kTeams);
                if (next.more) fetched_queries(sm.q_full[team]);
            }
            fence_after();
            // the sums: over the lanes, then (in what follows) over the warps
            constexpr int c32 = C / 32 * 32, c16 = (C - c32) / 16 * 16, c8 = C - c32 - c16;
            float* const sums = ts.part[quarter] + c0;
#pragma unroll
            for (int c = 0; c < c32; c += 32) sums[c + lane] = across<32>(l + c, lane);
            if constexpr (c16 > 0) {
                const float x = across<16>(l + c32, lane);
                if (lane < 16) sums[c32 + lane] = x;
            }
            if constexpr (c8 > 0) {
                const float x = across<8>(l + c32 + c16, lane);
                if (lane < 8) sums[c32 + c16 + lane] = x;
            }
            const bool lost = team_any<kTeam>(bar, failed || gone), bad = w.s.bad || *static_cast<volatile int*>(&sm.bad[unit % kUnits]) != 0;
            const bool fix = *static_cast<volatile int*>(&ts.fix) != 0;
            float* part = leave_unit(a, sh, w, v.count, sm.joint, member);
            if (member < N) {
                const float sum = lost || (bad && member < v.count && loses_row(a, w, member)) ? NAN : ts.part[0][member] + ts.part[1][member] + ts.part[2][member] + ts.part[3][member];
                if (part && member < v.count) {
                    part[member] = -ts.mref[member];
                    part[a.rows + member] = sum;
                }
                ts.part[0][member] = sum == 0.f ? of_nothing(a, w.s, w.r0 + member) : 1.f / sum;
            }
            team_sync<kTeam>(bar);
            if (member == 0) ts.fix = ts.far = sm.bad[unit % kUnits] = 0;         // (everybody has read them; the unit's last barrier is still to come)
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + w.b * a.os[0] + w.h * a.group * a.os[2];
            // Eight rows at a time, in a loop: instructions are what this costs, and those of a loop are fetched once.  Two halves put their rows side
            // by side where the weights lay (their products are done), from where they go out in whole vectors.
            constexpr bool kStaged = Sh::kHalves == 2;
            constexpr int kWide = 64 * NP;
            __nv_bfloat16* const stage = reinterpret_cast<__nv_bfloat16*>(sm.p[0]);
            static_assert(!kStaged || N * kWide * 2 <= Sh::kP, "rows in the place of weights");
#pragma unroll 1
            for (int c = 0; c < C && c0 + c < v.count; c += 8) {
                float o[8];
                __syncwarp();
                ld8(o_at + c, o);
                wait_ld8(o);
                if (fix && has_dim) {
                    // what is not finite among the values that some rows see and others do not
#pragma unroll 1
                    for (int i = w.i; i < w.upto; ++i) {
                        int start;
                        const int keys = tile_keys(a, tile_at(w.u, i), &start);
                        if (whole_tile(a, v, start, keys)) continue;
#pragma unroll 1
                        for (int x = 0; x < keys; ++x) {
                            const int p = start + x;
                            if (!any_sees(a, v, p) || all_see(a, v, p)) continue;
                            const int j = a.by_page(p), page = __ldg(a.table + static_cast<long long>(w.b) * a.width + j);
                            if (page < 0 || page >= a.num_pages) continue;
                            const float val = to_float((static_cast<const __nv_bfloat16*>(a.v) + page * a.vs[0] + w.h * a.vs[1] + (p - j * a.page) * a.vs[2])[dim]);
                            if (isfinite(val)) continue;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int pos = w.s.base + a.by_group(w.r0 + c0 + c + e);
                                if (p <= pos && (p >= low_of(a, pos) || p < a.sinks)) o[e] += val;
                            }
                        }
                    }
                }
                const int left = has_dim ? v.count - c0 - c : 0;
                if (part) {
                    float* at = part + 2 * a.rows + (c0 + c) * a.D + dim;
#pragma unroll
                    for (int e = 0; e < 8; ++e, at += a.D)
                        if (e < left) *at = o[e];
                    continue;
                }
                const float4 fa = *reinterpret_cast<const float4*>(ts.part[0] + c0 + c), fb = *reinterpret_cast<const float4*>(ts.part[0] + c0 + c + 4);
                const float f[8] = {fa.x, fa.y, fa.z, fa.w, fb.x, fb.y, fb.z, fb.w};
                if constexpr (kStaged) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (has_dim) stage[(c0 + c + e) * kWide + dim] = __float2bfloat16_rn(o[e] * f[e]);
                } else {
                    long long off[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) off[e] = ts.off[c0 + c + e];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) out[off[e] + dim] = __float2bfloat16_rn(o[e] * f[e]);
                }
            }
            if (kStaged && !part) {
                team_sync<kTeam>(bar);
                constexpr int kPer = 8 * NP;
                const int d = member % kPer * 8;
                if (vec & 2) {
#pragma unroll
                    for (int x = 0; x < N; x += kTeam / kPer) {
                        const int row = x + member / kPer;
                        if (row < v.count && d < a.D) *reinterpret_cast<uint4*>(out + ts.off[row] + d) = *reinterpret_cast<const uint4*>(stage + row * kWide + d);
                    }
                } else {
#pragma unroll 1
                    for (int row = member / kPer; row < v.count; row += kTeam / kPer)
                        for (int e = 0; e < 8 && d < a.D; ++e) out[ts.off[row] + d + e] = stage[row * kWide + d + e];
                }
            }
            const int skipped = ts.skipped;
            fence_before();
            team_sync<kTeam>(bar);
            w = next;
            v = nv;
            g += skipped;
            unit += Sh::kTeams;
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == Sh::kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Sh::kColumns) : "memory");
    join_units<__nv_bfloat16>(a, sm.joint, tid, Sh::kThreads);
}

// ---- launch ------------------------------------------------------------------------------------------------------------

// The map of a pool: columns, tokens of a page, heads, pages; a box is 64 columns (128 bytes) of a page's tokens, at most 128.
bool encode(const AttendArgs& a, const void* pool, const long long* stride, CUtensorMap* map) {
    const Encode fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(a.D), static_cast<cuuint64_t>(a.page), static_cast<cuuint64_t>(a.Hkv), static_cast<cuuint64_t>(a.num_pages)};
    // (the stride of an axis of one is nobody's concern, but has to be one that the map takes)
    cuuint64_t st[3] = {static_cast<cuuint64_t>(stride[2]) * 2, static_cast<cuuint64_t>(a.Hkv > 1 ? stride[1] : a.D) * 2, static_cast<cuuint64_t>(a.num_pages > 1 ? stride[0] : a.D) * 2};
    if (st[0] == 0 || st[1] == 0 || st[2] == 0) return false;        // (heads or pages that are one and the same: not for a map)
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(a.box), 1, 1}, ones[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, st, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NP, int N>
cudaError_t launch(const AttendArgs& a, const CUtensorMap& k, const CUtensorMap& v, int vec, int ctas, cudaStream_t stream) {
    static std::atomic<unsigned long long> asked{0};
    const cudaError_t e = allow_shared(attend_tiles_kernel<NP, N>, Shape<NP, N>::kBytes, asked);
    if (e != cudaSuccess) return e;
    return launch_together(attend_tiles_kernel<NP, N>, ctas, Shape<NP, N>::kThreads, Shape<NP, N>::kBytes, stream, a, k, v, vec);
}
template <int NP>
cudaError_t pick(const AttendArgs& a, const CUtensorMap& k, const CUtensorMap& v, int vec, int ctas, cudaStream_t stream) {
    switch (a.rows) {
        case 16: return launch<NP, 16>(a, k, v, vec, ctas, stream);
        case 32: return launch<NP, 32>(a, k, v, vec, ctas, stream);
        case 48: return launch<NP, 48>(a, k, v, vec, ctas, stream);
        case 64: return launch<NP, 64>(a, k, v, vec, ctas, stream);
        default: return launch<NP, 80>(a, k, v, vec, ctas, stream);
    }
}

}  // namespace

bool attend_tiles_takes(const AttendArgs& a) { return a.D >= 16 && a.D <= 128 && a.D % 8 == 0 && a.page % 8 == 0 && a.page <= (1 << 20); }
void attend_tiles_plan(AttendArgs* a) {
    // the fewest tiles of rows, of sizes as even as multiples of 16 are
    const int rows = a->n * a->group, tiles = (rows + 79) / 80;
    a->rows = ((rows + tiles - 1) / tiles + 15) / 16 * 16;
    // A box is a page, or a tile's share of one; where that leaves an eighth of the tiles' rows empty or more (pages of 48: 96 of 128) tiles go on
    // across the pages, in boxes that divide both.
    a->span = a->page <= kTile ? kTile / a->page * a->page : kTile;
    a->per_page = a->page <= kTile ? 1 : (a->page + kTile - 1) / kTile;
    a->box = a->page < kTile ? a->page : kTile;
    if (8 * (a->per_page > 1 ? a->page : a->span) <= 7 * kTile * a->per_page) {
        a->box = std::gcd(a->page, kTile);
        a->span = kTile;
        a->per_page = 1;
    }
    // A unit's beginning and end: 4.3 us at 72 rows, where a tile takes 1.4; at up to 32 rows, where teams overlap, 1 to 2 us, where a tile
    // takes 0.75 (D = 64) or 1.5.  (128 blocks of 9 tokens over up to 4000 keys with 3, 4, 5: 121, 122, 128 us; 128 of 3 over up to 2000, D = 64,
    // with 1, 2, 3: 54, 48, 47; D = 128 with 1, 2: 64, 66.)
    a->extra = a->rows >= 48 ? 4 : a->D <= 64 ? 2 : 1;
    // A second CTA for a unit costs a join, 2 to 3 us: 4 tiles take 9.7 and 13.6 us (4 and 72 rows) by one CTA, 10.4 and 14.7 by four, 8 tiles
    // 12.8 and 18.6 against 10.8 and 14.3 by eight.
    a->whole = 4;
    a->slack = a->extra;
}
cudaError_t launch_attend_tiles(const AttendArgs& a, bool q_vec, bool out_vec, int ctas, cudaStream_t stream, bool* taken) {
    const int vec = q_vec + 2 * out_vec;
    CUtensorMap k, v;
    *taken = encode(a, a.k, a.ks, &k) && encode(a, a.v, a.vs, &v);
    if (!*taken) return cudaSuccess;
    return a.D <= 64 ? pick<1>(a, k, v, vec, ctas, stream) : pick<2>(a, k, v, vec, ctas, stream);
}

}  // namespace bv
