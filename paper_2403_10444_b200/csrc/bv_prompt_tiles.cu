// Attention of packed prompts in 16 bits on the tensor cores: bv_prompt_attend for bf16, D a multiple of 8 up to 128, rows at 16-byte strides.
//
// A tile has 128 query rows: a key-value head's group of query heads for as many tokens as fit, a token's heads one after the other, so that a
// tile's keys serve the whole group and few keys of its last tiles are seen by some rows only.  A CTA goes through units of two such tiles with the
// same keys, 128 at a time:
//   S [128, 128] = Q K^T     both from shared memory
//   O [128, D]  += P V       P from tensor memory, where it takes the place of S
// and while the tensor cores are at one tile's products the other's scores become weights: 128 threads have a row each, so that maxima, sums and
// masks need no other lane.  References lag by up to 8 powers of two (a row's sums and weights have the range), so O is hardly ever scaled.
//
// One thread issues the products, one the loads (TMA, 128-byte swizzle, a ring of slots that hold 128 keys or values), and two warps look after values
// that some rows of the unit do not see: nobody's are set to 0 in shared memory, others keep their finite elements there, and what is
// not finite is added where it belongs when the unit ends, from global memory.
//
// Units are in the order of their cost, largest first.  The launch has a CTA for each of them, and a CTA that is at work asks for the next one that has not begun
// and does its unit as well (cluster launch control): memory, barriers and the order of the units are made once, loads go on from unit to unit, and no counter
// has to be kept between launches.  Against units handed out forth and back, in turn on one GPU: 3 prompts of 3000 tokens, 16 heads on 2, D = 64: 98 -> 86 us; one of 1200,
// 32 on 8, D = 128: 47 -> 45; 16 of up to 2048: 325 -> 319; one of 32768 as it was.  Dearest where half of the
// CTAs find no unit: 1000 prompts of 64 tokens, 32 heads on 8: 415 -> 421.
//
// One prompt of 32768 tokens, 32 heads on 8, D = 128: 8.6 ms, 1.02 PFLOP/s (7.3 to 7.9 ms, up to 1.2 PFLOP/s, a few calls after a pause); 16 prompts of up to 2048: 345 us,
// 655 TFLOP/s (319 us a few calls after a pause).  A key tile of both tiles of rows takes 3700 clocks (2048 of products): 1800 in which a row's 128 scores become weights, some ten instructions each
// by one warp a scheduler, 600 for reading them and their maximum, 1200 until the next scores are there.  Short prompts: the 16 above have 102 such steps an SM, two thirds of
// their time; the rest is units' first tiles and results, which the next unit's weights wait for.
// Measured and not kept: tiles of 64 keys with two S each, so that scores run ahead (products of 64 columns take as long as those of 128: 9.6 ms); a quarter of the
// exponentials on the FMA pipe (more instructions: 8.8 ms, 361 us); warps that share a scheduler taking turns at exponentials (8.7 against 7.3 ms); one signal a
// tile instead of two (8.95 ms); sums of weights before their rounding (7.9 against 7.6 ms, and less exact); two
// threads a row, 16 warps at the softmax (88 registers a thread are too few: 21 ms, 714 us).
#include "bv_launch.h"
#include "bv_prompt.cuh"
#include "bv_tensor.cuh"

namespace bv {
namespace {

constexpr int kTile = 128;
constexpr int kPromptThreads = 384, kSoftWarps = 8, kIssueWarp = 8, kLoadWarp = 9, kCleanWarp = 10, kCleaners = 64;
constexpr float kNone = -3.0e38f;              // the reference of a row that has seen no score
constexpr float kLag = 8.f;
constexpr int kFirstKeys = 96;                 // of a tile, whose weights are multiplied while the others are formed
constexpr int kMostPrompts = 1024;             // of a launch
constexpr int kTold = 4;                       // units that the loading thread may be ahead of who is last to hear of them
// Marks of units: who is last to hear of units may still be at unit r (the second tile's weights, where later units have no such tile) when unit r + kTold is
// told and the cleaning warps clear its mark.
constexpr int kUnits = kTold + 1;

// Asks for a CTA of the launch that has not begun, whose work this one then does; the answer is 16 bytes, signalled at bar.
__device__ __forceinline__ void ask(uint32_t answer, uint32_t bar) {
    fence_async();                             // (the last answer has been read)
    mbar_arrive_expect(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
// Its index, or -1.
__device__ __forceinline__ int answered(uint32_t answer) {
    uint32_t got, x = 0;
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t.reg .b32 y, z, w;\n\tld.shared.b128 h, [%2];\n\tclusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, h;\n\t}"
                 : "=r"(got), "+r"(x)
                 : "r"(answer)
                 : "memory");
    return got ? static_cast<int>(x) : -1;
}

__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap* map, int x, int head, int token, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(head),
                 "r"(token), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void ld32(uint32_t addr, float* x) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
                 "%26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void st32(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
                 "%26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
                 "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
                 "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}

__device__ __forceinline__ void st16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

template <int NP>
struct PromptShape {
    static constexpr int kPanel = kTile * 128, kSlot = NP * kPanel;        // a slot: NP panels of 128 rows of 64 columns
    static constexpr int kRest = 16 * 1024;
    static constexpr int kFit = (227 * 1024 - kRest - 2 * kSlot) / kSlot;
    static constexpr int kSlots = kFit < 8 ? kFit : 8;
    static constexpr int kBytes = (2 + kSlots) * kSlot + kRest;
    static_assert(kSlots >= 4, "two tiles of keys and values");
};
template <int NP>
struct __align__(1024) PromptSmem {
    using Sh = PromptShape<NP>;
    char q[2][Sh::kSlot];
    char ring[Sh::kSlots][Sh::kSlot];
    ulonglong2 answer;                     // to the request for a unit that has not begun
    unsigned long long asked, told[kTold], heard[kTold];
    int next[kTold];                       // units after the first one, by their places in the CTA's order; -1: none
    unsigned long long q_full[2], q_empty[2], full[8], empty[8], unclean[8], s_full[2], s_read[2], p_part[2], p_full[2], o_done[2], drain;
    uint32_t tmem;
    int abort;
    int fix[kUnits][2];                    // by unit, by cleaning warp: values that are not finite among those that some rows see
    int sequences, units;                  // with rows; pairs of tiles of one head
    unsigned long long order[kMostPrompts];            // pairs of tiles, and which sequence, most first
    int before[kMostPrompts];              // pairs that come before the levels at which a sequence is the last
};

// Unit u of the launch: a pair of tiles of a sequence's key-value head.
struct Pair {
    int b, h, first, length;               // the sequence's first row and its rows
    int t0;                                // the first tile's first token
    int p1;                                // the last token of both tiles
    int low;                               // where the window of the first row begins
    int tiles[2];                          // of keys, that each of the two goes through: the first has the beginning of the list
    int sink_tiles, jump;                  // tiles 0 .. sink_tiles - 1 of the list are the sinks', the others begin with tile `jump`
};
__device__ __forceinline__ int key_tile(const Pair& p, int i) { return i < p.sink_tiles ? i : i - p.sink_tiles + p.jump; }

template <int NP>
__device__ __forceinline__ bool pair_at(const PromptArgs& a, const PromptSmem<NP>& sm, int tokens_each, int base, int u, Pair* p) {
    if (u < 0 || u >= static_cast<long long>(sm.units) * a.Hkv) return false;
    const int x = u / a.Hkv;
    p->h = u - x * a.Hkv;
    // the levels at which sequences 0 .. j have pairs: from the longest's down to one above the next one's
    int lo = 0, hi = sm.sequences;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (sm.before[mid] <= x) lo = mid;
        else hi = mid;
    }
    const int y = x - sm.before[lo], down = y / (lo + 1), s = y - down * (lo + 1);
    const int level = static_cast<int>(sm.order[lo] >> 32) - 1 - down;
    if (level < 0) return false;           // (offsets in no order may be more rows than are counted)
    p->b = base + static_cast<int>(0xffffffffu - static_cast<unsigned>(sm.order[s]));
    const Prompt seq = prompt_of(a, p->b);
    p->first = seq.first;
    p->length = seq.length;
    p->t0 = level * 2 * tokens_each;
    if (p->t0 >= seq.length) return false;
    const int last0 = (p->t0 + tokens_each < seq.length ? p->t0 + tokens_each : seq.length) - 1;
    p->p1 = (p->t0 + 2 * tokens_each < seq.length ? p->t0 + 2 * tokens_each : seq.length) - 1;
    p->low = low_of(a, p->t0);
    // the list: tiles that hold sinks and lie before the first row's window, then from that window on
    p->jump = p->low / kTile;
    const int sinks = a.window > 0 ? (a.sinks + kTile - 1) / kTile : 0;
    p->sink_tiles = sinks < p->jump ? sinks : p->jump;
    const int count0 = last0 / kTile - p->jump + 1 + p->sink_tiles;
    p->tiles[0] = count0;
    p->tiles[1] = p->t0 + tokens_each < seq.length ? p->p1 / kTile - p->jump + 1 + p->sink_tiles : 0;
    return true;
}
__device__ __forceinline__ int list_length(const Pair& p) { return p.tiles[1] > p.tiles[0] ? p.tiles[1] : p.tiles[0]; }
// Do tokens p0 .. p1 see all of tile j?
__device__ __forceinline__ bool whole_tile(const PromptArgs& a, int p0, int p1, int j) {
    const int start = j * kTile;
    return start + kTile - 1 <= p0 && (start >= low_of(a, p1) || start + kTile <= a.sinks);
}

// The lowest n bits.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1; }

// 2 floats at a time.
__device__ __forceinline__ unsigned long long pair2(float x, float y) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpair2(unsigned long long r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// A wait by one thread or by a whole warp that gives up when another has.
template <int NP> __device__ __forceinline__ bool wait_on(PromptSmem<NP>& sm, unsigned long long& bar, int parity, int* status, uint32_t limit) {
    const uint32_t at = smem_u32(&bar);
    for (uint32_t spins = 0; !mbar_try_wait_now(at, parity & 1); ++spins) {
        if ((spins & 255) == 255 && *static_cast<volatile int*>(&sm.abort)) return false;
        if (spins > limit) {
            atomicExch(&sm.abort, 1);
            if (status) atomicExch(status, 1);
            return false;
        }
    }
    return true;
}

// The CTA's next unit, for one thread or a whole warp that is not the loading one: the first is the CTA's own, of the others that thread tells.
template <int NP, bool WARP>
__device__ __forceinline__ bool next_pair(const PromptArgs& a, PromptSmem<NP>& sm, int tokens_each, int base, int round, uint32_t limit, Pair* p) {
    int u = static_cast<int>(blockIdx.x);
    if (round > 0) {
        const int slot = (round - 1) % kTold;
        bool ok = wait_on<NP>(sm, sm.told[slot], (round - 1) / kTold, a.status, limit);
        if (WARP) ok = __all_sync(0xffffffffu, ok);
        if (!ok) return false;
        u = *static_cast<volatile int*>(&sm.next[slot]);
        if (WARP) __syncwarp();
        if (!WARP || (threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sm.heard[slot]));
    }
    return pair_at<NP>(a, sm, tokens_each, base, u, p);
}

template <int NP>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_tiles_kernel(const PromptArgs a, const int base, const int sequences, const __grid_constant__ CUtensorMap q_map,
                                                                         const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const int tokens_each,
                                                                         const int out_vec) {
    extern __shared__ __align__(1024) char raw[];
    using Sh = PromptShape<NP>;
    PromptSmem<NP>& sm = *reinterpret_cast<PromptSmem<NP>*>(raw);
    static_assert(sizeof(PromptSmem<NP>) <= Sh::kBytes, "the rest fits");
    constexpr int kSlots = Sh::kSlots;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t limit = a.wait_limit ? a.wait_limit : 1u << 24;

    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    } else if (warp == kLoadWarp && lane == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.q_full[i]), 1);
            mbar_init(smem_u32(&sm.s_full[i]), 1);
            mbar_init(smem_u32(&sm.s_read[i]), kTile);
            mbar_init(smem_u32(&sm.p_part[i]), kTile);
            mbar_init(smem_u32(&sm.p_full[i]), kTile);
            mbar_init(smem_u32(&sm.q_empty[i]), 1);
            mbar_init(smem_u32(&sm.o_done[i]), 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_u32(&sm.full[i]), 2);
            mbar_init(smem_u32(&sm.empty[i]), 1);
            mbar_init(smem_u32(&sm.unclean[i]), 1);
        }
        mbar_init(smem_u32(&sm.drain), 1);
        mbar_init(smem_u32(&sm.asked), 1);
        for (int i = 0; i < kTold; ++i) {
            mbar_init(smem_u32(&sm.told[i]), 1);
            mbar_init(smem_u32(&sm.heard[i]), kSoftWarps + 3);      // (the issuing thread, two warps that clean)
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.abort = 0;
    }
    // ---- the order of the work: sequences by how many pairs of tiles they have ----
    {
        int size = 1;
        while (size < sequences) size *= 2;
        for (int i = tid; i < size; i += kPromptThreads) {
            const int length = i < sequences ? prompt_of(a, base + i).length : 0;
            const unsigned pairs = static_cast<unsigned>((length + 2 * tokens_each - 1) / (2 * tokens_each));
            // (the lower index first among equals: the same order in every CTA)
            sm.order[i] = static_cast<unsigned long long>(pairs) << 32 | (0xffffffffu - static_cast<unsigned>(i));
        }
        __syncthreads();
        for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                for (int i = tid; i < size; i += kPromptThreads) {
                    const int o = i ^ j;
                    if (o > i) {
                        const unsigned long long x = sm.order[i], y = sm.order[o];
                        if ((x < y) == ((i & k) == 0)) { sm.order[i] = y; sm.order[o] = x; }
                    }
                }
                __syncthreads();
            }
        // pairs before the levels where sequence j is the last: sum over i < j of (i + 1) (n_i - n_{i+1}) = sum over i < j of n_i less j n_j
        if (warp == 0) {
            int sum = 0, live = 0;
            for (int i0 = 0; i0 < sequences; i0 += 32) {
                const int n = i0 + lane < sequences ? static_cast<int>(sm.order[i0 + lane] >> 32) : 0;
                int inc = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += x;
                }
                if (i0 + lane < sequences) sm.before[i0 + lane] = sum + inc - n - (i0 + lane) * n;
                sum += __shfl_sync(0xffffffffu, inc, 31);
                live += __popc(__ballot_sync(0xffffffffu, n > 0));
            }
            if (lane == 0) { sm.units = sum; sm.sequences = live; }
        }
        __syncthreads();
    }
    fence_after();
    const uint32_t tmem = sm.tmem;
    // Columns of tensor memory: S of both tiles, O of both, P of both, which has a place of its own where O is 64 columns wide (kOwn): there the next scores
    // can be formed as soon as the last ones have been read, and nobody waits for them (8 prompts of up to 8192 tokens with a window of 1024, D = 64: 434 -> 410 us).
    constexpr bool kOwn = NP == 1;
    constexpr uint32_t kS = 0, kO = 256, kOStep = NP * 64, kP = kOwn ? kO + 2 * kOStep : kS, kPStep = kOwn ? 64 : kTile;
    Pair p;

    if (warp >= kSoftWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == kLoadWarp) {
            if (lane == 0) {
                const uint32_t q_bytes = static_cast<uint32_t>(tokens_each) * a.group * 128 * NP;
                int x = 0, round = 0, q_uses[2] = {0, 0};
                unsigned unclean = 0, phases = 0;      // by slot: does its last copy go through the cleaning warps, how many have (parity)
                bool ok = true;
                int answers = 0;
                auto answer = [&] {
                    const uint32_t bar = smem_u32(&sm.asked), phase = answers++ & 1;
                    if (mbar_wait_now(bar, phase, a.status, limit)) return answered(smem_u32(&sm.answer));
                    // (given up: all others do too, and the answer is waited for once more, so that it does not come when the CTA has gone)
                    ok = false;
                    atomicExch(&sm.abort, 1);
                    return mbar_wait_now(bar, phase, a.status, limit) ? answered(smem_u32(&sm.answer)) : -1;
                };
                bool more = pair_at<NP>(a, sm, tokens_each, base, static_cast<int>(blockIdx.x), &p);
                for (; ok && more; ++round) {
                    const int tiles = list_length(p);
                    auto fetch = [&](int i) {
                        const int slot = x % kSlots;
                        ok = ok && wait_on<NP>(sm, sm.empty[slot], (x / kSlots & 1) ^ 1, a.status, limit);
                        if (!ok) return;
                        // values that some rows do not see are handed on by the cleaning warps
                        const bool through = (i & 1) && !whole_tile(a, p.t0, p.p1, key_tile(p, i / 2));
                        const uint32_t bar = smem_u32(through ? &sm.unclean[slot] : &sm.full[slot]);
                        mbar_arrive_expect(bar, Sh::kSlot);
                        if (!through) mbar_arrive(bar);
                        unclean = (unclean & ~(1u << slot)) | static_cast<unsigned>(through) << slot;
                        phases ^= static_cast<unsigned>(through) << slot;
                        const CUtensorMap* map = i & 1 ? &v_map : &k_map;
#pragma unroll
                        for (int c = 0; c < NP; ++c) tma_load3(smem_u32(sm.ring[slot]) + c * Sh::kPanel, map, c * 64, p.h, p.first + key_tile(p, i / 2) * kTile, bar);
                        ++x;
                    };
                    // (the first keys need not wait until the unit before has its last scores, as the queries do)
                    fetch(0);
                    for (int t = 0; t < (p.tiles[1] ? 2 : 1) && ok; ++t) {
                        ok = wait_on<NP>(sm, sm.q_empty[t], (q_uses[t] & 1) ^ 1, a.status, limit);
                        if (!ok) break;
                        const uint32_t bar = smem_u32(&sm.q_full[t]);
                        mbar_arrive_expect(bar, q_bytes);
                        ++q_uses[t];
#pragma unroll
                        for (int c = 0; c < NP; ++c) tma_load3(smem_u32(sm.q[t]) + c * Sh::kPanel, &q_map, c * 64, p.h * a.group, p.first + p.t0 + t * tokens_each, bar);
                    }
                    for (int i = 1; i < 2 * tiles - 1 && ok; ++i) fetch(i);
                    // (not before: who asks early gets the larger unit, whoever is free first: one prompt of 2000 tokens took 78 us for 63)
                    ask(smem_u32(&sm.answer), smem_u32(&sm.asked));
                    if (ok) fetch(2 * tiles - 1);
                    // (there may be more CTAs than units; after a no there is no other request)
                    auto another = [&] {
                        ask(smem_u32(&sm.answer), smem_u32(&sm.asked));
                        return answer();
                    };
                    int u = answer();
                    while (ok && u >= 0 && !pair_at<NP>(a, sm, tokens_each, base, u, &p)) u = another();
                    more = u >= 0;
                    const int slot = round % kTold;
                    ok = ok && wait_on<NP>(sm, sm.heard[slot], (round / kTold & 1) ^ 1, a.status, limit);
                    if (ok) {
                        *static_cast<volatile int*>(&sm.next[slot]) = u;
                        mbar_arrive(smem_u32(&sm.told[slot]));
                    }
                    // (a launch that gave up takes all that has not begun with it)
                    while (!ok && u >= 0) u = another();
                }
                // (a launch that gave up leaves when its copies are in)
                if (*static_cast<volatile int*>(&sm.abort)) {
                    for (int y = x > kSlots ? x - kSlots : 0; y < x; ++y) {
                        const int slot = y % kSlots;
                        if (unclean >> slot & 1) mbar_wait_now(smem_u32(&sm.unclean[slot]), (phases >> slot & 1) ^ 1, a.status, limit);
                        else mbar_wait_now(smem_u32(&sm.full[slot]), y / kSlots & 1, a.status, limit);
                    }
                    for (int t = 0; t < 2; ++t)
                        if (q_uses[t]) mbar_wait_now(smem_u32(&sm.q_full[t]), (q_uses[t] - 1) & 1, a.status, limit);
                }
            }
            __syncwarp();
        } else if (warp == kIssueWarp) {
            uint32_t one;
            asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
            if (one) {
                const uint32_t ring = smem_u32(sm.ring), wide = static_cast<uint32_t>((a.D + 15) / 16 * 16);
                constexpr uint32_t qk = instruction(kTile, kTile, false, false);
                const uint32_t pv = instruction(kTile, static_cast<int>(wide), false, true);
                const int steps = static_cast<int>(wide) / 16;
                int x = 0, round = 0, done[2] = {0, 0}, q_uses[2] = {0, 0};      // slots used; tiles done by each of the two
                bool ok = true;
                auto wait = [&](unsigned long long& bar, int parity) { ok = ok && wait_on<NP>(sm, bar, parity, a.status, limit); };
                for (; ok && next_pair<NP, false>(a, sm, tokens_each, base, round, limit, &p); ++round) {
                    const int tiles = list_length(p);
                    // scores of tile i of the list for tile t of the pair
                    auto scores = [&](int t, int i) {
                        const int slot = (x + 2 * i) % kSlots;
                        const uint32_t k_low = desc_low(ring + slot * Sh::kSlot, 16), q_low = desc_low(smem_u32(sm.q[t]), 16);
#pragma unroll
                        for (int s = 0; s < 4 * NP; ++s)
                            if (s < steps)
                                mma(tmem + kS + t * kTile, desc(q_low + (s / 4 * Sh::kPanel + s % 4 * 32) / 16, desc_high(1024, 2)),
                                    desc(k_low + (s / 4 * Sh::kPanel + s % 4 * 32) / 16, desc_high(1024, 2)), qk, s > 0);
                        if (a.never_signal != 1) commit(smem_u32(&sm.s_full[t]));
                        if (i + 1 == p.tiles[t]) commit(smem_u32(&sm.q_empty[t]));
                    };
                    wait(sm.full[x % kSlots], x / kSlots);
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (p.tiles[t] == 0) continue;
                        wait(sm.q_full[t], q_uses[t]++);
                        if (!ok) break;
                        fence_after();
                        scores(t, 0);
                    }
                    if (!ok) break;
                    commit(smem_u32(&sm.empty[x % kSlots]));
                    for (int i = 0; i < tiles && ok; ++i) {
                        const int v_at = x + 2 * i + 1, v_slot = v_at % kSlots, k_at = v_at + 1;
                        bool next_in = false;
                        auto next = [&](int t) {       // the scores of tile i + 1
                            if (i + 1 >= p.tiles[t]) return;
                            if (!next_in) wait(sm.full[k_at % kSlots], k_at / kSlots);
                            next_in = true;
                            if (kOwn) wait(sm.s_read[t], done[t]);
                            if (!ok) return;
                            fence_after();
                            scores(t, i + 1);
                        };
                        if constexpr (kOwn) {
                            for (int t = 0; t < 2; ++t) next(t);
                            if (!ok) break;
                            if (i + 1 < tiles) commit(smem_u32(&sm.empty[k_at % kSlots]));
                        }
                        wait(sm.full[v_slot], v_at / kSlots);
                        for (int t = 0; t < 2 && ok; ++t) {
                            if (i >= p.tiles[t]) continue;
                            const uint32_t v_low = desc_low(ring + v_slot * Sh::kSlot, Sh::kPanel);
                            auto products = [&](int from, int to) {
                                fence_after();
#pragma unroll
                                for (int s = 0; s < kTile / 16; ++s)
                                    if (s >= from && s < to)
                                        mma_ts(tmem + kO + t * kOStep, tmem + kP + t * kPStep + s * 8, desc(v_low + s * 128, desc_high(1024, 2)), pv, i > 0 || s > 0);
                            };
                            wait(sm.p_part[t], done[t]);
                            if (!ok) break;
                            products(0, kFirstKeys / 16);
                            wait(sm.p_full[t], done[t]);
                            if (!ok) break;
                            products(kFirstKeys / 16, kTile / 16);
                            commit(smem_u32(&sm.o_done[t]));
                            if (!kOwn) next(t);
                            if (kOwn && i + 1 == p.tiles[t]) wait(sm.s_read[t], done[t]);      // (every phase is waited for)
                            ++done[t];
                        }
                        if (!ok) break;
                        commit(smem_u32(&sm.empty[v_slot]));
                        if (!kOwn && i + 1 < tiles) commit(smem_u32(&sm.empty[k_at % kSlots]));
                    }
                    x += 2 * tiles;
                }
                if (!ok) {
                    commit(smem_u32(&sm.drain));
                    mbar_wait_now(smem_u32(&sm.drain), 0, a.status, limit);
                }
            }
            __syncwarp();
        } else {
            // ---- values that some row does not see ----
            const int member = tid - kCleanWarp * 32;
            int x = 0;
            unsigned phases = 0;
            bool ok = true;
            for (int round = 0; ok && next_pair<NP, true>(a, sm, tokens_each, base, round, limit, &p); ++round) {
                const int tiles = list_length(p), low1 = low_of(a, p.p1);
                if (lane == 0) sm.fix[round % kUnits][member >> 5] = 0;
                __syncwarp();
                for (int i = 0; i < tiles && ok; ++i) {
                    const int j = key_tile(p, i), start = j * kTile, at = x + 2 * i + 1, slot = at % kSlots;
                    if (whole_tile(a, p.t0, p.p1, j)) continue;
                    ok = __all_sync(0xffffffffu, wait_on<NP>(sm, sm.unclean[slot], phases >> slot & 1, a.status, limit));
                    if (!ok) break;
                    phases ^= 1u << slot;
                    bool odd = false;
                    // the keys before the last row's window, and those behind the first row
                    const int pre = a.window > 0 && low1 > start ? (low1 - start < kTile ? low1 - start : kTile) : 0;
                    const int sure = p.t0 + 1 - start < kTile ? p.t0 + 1 - start : kTile, post = sure > pre ? sure : pre;
                    // (four vectors on their way together: one after the other a tile's took 4000 clocks, which its products wait for)
                    constexpr int kBatch = 4;
                    const int items = (pre + kTile - post) * 8 * NP;
                    for (int z0 = member; z0 < items; z0 += kBatch * kCleaners) {
                        uint4 val[kBatch];
                        uint4* to[kBatch];
                        bool any[kBatch], some[kBatch];      // some row sees it; not all do
#pragma unroll
                        for (int u = 0; u < kBatch; ++u) {
                            const int z = z0 + u * kCleaners, e = z % (8 * NP), y = z / (8 * NP), r = y < pre ? y : y - pre + post, pos = start + r;
                            any[u] = pos <= p.p1 && (pos >= p.low || pos < a.sinks);
                            some[u] = z < items && !(any[u] && pos <= p.t0 && (pos >= low1 || pos < a.sinks));
                            to[u] = reinterpret_cast<uint4*>(sm.ring[slot] + e / 8 * Sh::kPanel + r * 128 + e % 8 * 16);
                            val[u] = make_uint4(0, 0, 0, 0);
                            if (some[u] && any[u]) val[u] = *to[u];
                        }
#pragma unroll
                        for (int u = 0; u < kBatch; ++u) {
                            // (exponents of ones carry into the sign's place)
                            auto ones = [](uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };
                            const bool here = (ones(val[u].x) | ones(val[u].y) | ones(val[u].z) | ones(val[u].w)) != 0;
                            if (here) {
                                auto finite = [&](uint32_t& w) {
                                    const uint32_t x = ones(w);
                                    w &= ~((x & 0x8000u ? 0xffffu : 0u) | (x & 0x80000000u ? 0xffff0000u : 0u));
                                };
                                finite(val[u].x); finite(val[u].y); finite(val[u].z); finite(val[u].w);
                                odd = true;
                            }
                            if (some[u] && (here || !any[u])) *to[u] = val[u];
                        }
                    }
                    if (odd) sm.fix[round % kUnits][member >> 5] = 1;
                    fence_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sm.full[slot]));
                }
                x += 2 * tiles;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ---- weights: a thread has a row ----
        const int t = warp >> 2, row = tid & (kTile - 1);
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16, s_at = tmem + lanes + kS + t * kTile, o_at = tmem + lanes + kO + t * kOStep, p_at = tmem + lanes + kP + t * kPStep;
        const int rows = tokens_each * a.group, token = a.by_group(row), head = row - token * a.group;
        const int wide = (a.D + 15) / 16 * 16;
        int done = 0;
        bool ok = true;
        for (int round = 0; next_pair<NP, true>(a, sm, tokens_each, base, round, limit, &p); ++round) {
            const int tiles = p.tiles[t];
            if (tiles == 0) continue;
            const int p0 = p.t0 + t * tokens_each, pos = p0 + token;
            const int last = p0 + tokens_each - 1 < p.length - 1 ? p0 + tokens_each - 1 : p.length - 1;
            const bool live = row < rows && pos < p.length;
            const int low = low_of(a, pos);
            float m = kNone, l = 0.f;
            for (int i = 0; i < tiles; ++i, ++done) {
                const int j = key_tile(p, i), start = j * kTile;
                ok = __all_sync(0xffffffffu, wait_on<NP>(sm, sm.s_full[t], done, a.status, limit));
                if (!ok) break;
                fence_after();
                float s[kTile];
#pragma unroll
                for (int c = 0; c < kTile; c += 32) ld32(s_at + c, s + c);
#pragma unroll
                for (int c = 0; c < kTile; c += 8) wait_ld8(s + c);
                if (kOwn) {
                    fence_before();
                    mbar_arrive(smem_u32(&sm.s_read[t]));
                }
                if (!whole_tile(a, p0, last, j)) {
                    // seen: c <= hi and (c >= lo or c < sinks); a bit a key
                    const int hi = pos - start, lo = low - start, sinks = a.sinks - start;
#pragma unroll
                    for (int w = 0; w < kTile; w += 32) {
                        const uint32_t seen = below(hi + 1 - w) & (~below(lo - w) | below(sinks - w));
#pragma unroll
                        for (int c = 0; c < 32; ++c) s[w + c] = seen >> c & 1 ? s[w + c] : -INFINITY;
                    }
                }
                float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int c = 4; c < kTile; c += 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[e] = fmaxf(top[e], s[c + e]);
                }
                // (a row that is nobody's holds another prompt's queries, or what an earlier unit left: it has no reference, and no say in what its warp does)
                const float most = live ? __fmul_rn(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), a.kf) : -INFINITY;
                // (a row without a reference takes the first it can have)
                const bool need = most > m + kLag || (m == kNone && most > -INFINITY);
                if (__any_sync(0xffffffffu, need)) {
                    const float now = need ? most : m;
                    if (i > 0) {
                        const float f = need && m != kNone ? ex2(m - now) : 1.f;
                        l *= f;
                        ok = __all_sync(0xffffffffu, wait_on<NP>(sm, sm.o_done[t], done - 1, a.status, limit));
                        if (!ok) break;
                        fence_after();
#pragma unroll 1
                        for (int c = 0; c < wide; c += 16) {
                            float o[16];
                            ld16(o_at + c, o);
                            wait_ld8(o);
                            wait_ld8(o + 8);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= f;
                            st8(o_at + c, o);
                            st8(o_at + c + 8, o + 8);
                        }
                        wait_st();
                    }
                    m = now;
                }
                const float ref = m == kNone ? 0.f : m;
                // From 2^20 on the fused difference is off by too much of a power of two: rows of such references are weighed by products that are
                // rounded as the reference was.
                if (__any_sync(0xffffffffu, fabsf(ref) >= 1048576.f)) {
#pragma unroll
                    for (int c = 0; c < kTile; ++c) s[c] = __fsub_rn(__fmul_rn(s[c], a.kf), ref);
                } else {
                    const unsigned long long kf2 = pair2(a.kf, a.kf), ref2 = pair2(-ref, -ref);
#pragma unroll
                    for (int c = 0; c < kTile; c += 2) unpair2(fma2(pair2(s[c], s[c + 1]), kf2, ref2), s[c], s[c + 1]);
                }
                // (the last weights have been multiplied: theirs is the place of these)
                if (kOwn && done > 0) {
                    ok = __all_sync(0xffffffffu, wait_on<NP>(sm, sm.o_done[t], done - 1, a.status, limit));
                    if (!ok) break;
                    fence_after();
                }
                uint32_t w[kTile / 2];
                unsigned long long sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < kTile; c += 2) {
                    const float x = ex2(s[c]), y = ex2(s[c + 1]);
                    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
                    w[c / 2] = *reinterpret_cast<const uint32_t*>(&h);
                    // The weights' one rounding, to 16 bits: the tensor cores multiply bf16 values by bf16 alone.  A row's error becomes 0.0017 to 0.0021 with it where its
                    // result's own rounding is 0.0016; the rest of a weight as a second operand would make half as many products again (2048 of a step's 3700 clocks).
                    // (the sum is of the rounded weights: error of a row 0.0022 against 0.0023 with the others; a row of one key is its value)
                    sum[c / 2 & 1] = add2(sum[c / 2 & 1], pair2(__uint_as_float(w[c / 2] << 16), __uint_as_float(w[c / 2] & 0xffff0000u)));
                    if (c == 62) st32(p_at, w);
                    if (c == kFirstKeys - 2) {
                        st16(p_at + 32, w + 32);
                        wait_st();
                        fence_before();
                        mbar_arrive(smem_u32(&sm.p_part[t]));
                    }
                }
                st16(p_at + 48, w + 48);
                float x, y;
                unpair2(add2(sum[0], sum[1]), x, y);
                l += x + y;
                wait_st();
                fence_before();
                mbar_arrive(smem_u32(&sm.p_full[t]));
            }
            if (!ok) break;
            ok = __all_sync(0xffffffffu, wait_on<NP>(sm, sm.o_done[t], done - 1, a.status, limit));
            if (!ok) break;
            fence_after();
            const bool fix = (*static_cast<volatile int*>(&sm.fix[round % kUnits][0]) | *static_cast<volatile int*>(&sm.fix[round % kUnits][1])) != 0;
            const float f = l == 0.f ? NAN : 1.f / l;
            __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(a.out) + (p.first + static_cast<long long>(pos)) * a.os[0] + (p.h * a.group + head) * a.os[1];
            // 32 columns at a time.  A lane has a row's 64 bytes; four lanes exchange them, so that a store of the warp is eight rows' whole sectors instead of
            // 16 bytes of each of 32 (which were four times the time).
            const long long out_at = reinterpret_cast<long long>(out);
            const bool some = __any_sync(0xffffffffu, live);
#pragma unroll 1
            for (int c = 0; c < wide && some; c += 32) {
                float o[32];
                __syncwarp();
                if (c + 16 < wide) {
                    ld32(o_at + c, o);
                } else {
                    ld16(o_at + c, o);
                }
#pragma unroll
                for (int e = 0; e < 32; e += 8) wait_ld8(o + e);
                if (fix && live) {
                    // what is not finite among the values that some rows of the unit see and others do not
                    for (int i = 0; i < p.tiles[t]; ++i) {
                        const int j = key_tile(p, i);
                        if (whole_tile(a, p.t0, p.p1, j)) continue;
                        for (int z = j * kTile; z < (j + 1) * kTile && z <= pos; ++z) {
                            if (z < low && z >= a.sinks) continue;
                            // (those that all see have stayed where they were)
                            if (z <= p.t0 && (z >= low_of(a, p.p1) || z < a.sinks)) continue;
                            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v) + (p.first + static_cast<long long>(z)) * a.vs[0] + p.h * a.vs[1];
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                if (c + e >= a.D) break;
                                const float val = __bfloat162float(v[c + e]);
                                if (!isfinite(val)) o[e] += val;
                            }
                        }
                    }
                }
                __syncwarp();
                uint4 w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t* const x = reinterpret_cast<uint32_t*>(&w[e]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(o[8 * e + 2 * y] * f, o[8 * e + 2 * y + 1] * f);
                        x[y] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
                if (out_vec) {
                    // w[e] of lane 4 r + l becomes w[l] of lane 4 r + e: bits of l and e are swapped one after the other
#pragma unroll
                    for (int step = 1; step < 4; step *= 2) {
                        const bool up = lane & step;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (e & step) continue;
                            uint4 &x = w[e], &y = w[e + step];
                            const uint4 send = up ? x : y;
                            uint4 got;
                            got.x = __shfl_xor_sync(0xffffffffu, send.x, step);
                            got.y = __shfl_xor_sync(0xffffffffu, send.y, step);
                            got.z = __shfl_xor_sync(0xffffffffu, send.z, step);
                            got.w = __shfl_xor_sync(0xffffffffu, send.w, step);
                            if (up) x = got;
                            else y = got;
                        }
                    }
                    const int d = c + (lane & 3) * 8;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // row e of the four
                        const int from = (lane & ~3) + e;
                        const long long to = __shfl_sync(0xffffffffu, out_at, from);
                        const bool there = __shfl_sync(0xffffffffu, static_cast<int>(live), from);
                        if (there && d < a.D) *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(to) + d) = w[e];
                    }
                } else if (live) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c + e < a.D) out[c + e] = __ushort_as_bfloat16(static_cast<unsigned short>(reinterpret_cast<const uint32_t*>(&w[e / 8])[e % 8 / 2] >> (e % 2 * 16)));
                }
            }
            fence_before();
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kIssueWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

bool encode_rows(const PromptArgs& a, const void* at, const long long* stride, int heads, int box_heads, int box_tokens, CUtensorMap* map) {
    const Encode fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.D), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(a.tokens)};
    // (the stride of an axis of one is nobody's concern, but has to be one that the map takes)
    const cuuint64_t st[2] = {static_cast<cuuint64_t>(heads > 1 ? stride[1] : a.D) * 2, static_cast<cuuint64_t>(a.tokens > 1 ? stride[0] : a.D) * 2};
    if (st[0] == 0 || st[1] == 0) return false;
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_tokens)}, ones[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(at), dims, st, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NP>
cudaError_t launch_tiles(const PromptArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int tokens_each, bool out_vec, cudaStream_t stream) {
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_shared(prompt_tiles_kernel<NP>, PromptShape<NP>::kBytes, asked);
    for (int base = 0; base < a.B && e == cudaSuccess; base += kMostPrompts) {
        const int n = a.B - base < kMostPrompts ? a.B - base : kMostPrompts;
        const long long pairs = static_cast<long long>(a.tokens) / (2 * tokens_each) + n, units = pairs * a.Hkv;      // (as many as there may be)
        prompt_tiles_kernel<NP><<<static_cast<unsigned>(units), kPromptThreads, PromptShape<NP>::kBytes, stream>>>(a, base, n, q, k, v, tokens_each, out_vec);
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace

int prompt_tiles_launches(int B) { return (B + kMostPrompts - 1) / kMostPrompts; }
// (scores are multiplied by a number that keeps their order, and -inf as it is)
bool prompt_tiles_takes(const PromptArgs& a) { return a.D >= 16 && a.D <= 128 && a.D % 8 == 0 && a.group <= kTile && a.kf > 0.f; }
cudaError_t launch_prompt_tiles(const PromptArgs& a, bool out_vec, cudaStream_t stream, bool* taken) {
    const int tokens_each = kTile / a.group;
    CUtensorMap q, k, v;
    *taken = encode_rows(a, a.q, a.qs, a.Hkv * a.group, a.group, tokens_each, &q) && encode_rows(a, a.k, a.ks, a.Hkv, 1, kTile, &k) && encode_rows(a, a.v, a.vs, a.Hkv, 1, kTile, &v);
    if (!*taken) return cudaSuccess;
    return a.D <= 64 ? launch_tiles<1>(a, q, k, v, tokens_each, out_vec, stream) : launch_tiles<2>(a, q, k, v, tokens_each, out_vec, stream);
}

}  // namespace bv
