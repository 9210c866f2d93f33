// Rows of logits cut by top-k, top-p and min-p, and the drawing of a token from what is left: bv_sample_filtered, bv_filter_logits.
//
// Tokens in order, larger logits first and equal ones by index: what is kept is a beginning of that order, up to a last one, (key, index).  The
// top-k largest: the first k.  top-p: those before which less than top_p of the mass of the k lies.  min-p: those not
// below max + T ln(min_p).  So a row's outcome is one pair: a token is kept if its key is larger, or equal and its index not larger.
//
// A row is a cluster's, up to eight CTAs that hold it in shared memory from the one time it is read until it is written (or one CTA's that reads it again).  The
// last kept one is found by one of
//   candidates   top-k of up to 1024: the k-th largest of the vectors' maxima, from a histogram, bounds the k-th token; what is not below goes into a list, which the
//                first CTA puts in order, and the rest (top-p, min-p, the token) follows from the list
//   values       16 bits: the tokens of each value are counted, so that a mass is a count times a weight
//   masses       32 bits: a histogram over the distance from the largest bounds the masses, so that only the tokens of a few bins have to be put in order
//   digits       whatever the others leave (lists that do not fit, infinities where the bins would be): 11, 11 and 10 bits of the keys, a histogram each, of counts or of
//                weights as multiples of 2^-69 of the largest in 96 bits, whose sums do not depend on the order of the additions (64 bits held 2^-45 for 128256 tokens,
//                2^-35 for 2^26, where a tail of lighter tokens was taken for nothing)
// Weights are exponentials in 64 bits: a border between tokens of 10^-6 each is off by 10^-5 of a token for an error of 10^-11.
//
// One row of 32000, top_k 50, top_p 0.95: 14.5 us (13 on the GPU), a chain of barriers and exchanges between CTAs; 64 rows of 128256, top_p 0.9: 35 us, the same
// chain and the histogram's additions (8 of 35); 576 rows, top_k 1000: 124 us, a row's sweeps one after the other (read, read again, filled) with two CTAs an SM, HBM at a
// third; 37 rows of 50257 in 32 bits, all kinds of cuts: 31 us, of which those with top_p alone take longest (37 of one kind: top_p 0.9 36 us, nothing cut 21,
// top_k of 1 to 200 with or without top_p 20 to 23, min_p 14): a third of the warps' waits is for barriers, the pipe for 64 bits is at 3 % (21 % on the busiest SM).  By digits, where
// thousands of tokens about the border are nearly equal: 37 rows of 50257, top_p 0.9, equal logits 262 us, steps of a quarter 297, within some hundredths 158.
// Measured and not kept: bins of fixed values counted while a row is read (64 rows 49 us against 39 then); a wider ring of loads for rows that are read again.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

#include "bv_cache.cuh"
#include "bv_device.cuh"
#include "bv_launch.h"

#include "../../include/bv.h"

namespace bv {
namespace {

namespace cg = cooperative_groups;

constexpr int kFThreads = 512, kFWarps = kFThreads / 32;
constexpr int kDigits = 2048;
constexpr int kAll = 0x7fffffff;

struct FilterArgs {
    const char* logits;
    long long stride, out_stride;        // bytes between rows
    const float* uniforms;               // null: nothing is drawn
    float temperature, top_p, min_p;
    int top_k;
    const float *temperatures, *top_ps, *min_ps;      // [rows] or null: the numbers above
    const int32_t* top_ks;
    int32_t* tokens;
    float* lse;                          // null: not wanted
    char* out;                           // null: not wanted
    int V, per_cta;                      // elements of a CTA's part
    bool vec_in, vec_out;
};

// 2^(y / 16) for y <= 0, but for some 10^-13: a sixteenth of a power of two from a table (roots[i] = 2^(i / 16), in shared memory, where no two of them
// share a bank), the rest, at most half a sixteenth, by the series of the exponential.  Twelve operations with the sum, where a series about the nearest
// integer takes 21, and the pipe for 64 bits is what a pass over a whole vocabulary waits for.  (No branch: a thread's several are under way together.)
constexpr int kRoots = 16;
__device__ __forceinline__ double pow2_16th(double y, const double* roots) {
    const double magic = 6755399441055744.0;         // 1.5 2^52
    constexpr double c = 0.69314718055994530942 / kRoots;
    const bool some = y > -1000.0 * kRoots;
    y = some ? y : 0.0;
    const double t = y + magic, f = y - (t - magic);
    const int n = __double2loint(t);
    double s = c * c * c * c * c / 120.0;
    s = fma(s, f, c * c * c * c / 24.0);
    s = fma(s, f, c * c * c / 6.0);
    s = fma(s, f, c * c / 2.0);
    s = fma(s, f, c);
    const double r = roots[n & (kRoots - 1)];
    s = fma(s * f, r, r);
    const double w = __hiloint2double(__double2hiint(s) + (n >> 4 << 20), __double2loint(s));
    return some ? w : 0.0;
}

template <int DT> struct Row;
template <> struct Row<kF32> {
    using E = uint32_t;
    static constexpr int kN = 4;
    static constexpr uint32_t kNegInf = 0xff800000u, kNaN = 0x7fc00000u;
    static constexpr float kLeast = -3.40282347e38f;
    // The largest of a vector's, NaN if one is.
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
        return __float_as_uint(r);
    }
    static __device__ __forceinline__ float top(const uint4& v) { return __uint_as_float(larger(larger(v.x, v.y), larger(v.z, v.w))); }
    static __device__ __forceinline__ float get(const uint4& v, int i) { return __uint_as_float(reinterpret_cast<const uint32_t*>(&v)[i]); }
    // Which elements are not below z (at_least: of the type, rounded down), a bit each: element i is bit(i).
    static constexpr __device__ __forceinline__ int bit(int i) { return i; }
    static __device__ __forceinline__ float at_least(float z) { return z; }
    static __device__ __forceinline__ unsigned from(const uint4& v, float z) {
        return static_cast<unsigned>(get(v, 0) >= z) | static_cast<unsigned>(get(v, 1) >= z) << 1 | static_cast<unsigned>(get(v, 2) >= z) << 2 | static_cast<unsigned>(get(v, 3) >= z) << 3;
    }
};
template <> struct Row<kBF16> {
    using E = uint16_t;
    static constexpr int kN = 8;
    static constexpr uint32_t kNegInf = 0xff80ff80u, kNaN = 0x7fc07fc0u;
    static constexpr float kLeast = -3.38953139e38f;
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float top(const uint4& v) {
        const uint32_t x = larger(larger(v.x, v.y), larger(v.z, v.w));
        return __uint_as_float(larger(x, x << 16) & 0xffff0000u);
    }
    static __device__ __forceinline__ float get(const uint4& v, int i) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&v)[i / 2];
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    static constexpr __device__ __forceinline__ int bit(int i) { return i / 2 + i % 2 * 16; }
    static __device__ __forceinline__ float at_least(float z) { return __bfloat162float(__float2bfloat16_rd(z)); }
    static __device__ __forceinline__ unsigned from(const uint4& v, float z) {
        const __nv_bfloat162 b = __float2bfloat162_rn(z);
        auto pair = [&](uint32_t w) { return __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w), b); };
        return (pair(v.x) & 0x00010001u) | (pair(v.y) & 0x00020002u) | (pair(v.z) & 0x00040004u) | (pair(v.w) & 0x00080008u);
    }
};

// The order of floats as that of integers; zeros are one value.  (In 16 bits the lower half is 0, negative ones' too.)
template <int DT> constexpr uint32_t kKeyBits = DT == kF32 ? 0xffffffffu : 0xffff0000u;
template <int DT> constexpr uint32_t kLowest = 0x007fffffu & kKeyBits<DT>;      // the key of -inf
template <int DT> __device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return (u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u)) & kKeyBits<DT>;
}
template <int DT> __device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u ? key ^ 0x80000000u : ~key) & kKeyBits<DT>); }

// What is kept: keys above `key`, and equal ones up to index `last`.
struct Border {
    uint32_t key;
    int last;
    __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

constexpr int kBins = 2048;              // of a histogram over values: four a thread
constexpr float kPerNat = 64.f;          // bins of top-p's to a factor e of the weights
static_assert(kBins == 4 * kFThreads, "");
constexpr int kList = 4096;              // tokens that are put in order one by one
constexpr int kShort = kList / 2;        // of a list that leaves room for buckets behind it
constexpr int kWide = 8192;              // bins by the upper 13 bits of keys: 16 to a power of two
constexpr int kMostK = 1024;             // of a top-k by candidates
constexpr int kFew = 2048;               // tokens of which all are candidates

// Values of 16 bits to bins, a bin a value from the largest down: keys from kM down to pos_lo, one bin for those between pos_lo and neg_hi (values next to 0),
// then from neg_hi down; the last bin takes all the rest.  neg_hi below 0: no such bin between.
struct KeyBins {
    int kM, pos_lo, neg_hi, base;
    __device__ __forceinline__ int bin(float z) const {
        const int key = static_cast<int>(key_of<kBF16>(z) >> 16), i = key >= pos_lo ? kM - key : key > neg_hi ? base : base + 1 + neg_hi - key;
        return i < kBins - 1 ? i : kBins - 1;
    }
    __device__ __forceinline__ bool shared(int b) const { return b == kBins - 1 || (neg_hi >= 0 && b == base); }
    __device__ __forceinline__ float value(int b) const { return value_of<kBF16>(static_cast<uint32_t>(neg_hi < 0 || b < base ? kM - b : neg_hi - (b - base - 1)) << 16); }
};
struct FilterSmem {
    union {
        unsigned bins[kBins];
        struct {
            unsigned count[kDigits];
            unsigned carry[kDigits];     // of the masses: what is above 64 bits
            unsigned long long mass[kDigits];
        };
        unsigned long long list[kList];  // key, then the index turned round: in order when they descend
        unsigned wide[kWide];
    };
    double roots[kRoots];
    double warp_mass[kFWarps], warp_above[kFWarps];      // read by the other CTAs, as are the next four
    unsigned warp_count[kFWarps];
    float cta_top, cta_low;
    int cta_bad;
    Border border;                       // from the first CTA
    unsigned listed;                     // (the first CTA's: tokens in its list)
    float warp_top[kFWarps], warp_low[kFWarps];
    int warp_bad[kFWarps];
    unsigned scan_count[kFWarps];
    double scan_a[kFWarps], scan_b[kFWarps];
    // what a step found
    double above_mass;
    unsigned digit, found, above;
    int index;
};

template <typename T> __device__ __forceinline__ T scanned(T x, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T u = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += u;
    }
    return x;
}
__device__ __forceinline__ double summed(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// The n numbers of a list in descending order, by all threads.  bucket(x) in 0 .. kShort - 1, not falling as x falls.  Up to kShort of them by buckets: counted,
// placed, and within a bucket by comparison with the others there; more by a network.  (2048 by the network: 47000 clocks.)
template <typename F> __device__ __forceinline__ void order_list(FilterSmem& sm, int n, F bucket) {
    unsigned long long* const list = sm.list;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __syncthreads();
    if (n <= kShort) {
        constexpr int kMine = kShort / kFThreads;
        unsigned* const count = reinterpret_cast<unsigned*>(list + kShort);      // [kShort] how many, then where they begin
        unsigned long long x[kMine];
        unsigned at[kMine];
        int in[kMine];
        for (int i = tid; i < kShort; i += kFThreads) count[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (tid + i * kFThreads >= n) break;
            x[i] = list[tid + i * kFThreads];
            in[i] = bucket(x[i]);
            at[i] = atomicAdd(&count[in[i]], 1u);
        }
        __syncthreads();
        uint4& mine = reinterpret_cast<uint4*>(count)[tid];
        static_assert(kShort == 4 * kFThreads, "four buckets a thread");
        const uint4 c = mine;
        unsigned b = scanned(c.x + c.y + c.z + c.w, lane);
        if (lane == 31) sm.scan_count[warp] = b;
        __syncthreads();
        b -= c.x + c.y + c.z + c.w;
        for (int w = 0; w < warp; ++w) b += sm.scan_count[w];
        mine = make_uint4(b, b + c.x, b + c.x + c.y, b + c.x + c.y + c.z);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (tid + i * kFThreads >= n) break;
            list[count[in[i]] + at[i]] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (tid + i * kFThreads >= n) break;
            const unsigned from = count[in[i]], to = in[i] + 1 < kShort ? count[in[i] + 1] : n;
            at[i] = from;
            for (unsigned o = from; o < to; ++o) at[i] += list[o] > x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (tid + i * kFThreads >= n) break;
            list[at[i]] = x[i];
        }
        __syncthreads();
        return;
    }
    for (int i = n + tid; i < kList; i += kFThreads) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= kList; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int x = tid; x < kList / 2; x += kFThreads) {
                const int i = 2 * x - (x & (j - 1)), o = i + j;      // (i: the x-th index without bit j)
                const unsigned long long u = list[i], v = list[o];
                if ((u < v) == ((i & k) == 0)) { list[i] = v; list[o] = u; }
            }
            __syncthreads();
        }
}

// A CTA's part of a row lies in shared memory where that holds it (RES), else it is read anew in each pass.
template <int DT, bool RES>
__global__ void __launch_bounds__(kFThreads, 2) filter_kernel(const FilterArgs a) {
    using R = Row<DT>;
    using E = typename R::E;
    constexpr int N = R::kN;
    extern __shared__ __align__(16) char raw[];
    FilterSmem& sm = *reinterpret_cast<FilterSmem*>(raw);
    uint4* const part = reinterpret_cast<uint4*>(raw + (sizeof(FilterSmem) + 15) / 16 * 16);
    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int row = static_cast<int>(blockIdx.x) / C;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const char* const in = a.logits + row * a.stride;
    FilterSmem* const first_cta = cluster.map_shared_rank(&sm, 0);

    // a warp has nv runs of 32 vectors, one after the other
    const int nv = a.per_cta / (kFThreads * N);
    const int warp_first = rank * a.per_cta + warp * nv * 32 * N;
    auto index_of = [&](int j) { return warp_first + (j * 32 + lane) * N; };
    auto load = [&](int j) {
        const int i = index_of(j);
        uint4 v = make_uint4(R::kNegInf, R::kNegInf, R::kNegInf, R::kNegInf);
        if (a.vec_in && i + N <= a.V) return ld_stream_v4(in + static_cast<long long>(i) * sizeof(E));
        E* e = reinterpret_cast<E*>(&v);
#pragma unroll
        for (int x = 0; x < N; ++x)
            if (i + x < a.V) e[x] = reinterpret_cast<const E*>(in)[i + x];
        return v;
    };
    uint4* const mine = part + warp * nv * 32 + lane;
    // f(vector, index of its first element), in the order of the row within a warp.  From shared memory the next vector is under way (and f is there
    // once: its instructions, which run a few times a launch, are fetched for it); from memory four vectors are.
    auto each = [&](auto&& f) {
        if constexpr (RES) {
            uint4 next = mine[0];
#pragma unroll 1
            for (int j = 0; j < nv; ++j) {
                const uint4 v = next;
                if (j + 1 < nv) next = mine[(j + 1) * 32];
                f(v, index_of(j));
            }
        } else {
#pragma unroll 1
            for (int j0 = 0; j0 < nv; j0 += 4) {
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j0 + j < nv) v[j] = load(j0 + j);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j0 + j < nv) f(v[j], index_of(j0 + j));
            }
        }
    };

    // ---- the largest of all, the least of the threads' largest, and what cannot be read ----
    const float T = a.temperatures ? a.temperatures[row] : a.temperature, p = a.top_ps ? a.top_ps[row] : a.top_p, m = a.min_ps ? a.min_ps[row] : a.min_p;
    int k = a.top_ks ? a.top_ks[row] : a.top_k;
    if (k <= 0 || k > a.V) k = a.V;
    if (p == 0.f) k = 1;                               // (the first one always)
    // (few from each CTA are found faster than all values are counted: k = 50 of 32000, 14.5 us against 18)
    const bool counting = DT == kBF16 && (k < a.V || (p < 1.f && p > 0.f)) && !(k < a.V && C * k <= kMostK && a.V > kFew);
    // Each CTA's own k-th where those of all together are few: no histogram of all to wait for, and the vectors' maxima are counted while the row is read.
    const bool own = k < a.V && k <= kMostK && (C == 1 || C * k <= kMostK) && a.V > kFew;
    for (int x = tid; x < (own ? kWide : kBins); x += kFThreads) sm.wide[x] = 0;
    if (own) __syncthreads();
    if (tid == 0) sm.listed = 0;
    if (tid < kRoots) sm.roots[tid] = exp2(static_cast<double>(tid) / kRoots);
    float top = -INFINITY;
    bool bad = false;
    {
        constexpr int kAhead = 4;
#pragma unroll 1
        for (int j0 = 0; j0 < nv; j0 += kAhead) {
            uint4 v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (j0 + j < nv) v[j] = load(j0 + j);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (j0 + j >= nv) break;
                if (RES) mine[(j0 + j) * 32] = v[j];
                const float z = R::top(v[j]);
                bad |= !(z < INFINITY);
                top = fmaxf(top, z);
                if (own) atomicAdd(&sm.wide[kWide - 1 - (key_of<DT>(z) >> 19)], 1u);
            }
        }
        // (threads without an element that is finite have no part in the least)
        float low = top > -INFINITY ? top : INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        }
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) { sm.warp_top[warp] = top; sm.warp_low[warp] = low; sm.warp_bad[warp] = bad; }
        __syncthreads();
        if (warp == 0) {
            top = lane < kFWarps ? sm.warp_top[lane] : -INFINITY;
            low = lane < kFWarps ? sm.warp_low[lane] : INFINITY;
            bad = lane < kFWarps && sm.warp_bad[lane];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
            }
            bad = __any_sync(0xffffffffu, bad);
            if (lane == 0) { sm.cta_top = top; sm.cta_low = low; sm.cta_bad = bad; }
        }
    }
    cluster.sync();
    float low = INFINITY;
    {
        const FilterSmem* o = cluster.map_shared_rank(&sm, lane < C ? lane : 0);
        top = o->cta_top;
        low = o->cta_low;
        bad = o->cta_bad != 0;
#pragma unroll
        for (int x = 4; x > 0; x >>= 1) {              // (8 CTAs at most; lanes beyond them have the first's)
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, x));
            bad |= __shfl_xor_sync(0xffffffffu, static_cast<int>(bad), x) != 0;
        }
        top = __shfl_sync(0xffffffffu, top, 0);
        low = __shfl_sync(0xffffffffu, low, 0);
        bad = __shfl_sync(0xffffffffu, static_cast<int>(bad), 0) != 0;
    }
    const bool wrong = !(T > 0.f && T < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f);
    bad |= top == -INFINITY || wrong;
    const double scale = kRoots * 1.4426950408889634073599246810019 / static_cast<double>(T), M = static_cast<double>(top), share = static_cast<double>(p);
    auto weight = [&](float z) { return pow2_16th((static_cast<double>(z) - M) * scale, sm.roots); };
    // min-p: the lowest value of the type that is not below its border
    uint32_t least = 0;
    if (m > 0.f) {
        float x = __double2float_ru(M + static_cast<double>(T) * log(static_cast<double>(m)));
        if constexpr (DT == kBF16) x = __bfloat162float(__float2bfloat16_ru(x));
        least = key_of<DT>(x);
    }
    Border border{kLowest<DT>, kAll};
    // Into the CTA's list: the tokens of which which(vector, index of its first) has a bit.
    auto enlist = [&](auto&& which) {
        each([&](const uint4& v, int i) {
            const unsigned w = which(v, i);
            if (w == 0) return;
            unsigned at = atomicAdd(&sm.listed, static_cast<unsigned>(__popc(w)));
#pragma unroll
            for (int x = 0; x < N; ++x)
                if (w >> R::bit(x) & 1) {
                    if (at < kList) sm.list[at] = static_cast<unsigned long long>(key_of<DT>(R::get(v, x))) << 32 | (0xffffffffu - static_cast<unsigned>(i + x));
                    ++at;
                }
        });
    };
    // ... and all lists into the first CTA's, behind what it has; how many there are in all (more than kList: not all of them are there).
    // (One remote addition a CTA: one for each of a warp's tokens was a microsecond each, 55 us for a row with 1300 candidates.)
    // arrived: every thread has come to the cluster's barrier since it last read what the list lies over; the wait for the others is here, so that
    // the listing between hides it.
    auto collect = [&](bool arrived) {
        __syncthreads();
        if (arrived) cluster.barrier_wait();
        if (rank > 0) {
            const unsigned n = sm.listed;
            if (tid == 0) sm.above = n ? atomicAdd(&first_cta->listed, n) : 0;
            __syncthreads();
            const unsigned at = sm.above;
            for (unsigned x = tid; x < n && x < kList && at + x < kList; x += kFThreads) first_cta->list[at + x] = sm.list[x];
        }
        cluster.sync();
        return first_cta->listed;
    };
    // This CTA's and the others' bins, four a thread from 4 tid on.
    auto gather = [&](unsigned (&c)[4]) {
        uint4 u[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) u[r] = r < C ? reinterpret_cast<const uint4*>(cluster.map_shared_rank(&sm, r)->bins)[tid] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < 4; ++x) c[x] = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) { c[0] += u[r].x; c[1] += u[r].y; c[2] += u[r].z; c[3] += u[r].w; }
    };
    // The sum of x over the threads before this one; `all`: of all threads.
    auto before_me = [&](double x, double* slots, double* all) {
        const double inc = scanned(x, lane);
        if (lane == 31) slots[warp] = inc;
        __syncthreads();
        double b = inc - x, total = 0.0;
        for (int w = 0; w < kFWarps; ++w) {
            if (w < warp) b += slots[w];
            total += slots[w];
        }
        *all = total;
        return b;
    };
    // In the first CTA: of its list of n in order, which are the row's first but for what has `above` of the mass, those before which there is less than
    // `target`, at most `most` of them.
    auto end_of_list = [&](int n, int most, double above, double target) {
        if (n > most) n = most;
        // a thread has consecutive ones
        const int each_has = (n + kFThreads - 1) / kFThreads, i0 = tid * each_has;
        double w = 0.0, all;
        for (int x = i0; x < i0 + each_has && x < n; ++x) w += weight(value_of<DT>(static_cast<uint32_t>(sm.list[x] >> 32)));
        double b = above + before_me(w, sm.scan_a, &all);
        if (tid == 0) sm.found = 0;
        __syncthreads();
        const double limit = target < 0.0 ? share * (above + all) : target;
        unsigned kept = 0;
        for (int x = i0; x < i0 + each_has && x < n; ++x) {
            if (p < 1.f && !(b < limit) && !(above == 0.0 && x == 0)) break;
            kept = x + 1;
            b += weight(value_of<DT>(static_cast<uint32_t>(sm.list[x] >> 32)));
        }
        if (kept) atomicMax(&sm.found, kept);
        __syncthreads();
        return static_cast<int>(sm.found);
    };
    // The first CTA's list in order, by buckets between its largest and its smallest value.
    auto order_by_value = [&](int n) {
        if (tid == 0) { sm.digit = 0; sm.found = 0xffffffffu; }
        __syncthreads();
        unsigned hi = 0, lo = 0xffffffffu;
        for (int x = tid; x < n; x += kFThreads) {
            const unsigned key = static_cast<unsigned>(sm.list[x] >> 32);
            hi = key > hi ? key : hi;
            lo = key < lo ? key : lo;
        }
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        if (lane == 0) { atomicMax(&sm.digit, hi); atomicMin(&sm.found, lo); }
        __syncthreads();
        const float from = value_of<DT>(sm.digit), wide = from - value_of<DT>(sm.found), fine = wide > 0.f ? (kShort - 1) / wide : 0.f;
        // (a width that is infinite or next to nothing leaves buckets of any size, in order all the same)
        order_list(sm, n, [&](unsigned long long x) {
            const float d = (from - value_of<DT>(static_cast<uint32_t>(x >> 32))) * fine;
            return d < static_cast<float>(kShort - 1) ? static_cast<int>(d) : kShort - 1;
        });
    };
    auto entry = [&](int x) { return Border{static_cast<uint32_t>(sm.list[x] >> 32), static_cast<int>(0xffffffffu - static_cast<uint32_t>(sm.list[x]))}; };
    auto announce = [&](Border b) {
        if (tid < C) cluster.map_shared_rank(&sm, tid)->border = b;
    };
    // The index of the some-th token, in the order of the vocabulary, of this key.
    auto last_tie = [&](uint32_t key, unsigned some) {
        const float z = value_of<DT>(key);
        // the index of the last of them: ties by warp, then in the warp that has it
        unsigned own = 0;
        each([&](const uint4& v, int) {
#pragma unroll
            for (int x = 0; x < N; ++x) own += R::get(v, x) == z;
        });
        own = __reduce_add_sync(0xffffffffu, own);
        if (lane == 0) sm.warp_count[warp] = own;
        cluster.sync();
        unsigned before = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int w = 4 * lane + x;
            if (w < rank * kFWarps + warp) before += cluster.map_shared_rank(&sm, w / kFWarps)->warp_count[w % kFWarps];
        }
        before = __reduce_add_sync(0xffffffffu, before);
        if (before < some && before + own >= some) {
            unsigned need = some - before;
            int last = -1;
            each([&](const uint4& v, int i) {
                unsigned n = 0;
#pragma unroll
                for (int x = 0; x < N; ++x) n += R::get(v, x) == z;
                unsigned inc = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const unsigned u = __shfl_up_sync(0xffffffffu, inc, o);
                    if (lane >= o) inc += u;
                }
                const unsigned all = __shfl_sync(0xffffffffu, inc, 31);
                if (need > inc - n && need <= inc) {
                    unsigned left = need - (inc - n);
#pragma unroll
                    for (int x = 0; x < N; ++x)
                        if (R::get(v, x) == z && --left == 0) last = i + x;
                }
                need = need > all ? need - all : 0;                   // (0: found; no later one is)
            });
            if (last >= 0)
                for (int r = 0; r < C; ++r) cluster.map_shared_rank(&sm, r)->index = last;
        }
        cluster.sync();
        return sm.index;
    };
    // One digit after the other, from the top: the largest key of which `enough` is true once all larger ones and its own are counted in.
    auto select = [&](bool by_mass, int k, double target_share) {
        const Border among = border;
        uint32_t prefix = 0;
        unsigned above = 0, ties = 0;
        double above_mass = 0.0, target = 0.0;
        constexpr int kLevels = DT == kBF16 ? 2 : 3;
#pragma unroll 1
        for (int level = 0; level < kLevels; ++level) {
            const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, digits = level == 2 ? 1024 : kDigits;
            for (int x = tid; x < kDigits; x += kFThreads) { sm.count[x] = 0; sm.carry[x] = 0; sm.mass[x] = 0; }
            __syncthreads();
            each([&](const uint4& v, int i) {
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float z = R::get(v, x);
                    const uint32_t key = key_of<DT>(z);
                    const bool in_range = level == 0 || (key >> (level == 1 ? 21 : 10)) == prefix;
                    if (key > kLowest<DT> && in_range && among.keeps(key, i + x)) {
                        const int d = key >> shift & (digits - 1);
                        atomicAdd(&sm.count[d], 1u);
                        if (by_mass) {
                            // (at most 32 wholes of 2^-5 and 2^64 parts of one; up to 2^26 of them stay below 2^96)
                            const double w = 32.0 * weight(z);
                            const unsigned whole = __double2uint_rz(w);
                            const unsigned long long part = __double2ull_rz((w - whole) * 18446744073709551616.0), was = atomicAdd(&sm.mass[d], part);
                            const unsigned over = whole + (was + part < was);
                            if (over) atomicAdd(&sm.carry[d], over);
                        }
                    }
                }
            });
            cluster.sync();
            // four digits a thread, the largest first
            unsigned c[4], cs = 0;
            double w[4], ws = 0.0, all;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int d = kDigits - 1 - (4 * tid + x);
                unsigned long long part = 0, whole = 0;
                c[x] = 0;
                for (int r = 0; r < C; ++r) {
                    const FilterSmem* o = cluster.map_shared_rank(&sm, r);
                    c[x] += o->count[d];
                    if (by_mass) {
                        part += o->mass[d];
                        whole += o->carry[d] + (part < o->mass[d]);
                    }
                }
                // (one rounding; sums of these in one order, whatever that of the additions was)
                w[x] = static_cast<double>(whole) / 32.0 + static_cast<double>(part) / 590295810358705651712.0;
                cs += c[x];
                ws += w[x];
            }
            const unsigned inc = scanned(cs, lane);
            if (lane == 31) sm.scan_count[warp] = inc;
            if (tid == 0) sm.found = 0;
            const double first = above_mass + before_me(ws, sm.scan_a, &all);      // (a barrier in it)
            unsigned before = above + inc - cs;
            for (int x = 0; x < warp; ++x) before += sm.scan_count[x];
            if (level == 0) target = target_share * all;
            unsigned cb = before;
            double wb = first;
            // by count: the digit with which k is reached; by mass: the last digit before which there is less than the target
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const bool here = by_mass ? wb < target : cb < static_cast<unsigned>(k);
                if (c[x] > 0 && here) atomicMax(&sm.found, 4u * tid + x + 1);
                cb += c[x];
                wb += w[x];
            }
            __syncthreads();
            const int found = static_cast<int>(sm.found) - 1;         // (there is one: the largest key's)
            if (found >= 4 * tid && found < 4 * tid + 4) {
                cb = before;
                wb = first;
                for (int x = 0; x < found - 4 * tid; ++x) { cb += c[x]; wb += w[x]; }
                sm.digit = kDigits - 1 - found;
                sm.above = cb;
                sm.above_mass = wb;
                sm.index = static_cast<int>(c[found - 4 * tid]);
            }
            __syncthreads();
            prefix = level == 2 ? prefix << 10 | sm.digit : prefix << 11 | sm.digit;
            above = sm.above;
            above_mass = sm.above_mass;
            ties = static_cast<unsigned>(sm.index);
            cluster.sync();                                           // (the histograms have been read)
        }
        const uint32_t key = DT == kBF16 ? prefix << 10 : prefix;
        // how many of the tokens of this key
        unsigned some = ties;
        if (!by_mass) {
            if (static_cast<unsigned>(k) - above < ties) some = static_cast<unsigned>(k) - above;
        } else {
            const double w = weight(value_of<DT>(key));
            if (w > 0.0) {
                double i = ceil((target - above_mass) / w);
                if (i < 1.0) i = 1.0;
                if (i < static_cast<double>(ties)) some = static_cast<unsigned>(i);
            }
        }
        // (all that are left of this key: an earlier cut may have taken some)
        border = Border{key, key == among.key ? among.last : kAll};
        if (some == ties) return;
        border.last = last_tie(key, some);
    };

    int listed_kept = 0;                                 // (the first CTA's: with how many kept tokens its list begins)
    // In the first CTA: the token, of the `kept` ones in its list.
    auto draw = [&](int kept) {
        // the kept ones in the order of the vocabulary: the same entries, turned round, their keys behind
        __syncthreads();
        for (int x = tid; x < kept; x += kFThreads) sm.list[x] = sm.list[x] << 32 | sm.list[x] >> 32;
        const float share_of = static_cast<float>(kShort - 1) / static_cast<float>(a.V);
        order_list(sm, kept, [&](unsigned long long x) { return static_cast<int>(static_cast<float>(0xffffffffu - static_cast<uint32_t>(x >> 32)) * share_of); });
        const int each_has = (kept + kFThreads - 1) / kFThreads, i0 = tid * each_has;
        double w = 0.0, W;
        for (int x = i0; x < i0 + each_has && x < kept; ++x) w += weight(value_of<DT>(static_cast<uint32_t>(sm.list[x])));
        double c = before_me(w, sm.scan_b, &W);
        const double t = static_cast<double>(a.uniforms[row]) * W;
        if (tid == 0) sm.found = 0xffffffffu;
        __syncthreads();
        for (int x = i0; x < i0 + each_has && x < kept; ++x) {
            const double y = weight(value_of<DT>(static_cast<uint32_t>(sm.list[x])));
            c += y;
            if (y > 0.0 && c > t) { atomicMin(&sm.found, static_cast<unsigned>(x)); break; }
        }
        __syncthreads();
        if (tid == 0) {
            int x = static_cast<int>(sm.found);
            // (where rounding leaves none, the last that weighs anything)
            if (x < 0)
                for (x = kept - 1; x > 0 && weight(value_of<DT>(static_cast<uint32_t>(sm.list[x]))) == 0.0;) --x;
            a.tokens[row] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(sm.list[x] >> 32));
            if (a.lse) a.lse[row] = static_cast<float>(M / static_cast<double>(T) + log(W));
        }
    };
    // In the first CTA, whose list begins with the `kept` first tokens in order: min-p, the border for all CTAs, the token.
    auto finish = [&](int kept) {
        // (of keys in order, those below min-p's border come last)
        if (least > 0) {
            __syncthreads();
            if (tid == 0) sm.found = 0;
            __syncthreads();
            for (int x = tid; x < kept; x += kFThreads)
                if (static_cast<uint32_t>(sm.list[x] >> 32) >= least) atomicMax(&sm.found, static_cast<unsigned>(x + 1));
            __syncthreads();
            kept = static_cast<int>(sm.found);
        }
        announce(entry(kept - 1));
        listed_kept = kept;
        if (a.uniforms) draw(kept);
    };
    // In the first CTA, which has a row's first n tokens in its list: what is kept of them, and the token.  target: the mass before which top-p keeps
    // (negative: its share of the k first ones).
    auto conclude = [&](int n, double target) {
        order_by_value(n);
        finish(end_of_list(n, k, 0.0, target));
    };
    // Top-k of up to kMostK by candidates: what is not below the k-th largest of the vectors' maxima, or nearly so.  False: too many.
    bool drew = false;
    auto by_candidates = [&]() {
        if (a.V > kFew) {
            float limit;
            if (own) {
                constexpr int kEach = kWide / kFThreads;
                const uint4* const c = reinterpret_cast<const uint4*>(sm.wide) + tid * (kEach / 4);
                unsigned sum = 0;
                for (int x = 0; x < kEach / 4; ++x) { const uint4 u = c[x]; sum += u.x + u.y + u.z + u.w; }
                const unsigned inc = scanned(sum, lane);
                if (lane == 31) sm.scan_count[warp] = inc;
                if (tid == 0) sm.found = kWide;
                __syncthreads();
                unsigned upto = inc - sum;
                for (int w = 0; w < warp; ++w) upto += sm.scan_count[w];
                if (upto < static_cast<unsigned>(k) && upto + sum >= static_cast<unsigned>(k)) {
                    int x = tid * kEach;
                    while ((upto += sm.wide[x]) < static_cast<unsigned>(k)) ++x;
                    sm.found = x;
                }
                __syncthreads();                         // (the bins have been read)
                // (the others write into the first CTA's list, which lies where its bins are, when it is through with them and not before)
                cluster.barrier_arrive();
                // the lowest value of that bin (a CTA with fewer than k vectors takes all of its own)
                const int bin = static_cast<int>(sm.found);
                limit = bin < kWide ? value_of<kF32>(static_cast<uint32_t>(kWide - 1 - bin) << 19) : -INFINITY;
            } else {
                const float step = (kBins - 1) / (top - low);
                if (!(step > 0.f && step < INFINITY)) return false;
                each([&](const uint4& v, int) {
                    const float d = (top - R::top(v)) * step;
                    if (d < kBins) atomicAdd(&sm.bins[static_cast<int>(d)], 1u);
                });
                cluster.sync();
                unsigned c[4], sum = 0;
                gather(c);
#pragma unroll
                for (int x = 0; x < 4; ++x) sum += c[x];
                const unsigned inc = scanned(sum, lane);
                if (lane == 31) sm.scan_count[warp] = inc;
                if (tid == 0) sm.found = kBins;
                __syncthreads();
                unsigned upto = inc - sum;
                for (int w = 0; w < warp; ++w) upto += sm.scan_count[w];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (upto < static_cast<unsigned>(k) && upto + c[x] >= static_cast<unsigned>(k)) sm.found = 4 * tid + x;
                    upto += c[x];
                }
                cluster.sync();                          // (the bins have been read)
                const int bin = static_cast<int>(sm.found);
                if (bin >= kBins) return false;
                // every vector of the bins up to this one has a maximum that is not below this (a hair lower, for the roundings)
                limit = top - (bin + 1) / step * 1.000001f - fabsf(top) * 1e-6f;
            }
            limit = R::at_least(limit > R::kLeast ? limit : R::kLeast);      // (-inf is nobody's candidate)
            enlist([&](const uint4& v, int) { return R::from(v, limit); });
        } else {
            enlist([&](const uint4& v, int) {
                unsigned which = 0;
#pragma unroll
                for (int x = 0; x < N; ++x) which |= static_cast<unsigned>(R::get(v, x) > -INFINITY) << R::bit(x);
                return which;
            });
        }
        const unsigned n = collect(own);
        if (n > kList) return false;
        if (rank == 0) {
            conclude(static_cast<int>(n), -1.0);
        }
        cluster.sync();
        border = sm.border;
        drew = true;
        return true;
    };

    // Top-p by a histogram over the distance from the largest, 1/64 of T a bin: counts bound the mass of each, so that only a few bins can hold the border;
    // their tokens are put in order, what lies before them is summed up.  False: too many.
    auto by_mass = [&]() {
        const Border among = border;
        const float among_z = value_of<DT>(among.key), step = kPerNat / T;
        // (a distance that 32 bits do not hold counts as the last bin, where it belongs but for temperatures near the largest there are)
        if (!(step < INFINITY) || T > 1e36f) return false;
        auto counts = [&](float z, int i) { return z > among_z || (z == among_z && i <= among.last && z > -INFINITY); };
        auto bin_of = [&](float z) { return static_cast<int>(fminf((top - z) * step, static_cast<float>(kBins - 1))); };
        each([&](const uint4& v, int i) {
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float z = R::get(v, x);
                if (counts(z, i + x)) atomicAdd(&sm.bins[bin_of(z)], 1u);
            }
        });
        cluster.sync();
        unsigned c[4];
        gather(c);
        // (a bin's weights lie between these but for some 10^-5: roundings of distances up to 32, of exponentials)
        double up[4], lo[4], u = 0.0, l = 0.0, all_u, all_l;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int b = 4 * tid + x;
            up[x] = c[x] ? c[x] * static_cast<double>(1.00003f * exp2f(-1.44269504f / kPerNat * b)) : 0.0;
            lo[x] = c[x] && b < kBins - 1 ? c[x] * static_cast<double>(0.99997f * exp2f(-1.44269504f / kPerNat * (b + 1))) : 0.0;
            u += up[x];
            l += lo[x];
        }
        double ub = before_me(u, sm.scan_a, &all_u), lb = before_me(l, sm.scan_b, &all_l);
        if (tid == 0) { sm.digit = 0; sm.found = kBins; sm.above = 0; sm.index = 0; }
        __syncthreads();
        // Bins that are kept whole: prefix (1 - p) < p rest for the largest prefix and the least rest.  Bins of which nothing is kept: the prefix
        // before them is enough in the worst case.
        unsigned whole = 0, none = kBins;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (none == kBins && lb * (1.0 - share) >= share * (all_u - ub) * 1.0000001) none = 4 * tid + x;
            ub += up[x];
            lb += lo[x];
            if (ub * (1.0 - share) < share * (all_l - lb) * 0.9999999) whole = 4 * tid + x + 1;
        }
        if (whole) atomicMax(&sm.digit, whole);
        if (none < kBins) atomicMin(&sm.found, none);
        __syncthreads();
        const int b0 = static_cast<int>(sm.digit);
        int b1 = static_cast<int>(sm.found) - 1;
        if (b1 < b0) b1 = b0;
        unsigned inside = 0, before = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (4 * tid + x < b0) before += c[x];
            else if (4 * tid + x <= b1) inside += c[x];
        }
        inside = __reduce_add_sync(0xffffffffu, inside);
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) { atomicAdd(&sm.above, inside); atomicAdd(&sm.index, static_cast<int>(before)); }
        cluster.sync();                                  // (the bins have been read)
        unsigned n = sm.above;
        if (n == 0 || n > kList) return false;
        // where all that may be kept is little, all of it goes into the list, and the token is drawn there
        const bool all_of_it = n + static_cast<unsigned>(sm.index) <= kShort;
        if (all_of_it) n += static_cast<unsigned>(sm.index);
        double above = 0.0, rest = 0.0;
        each([&](const uint4& v, int i) {
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float z = R::get(v, x);
                const double w = counts(z, i + x) ? weight(z) : 0.0;
                const bool sure = bin_of(z) < b0;
                above += sure ? w : 0.0;
                rest += sure ? 0.0 : w;
            }
        });
        above = summed(above);
        rest = summed(rest);
        if (lane == 0) { sm.warp_above[warp] = above; sm.warp_mass[warp] = rest; }
        const int from = all_of_it ? 0 : b0;
        enlist([&](const uint4& v, int i) {
            unsigned which = 0;
            if (bin_of(R::top(v)) > b1) return which;
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float z = R::get(v, x);
                const int b = bin_of(z);
                which |= static_cast<unsigned>(b >= from && b <= b1 && counts(z, i + x)) << R::bit(x);
            }
            return which;
        });
        collect(false);
        if (rank == 0) {
            const FilterSmem* o = cluster.map_shared_rank(&sm, tid < C * kFWarps ? tid / kFWarps : 0);
            const double x = tid < C * kFWarps ? o->warp_above[tid % kFWarps] : 0.0, y = tid < C * kFWarps ? o->warp_mass[tid % kFWarps] : 0.0;
            before_me(x, sm.scan_a, &above);
            before_me(y, sm.scan_b, &rest);
            const double target = share * (above + rest);
            __syncthreads();
            if (all_of_it) {
                conclude(static_cast<int>(n), target);
            } else {
                order_by_value(static_cast<int>(n));
                const int kept = end_of_list(static_cast<int>(n), static_cast<int>(n), above, target);
                // (none of them: the border lies before the first, whose index is the lowest of its value)
                announce(kept > 0 ? entry(kept - 1) : Border{entry(0).key, -1});
            }
        }
        cluster.sync();
        border = sm.border;
        drew = all_of_it;
        return true;
    };

    // In 16 bits, top-k and top-p by counting the tokens of each value: a bin a value from the largest down, so that a mass is a count times a weight, and
    // the border is where the formulas have it.  2048 bins hold 16 powers of two; where logits of both signs matter, the values next to 0 share one bin, as do the
    // least, and their masses are summed up (64 rows of 128256, top_p 0.9: 61 us with bins of equal width and all weights summed up, then 39).  How many are kept, or
    // -1: the border lies in a shared bin.
    auto by_keys = [&]() {
        const bool mass = p < 1.f && p > 0.f;
        const int kM = static_cast<int>(key_of<DT>(top) >> 16);
        float least_z = top - 32.f * T;
        if (low < least_z) least_z = low;
        const int kL = least_z > -3.0e38f ? static_cast<int>(key_of<kF32>(least_z) >> 16) : 0x80;
        KeyBins bins{kM, 0, -1, 0};                // (all keys are in the first part)
        if (kM - kL >= kBins - 1 && kM > 0x7fff - 128 && kL < 0x8000) {
            // powers of two from the least up whose values share a bin: so many that both signs' others fit, or those of the one that has any
            int powers = (kM - kL + 3 - kBins + 255) / 256;
            if (0x8000 + powers * 128 > kM) powers = (0x7fff - kL + 4 - kBins + 127) / 128;
            else if (0x7fff - powers * 128 < kL) powers = (kM - 0x8000 + 4 - kBins + 127) / 128;
            powers = powers < 1 ? 1 : powers;
            bins.pos_lo = 0x8000 + powers * 128;
            bins.neg_hi = 0x7fff - powers * 128;
            bins.base = kM >= bins.pos_lo ? kM - bins.pos_lo + 1 : 0;
        }
        each([&](const uint4& v, int) {
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float z = R::get(v, x);
                if (z > -INFINITY) atomicAdd(&sm.bins[bins.bin(z)], 1u);
            }
        });
        cluster.sync();
        auto shared = [&](int b) { return bins.shared(b); };
        auto value = [&](int b) { return bins.value(b); };
        auto bin_of = [&](float z) { return bins.bin(z); };
        unsigned c[4], cs = 0;
        gather(c);
        double w[4], ws = 0.0, all = 0.0, middle = 0.0, rest = 0.0;
        if (mass) {
            bool some = false;
#pragma unroll
            for (int x = 0; x < 4; ++x) some |= c[x] > 0 && shared(4 * tid + x);
            if (__syncthreads_or(some)) {
                each([&](const uint4& v, int) {
#pragma unroll
                    for (int x = 0; x < N; ++x) {
                        const float z = R::get(v, x);
                        const int b = bin_of(z);
                        if (shared(b)) {
                            const double y = weight(z);      // (of -inf: 0)
                            if (b == kBins - 1) rest += y;
                            else middle += y;
                        }
                    }
                });
                middle = summed(middle);
                rest = summed(rest);
                if (lane == 0) { sm.warp_above[warp] = middle; sm.warp_mass[warp] = rest; }
                cluster.sync();
                const FilterSmem* o = cluster.map_shared_rank(&sm, tid < C * kFWarps ? tid / kFWarps : 0);
                before_me(tid < C * kFWarps ? o->warp_above[tid % kFWarps] : 0.0, sm.scan_a, &middle);
                before_me(tid < C * kFWarps ? o->warp_mass[tid % kFWarps] : 0.0, sm.scan_b, &rest);
            }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int b = 4 * tid + x;
            cs += c[x];
            w[x] = !mass || c[x] == 0 ? 0.0 : b == kBins - 1 ? rest : shared(b) ? middle : c[x] * weight(value(b));
            ws += w[x];
        }
        const unsigned inc = scanned(cs, lane);
        if (lane == 31) sm.scan_count[warp] = inc;
        if (tid == 0) { sm.found = 0; sm.digit = kBins; sm.above = 0; sm.index = 0; }
        __syncthreads();
        unsigned cb = inc - cs, total = 0;
        for (int x = 0; x < kFWarps; ++x) {
            if (x < warp) cb += sm.scan_count[x];
            total += sm.scan_count[x];
        }
        double wb = mass ? before_me(ws, sm.scan_a, &all) : 0.0;
        const unsigned most = static_cast<unsigned>(k) < total ? static_cast<unsigned>(k) : total;
        // where the k-th lies, and the mass of the first k
        {
            unsigned u = cb;
            double m = wb;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (u < most && u + c[x] >= most) {
                    sm.digit = 4 * tid + x;
                    sm.above = u;
                    sm.scan_b[0] = u + c[x] == most ? m + w[x] : m + (most - u) * (w[x] / c[x]);
                }
                u += c[x];
                m += w[x];
            }
        }
        __syncthreads();
        const int kth = static_cast<int>(sm.digit);
        const unsigned before_kth = sm.above;
        if (mass) {
            // the last bin before which there is less than the target
            const double target = share * sm.scan_b[0];
            unsigned u = cb;
            double m = wb;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (c[x] > 0 && 4 * tid + x <= kth && (m < target || u == 0)) atomicMax(&sm.found, static_cast<unsigned>(4 * tid + x + 1));
                u += c[x];
                m += w[x];
            }
            __syncthreads();
            u = cb;
            m = wb;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (4 * tid + x + 1 == static_cast<int>(sm.found)) {
                    const unsigned there = 4 * tid + x == kth ? most - before_kth : c[x];
                    const double i = ceil((target - m) / (w[x] / c[x]));
                    sm.index = static_cast<int>(!(i >= 1.0) ? 1u : i < there ? static_cast<unsigned>(i) : there);
                    sm.above = u;
                    sm.listed = c[x];
                }
                u += c[x];
                m += w[x];
            }
        } else if (kth >= 4 * tid && kth < 4 * tid + 4) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (4 * tid + x == kth) sm.listed = c[x];
            sm.found = kth + 1;
            sm.index = static_cast<int>(most - before_kth);
        }
        cluster.sync();                                  // (the bins have been read)
        const int bin = static_cast<int>(sm.found) - 1;
        const unsigned some = static_cast<unsigned>(sm.index), there = sm.listed, kept = sm.above + some;
        __syncthreads();
        if (tid == 0) sm.listed = 0;
        // (the k-th in a shared bin has no mass that is known)
        if (shared(bin) || (mass && k < static_cast<int>(total) && shared(kth))) return -1;
        border = Border{key_of<DT>(value(bin)), kAll};
        // (a short list that a token is drawn from shows which of equal ones are kept)
        if (some < there && !(a.uniforms && kept - some + there <= kShort)) border.last = last_tie(border.key, some);
        return static_cast<int>(kept);
    };

    if (!bad) {
        bool dirty = own;                                // (something lies where the bins are)
        auto clean = [&]() {
            if (!dirty) return;
            for (int x = tid; x < kBins; x += kFThreads) sm.bins[x] = 0;
            if (tid == 0) sm.listed = 0;
            cluster.sync();
        };
        int known = -1;                                  // how many are kept, where that is known
        if constexpr (DT == kBF16) {
            if (counting) {
                dirty = true;
                known = by_keys();
                if (known < 0) border = Border{kLowest<DT>, kAll};
            }
        }
        if (known < 0) {
            if (k < a.V) {
                if (k <= kMostK) {
                    if (!own) clean();
                    dirty = true;
                    by_candidates();
                }
                if (!drew) {
                    dirty = true;
                    cluster.sync();
                    select(false, k, 0.0);
                }
            }
            if (!drew && p < 1.f && p > 0.f) {
                clean();
                if (!by_mass()) {
                    cluster.sync();
                    select(true, 0, share);
                }
            }
        }
        if (!drew) {
            if (a.uniforms && known > 0 && known <= kShort) {
                // Few are kept: they are listed, those equal to the last among them, put in order, and the token is drawn from the list.
                const float z0 = value_of<DT>(border.key);
                if (tid == 0) sm.listed = 0;
                cluster.sync();
                enlist([&](const uint4& v, int i) {
                    unsigned which = R::from(v, z0);
                    if (which == 0 || border.last == kAll) return which;
#pragma unroll
                    for (int x = 0; x < N; ++x)
                        if (R::get(v, x) == z0 && i + x > border.last) which &= ~(1u << R::bit(x));
                    return which;
                });
                const int n = static_cast<int>(collect(false));
                if (rank == 0) {
                    order_by_value(n);
                    finish(known < n ? known : n);
                }
                cluster.sync();
                border = sm.border;
                drew = true;
            } else if (least > border.key) {
                border = Border{least, kAll};
            }
        }
    }
    const float border_z = value_of<DT>(border.key);
    auto kept = [&](float z, int i) { return z > border_z || (z == border_z && i <= border.last); };

    // ---- the token ----
    if (a.uniforms && bad) {
        if (rank == 0 && tid == 0) {
            a.tokens[row] = -1;
            if (a.lse) a.lse[row] = __int_as_float(0x7fc00000);
        }
    } else if (a.uniforms && !drew) {
        double sum = 0.0;
        each([&](const uint4& v, int i) {
            if (!__any_sync(0xffffffffu, R::top(v) >= border_z)) return;
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float z = R::get(v, x);
                sum += kept(z, i + x) ? weight(z) : 0.0;
            }
        });
        sum = summed(sum);
        if (lane == 0) sm.warp_mass[warp] = sum;
        cluster.sync();
        // every warp: the sums of all warps in order, four a lane
        double s[4], inc = 0.0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int w = 4 * lane + x;
            s[x] = w < C * kFWarps ? cluster.map_shared_rank(&sm, w / kFWarps)->warp_mass[w % kFWarps] : 0.0;
            inc += s[x];
        }
        inc = scanned(inc, lane);
        const double W = __shfl_sync(0xffffffffu, inc, 31);
        double c = __shfl_up_sync(0xffffffffu, inc, 1);
        if (lane == 0) c = 0.0;
        const double t = static_cast<double>(a.uniforms[row]) * W;
        // the first segment with whose end the border is passed; where rounding leaves none, the last that holds anything
        int seg = -1, last = -1;
        double at = 0.0, at_last = 0.0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (s[x] > 0.0) {
                if (seg < 0 && c + s[x] > t) { seg = 4 * lane + x; at = c; }
                last = 4 * lane + x;
                at_last = c;
            }
            c += s[x];
        }
        const unsigned hit = __ballot_sync(0xffffffffu, seg >= 0), some = __ballot_sync(0xffffffffu, last >= 0);
        const int src = hit ? __ffs(hit) - 1 : 31 - __clz(some);
        seg = __shfl_sync(0xffffffffu, hit ? seg : last, src);
        at = __shfl_sync(0xffffffffu, hit ? at : at_last, src);
        if (seg == rank * kFWarps + warp) {
            int found = -1, latest = -1;
            double run = at;
            each([&](const uint4& v, int i) {
                bool any = false;
#pragma unroll
                for (int x = 0; x < N; ++x) any |= kept(R::get(v, x), i + x);
                if (found >= 0 || !__any_sync(0xffffffffu, any)) return;
                double w[N], n = 0.0;
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float z = R::get(v, x);
                    w[x] = kept(z, i + x) ? weight(z) : 0.0;
                    n += w[x];
                }
                const double upto = scanned(n, lane);
                double c = run + (upto - n);
                int here = -1;
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    c += w[x];
                    if (w[x] > 0.0) {
                        if (here < 0 && c > t) here = i + x;
                        latest = i + x;
                    }
                }
                const unsigned h = __ballot_sync(0xffffffffu, here >= 0);
                if (h) found = __shfl_sync(0xffffffffu, here, __ffs(h) - 1);
                run += __shfl_sync(0xffffffffu, upto, 31);
            });
            if (found < 0) found = __reduce_max_sync(0xffffffffu, latest);
            if (lane == 0) {
                a.tokens[row] = found;
                if (a.lse) a.lse[row] = static_cast<float>(M / static_cast<double>(T) + log(W));
            }
        }
    }

    // ---- the row ----
    // Where a CTA has the whole row and a list of what is kept, the row is not read again: all of it becomes -inf, the kept ones are put back.
    const bool place = !RES && C == 1 && drew && a.vec_out;
    if (a.out && place) {
        char* const out = a.out + row * a.out_stride;
        constexpr int kMine = kList / kFThreads;
        const int n = listed_kept;
        int at[kMine];
        E value[kMine];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int x = tid + i * kFThreads;
            if (x >= n) break;
            at[i] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(a.uniforms ? sm.list[x] >> 32 : sm.list[x]));
            value[i] = reinterpret_cast<const E*>(in)[at[i]];      // (before it is written: the row may be replaced where it lies)
        }
        __syncthreads();
        const uint4 none = make_uint4(R::kNegInf, R::kNegInf, R::kNegInf, R::kNegInf);
        const int whole = a.V / N;
        for (int x = tid; x < whole; x += kFThreads) reinterpret_cast<uint4*>(out)[x] = none;
        for (int x = whole * N + tid; x < a.V; x += kFThreads) reinterpret_cast<E*>(out)[x] = static_cast<E>(R::kNegInf >> (32 - 8 * sizeof(E)));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (tid + i * kFThreads >= n) break;
            reinterpret_cast<E*>(out)[at[i]] = value[i];
        }
    } else if (a.out) {
        char* const out = a.out + row * a.out_stride;
        each([&](const uint4& v, int i) {
            uint4 w = v;
            if (wrong) {
                w = make_uint4(R::kNaN, R::kNaN, R::kNaN, R::kNaN);
            } else if (!bad) {
                w = make_uint4(R::kNegInf, R::kNegInf, R::kNegInf, R::kNegInf);
                if (R::top(v) >= border_z) {
                    E* e = reinterpret_cast<E*>(&w);
                    const E* f = reinterpret_cast<const E*>(&v);
#pragma unroll
                    for (int x = 0; x < N; ++x)
                        if (kept(R::get(v, x), i + x)) e[x] = f[x];
                }
            }
            if (a.vec_out && i + N <= a.V) {
                *reinterpret_cast<uint4*>(out + static_cast<long long>(i) * sizeof(E)) = w;
            } else {
                const E* e = reinterpret_cast<const E*>(&w);
#pragma unroll
                for (int x = 0; x < N; ++x)
                    if (i + x < a.V) reinterpret_cast<E*>(out)[i + x] = e[x];
            }
        });
    }
    cluster.sync();                       // (nobody leaves while its shared memory may be read)
}

constexpr int kSmall = static_cast<int>((sizeof(FilterSmem) + 15) / 16 * 16);
template <int DT, bool RES>
cudaError_t launch(FilterArgs a, int rows, int C, int nv, cudaStream_t stream) {
    static std::atomic<unsigned long long> asked{0};
    const cudaError_t e = allow_shared(filter_kernel<DT, RES>, 227 * 1024, asked);
    if (e != cudaSuccess) return e;
    a.per_cta = nv * kFThreads * Row<DT>::kN;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = static_cast<unsigned>(C);
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(rows) * C);
    cfg.blockDim = dim3(kFThreads);
    cfg.dynamicSmemBytes = kSmall + (RES ? nv * kFThreads * 16 : 0);
    cfg.stream = stream;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, filter_kernel<DT, RES>, a);
}
template <int DT>
cudaError_t pick(const FilterArgs& a, int rows, int sms, cudaStream_t stream) {
    constexpr int N = Row<DT>::kN;
    const long long vecs = (static_cast<long long>(a.V) + N - 1) / N, runs = (vecs + kFThreads - 1) / kFThreads;      // vectors a thread of one CTA would have
    // CTAs of a row: as many as leave two on an SM (8 vectors a thread), and more where rows are fewer than SMs
    constexpr int kTwo = 8, kMost = (227 * 1024 - kSmall) / (kFThreads * 16);
    int C = 1;
    // Many rows that are cut to few tokens: a CTA a row, which reads it twice (from the second level cache or memory) and writes it without another look.  Rows of
    // 128256, top_k 1000: 104 of them 45 us, by four CTAs that hold each 53; 200: 59 and 80; 576: 123 and 216.  In 16 bits also rows for every SM that are cut in any
    // way: top_p 0.9, 148 of them 65 and 85, 300: 138 and 146.  (In 32 bits, 300 of 50257: 168 and 165.)
    const bool few = !a.top_ks && a.top_k > 0 && a.top_k <= kMostK && a.V > kFew;
    if (runs > kTwo && ((few && 10LL * rows > 7LL * sms) || (DT == kBF16 && rows >= sms))) return launch<DT, false>(a, rows, 1, static_cast<int>(runs), stream);
    while (C < 8 && (runs > static_cast<long long>(C) * kTwo || (runs > C && 2LL * C * rows <= sms))) C *= 2;
    const int nv = static_cast<int>((runs + C - 1) / C);
    return nv <= kMost ? launch<DT, true>(a, rows, C, nv, stream) : launch<DT, false>(a, rows, C, nv, stream);
}

bool on(const void* p, size_t x) { return reinterpret_cast<uintptr_t>(p) % x == 0; }

}  // namespace
}  // namespace bv

extern "C" int bv_sample_filtered(const void* logits, int64_t stride, const float* uniforms, int rows, int V, int dtype, const bv_cut* cut, int32_t* out_tokens,
                                  float* out_lse, void* out_logits, int64_t out_stride, void* stream) {
    using bv::on;
    if (!logits || !cut || rows < 0 || V < 1 || stride < 0 || out_stride < 0 || (dtype != BV_DTYPE_F32 && dtype != BV_DTYPE_BF16)) return BV_ERR_INVALID_ARG;
    if ((uniforms != nullptr) != (out_tokens != nullptr) || (!uniforms && (out_lse || !out_logits))) return BV_ERR_INVALID_ARG;
    const int es = dtype == BV_DTYPE_F32 ? 4 : 2;
    if (!on(logits, es) || (out_logits && !on(out_logits, es)) || !on(uniforms, 4) || !on(out_tokens, 4) || !on(out_lse, 4)) return BV_ERR_INVALID_ARG;
    if (!on(cut->temperatures, 4) || !on(cut->top_ks, 4) || !on(cut->top_ps, 4) || !on(cut->min_ps, 4)) return BV_ERR_INVALID_ARG;
    if (!cut->temperatures && (!(cut->temperature > 0.f) || !std::isfinite(cut->temperature))) return BV_ERR_INVALID_ARG;
    if (!cut->top_ps && !(cut->top_p >= 0.f)) return BV_ERR_INVALID_ARG;
    if (!cut->min_ps && !(cut->min_p >= 0.f && cut->min_p <= 1.f)) return BV_ERR_INVALID_ARG;
    if (out_logits && rows > 1 && out_stride < V) return BV_ERR_INVALID_ARG;
    if (V > (1 << 26) || rows > (1 << 27)) return BV_ERR_UNSUPPORTED;
    bv::note_launches(0);
    if (rows == 0) return BV_OK;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return bv::note_cuda_error(e);
    bv::FilterArgs a{};
    a.logits = static_cast<const char*>(logits);
    a.stride = stride * es;
    a.out_stride = out_stride * es;
    a.uniforms = uniforms;
    a.temperature = cut->temperature; a.top_p = cut->top_p; a.min_p = cut->min_p; a.top_k = cut->top_k;
    a.temperatures = cut->temperatures; a.top_ks = cut->top_ks; a.top_ps = cut->top_ps; a.min_ps = cut->min_ps;
    a.tokens = out_tokens; a.lse = out_lse; a.out = static_cast<char*>(out_logits);
    a.V = V;
    a.vec_in = on(logits, 16) && (rows == 1 || a.stride % 16 == 0);
    a.vec_out = on(out_logits, 16) && (rows == 1 || a.out_stride % 16 == 0);
    e = dtype == BV_DTYPE_F32 ? bv::pick<bv::kF32>(a, rows, sms, static_cast<cudaStream_t>(stream)) : bv::pick<bv::kBF16>(a, rows, sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return bv::note_cuda_error(e);
    bv::note_launches(1);
    return BV_OK;
}
