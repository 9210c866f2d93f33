// Rows of logits cut by top-k, top-p and min-p, and the drawing of a token from what is left: bv_sample_filtered, bv_filter_logits.
//
// Tokens in order, larger logits first and equal ones by index: what is kept is a beginning of that order, up to a last one, (key, index).  The
// top-k largest: the first k.  top-p: those before which less than top_p of the mass of the k lies.  min-p: those not
// below max + T ln(min_p).  So a row's outcome is one pair: a token is kept if its key is larger, or equal and its index not larger.
//
// A row is a cluster's, up to eight CTAs that hold it in registers from the one time it is read until it is written.  The last kept key is found digit
// by digit (11, 11 and 10 bits of keys in the order of the logits), a histogram a digit: counts for top-k, and for top-p weights as integers of
// up to 2^-45 of the largest, whose sums do not depend on the order of the additions.  Weights are exponentials in 64 bits: a
// border between tokens of 10^-6 each is off by 10^-5 of a token for an error of 10^-11.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

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
    int V, per_cta, fixed;               // elements of a CTA's part; bits of an integer weight
    bool vec_in, vec_out;
};

// 2^y for y <= 0, to 64 bits but for some 10^-14: the series of e^(f ln 2) about the nearest integer.
__device__ __forceinline__ double pow2(double y) {
    const double magic = 6755399441055744.0;         // 1.5 2^52
    if (!(y > -1000.0)) return 0.0;
    const double t = y + magic, f = (y - (t - magic)) * 0.69314718055994530942;
    double s = 1.0 / 479001600.0;
    s = fma(s, f, 1.0 / 39916800.0);
    s = fma(s, f, 1.0 / 3628800.0);
    s = fma(s, f, 1.0 / 362880.0);
    s = fma(s, f, 1.0 / 40320.0);
    s = fma(s, f, 1.0 / 5040.0);
    s = fma(s, f, 1.0 / 720.0);
    s = fma(s, f, 1.0 / 120.0);
    s = fma(s, f, 1.0 / 24.0);
    s = fma(s, f, 1.0 / 6.0);
    s = fma(s, f, 0.5);
    s = fma(s, f, 1.0);
    s = fma(s, f, 1.0);
    return __hiloint2double(__double2hiint(s) + (__double2loint(t) << 20), __double2loint(s));
}

template <int DT> struct Row;
template <> struct Row<kF32> {
    using E = uint32_t;
    static constexpr int kN = 4;
    static constexpr uint32_t kNegInf = 0xff800000u, kNaN = 0x7fc00000u;
    static __device__ __forceinline__ float get(const uint4& v, int i) { return __uint_as_float(reinterpret_cast<const uint32_t*>(&v)[i]); }
};
template <> struct Row<kBF16> {
    using E = uint16_t;
    static constexpr int kN = 8;
    static constexpr uint32_t kNegInf = 0xff80ff80u, kNaN = 0x7fc07fc0u;
    static __device__ __forceinline__ float get(const uint4& v, int i) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&v)[i / 2];
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
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

struct FilterSmem {
    unsigned count[kDigits];
    unsigned long long mass[kDigits];
    double warp_mass[kFWarps];           // read by the other CTAs
    unsigned warp_count[kFWarps];        // read by the other CTAs
    float warp_top[kFWarps];             // read by the other CTAs
    int warp_bad[kFWarps];
    unsigned scan_count[kFWarps];
    unsigned long long scan_mass[kFWarps];
    // what a step found
    unsigned digit, found, above;
    unsigned long long above_mass, total, digit_mass;
    int index;
    double before, whole;
    int segment;
};

// NV: vectors a thread holds; 0: it holds none and reads them anew in each pass.
template <int DT, int NV>
__global__ void __launch_bounds__(kFThreads, 1) filter_kernel(const FilterArgs a) {
    using R = Row<DT>;
    using E = typename R::E;
    constexpr int N = R::kN;
    __shared__ FilterSmem sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int row = static_cast<int>(blockIdx.x) / C;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const char* const in = a.logits + row * a.stride;

    // a warp has nv runs of 32 vectors, one after the other
    const int nv = NV ? NV : a.per_cta / (kFThreads * N);
    const int warp_first = rank * a.per_cta + warp * nv * 32 * N;
    auto index_of = [&](int j) { return warp_first + (j * 32 + lane) * N; };
    auto load = [&](int j) {
        const int i = index_of(j);
        uint4 v = make_uint4(R::kNegInf, R::kNegInf, R::kNegInf, R::kNegInf);
        if (a.vec_in && i + N <= a.V) return *reinterpret_cast<const uint4*>(in + static_cast<long long>(i) * sizeof(E));
        E* e = reinterpret_cast<E*>(&v);
#pragma unroll
        for (int x = 0; x < N; ++x)
            if (i + x < a.V) e[x] = reinterpret_cast<const E*>(in)[i + x];
        return v;
    };
    uint4 held[NV ? NV : 1];
#pragma unroll
    for (int j = 0; j < NV; ++j) held[j] = load(j);
    // f(vector, index of its first element), in the order of the row within a warp
    auto each = [&](auto&& f) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) f(held[j], index_of(j));
        } else {
#pragma unroll 1
            for (int j = 0; j < nv; ++j) f(load(j), index_of(j));
        }
    };

    // ---- the largest, and what cannot be read ----
    float top = -INFINITY;
    bool bad = false;
    each([&](const uint4& v, int) {
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const float z = R::get(v, x);
            bad |= !(z < INFINITY);
            top = fmaxf(top, z);
        }
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) { sm.warp_top[warp] = top; sm.warp_bad[warp] = bad; }
    cluster.sync();
    for (int r = 0; r < C; ++r) {
        const FilterSmem* o = cluster.map_shared_rank(&sm, r);
        for (int w = 0; w < kFWarps; ++w) {
            top = fmaxf(top, o->warp_top[w]);
            bad |= o->warp_bad[w] != 0;
        }
    }
    const float T = a.temperatures ? a.temperatures[row] : a.temperature, p = a.top_ps ? a.top_ps[row] : a.top_p, m = a.min_ps ? a.min_ps[row] : a.min_p;
    const int k = a.top_ks ? a.top_ks[row] : a.top_k;
    const bool wrong = !(T > 0.f && T < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f);
    bad |= top == -INFINITY || wrong;
    const double scale = 1.4426950408889634073599246810019 / static_cast<double>(T), M = static_cast<double>(top);
    auto weight = [&](float z) { return pow2((static_cast<double>(z) - M) * scale); };
    auto fixed = [&](float z) { return static_cast<unsigned long long>(__double2ull_rn(weight(z) * static_cast<double>(1ull << a.fixed))); };

    Border border{kLowest<DT>, kAll};
    // One digit after the other, from the top: the largest key of which `enough` is true once all larger ones and its own are counted in.
    auto select = [&](bool by_mass, int k, double target_share) {
        const Border among = border;
        uint32_t prefix = 0;
        unsigned above = 0, ties = 0;
        unsigned long long above_mass = 0;
        double target = 0.0;
        constexpr int kLevels = DT == kBF16 ? 2 : 3;
#pragma unroll 1
        for (int level = 0; level < kLevels; ++level) {
            const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, digits = level == 2 ? 1024 : kDigits;
            for (int x = tid; x < kDigits; x += kFThreads) { sm.count[x] = 0; sm.mass[x] = 0; }
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
                        if (by_mass) atomicAdd(&sm.mass[d], fixed(z));
                    }
                }
            });
            cluster.sync();
            // four digits a thread, the largest first
            unsigned c[4], cs = 0;
            unsigned long long w[4], ws = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int d = kDigits - 1 - (4 * tid + x);
                c[x] = 0;
                w[x] = 0;
                for (int r = 0; r < C; ++r) {
                    const FilterSmem* o = cluster.map_shared_rank(&sm, r);
                    c[x] += o->count[d];
                    w[x] += o->mass[d];
                }
                cs += c[x];
                ws += w[x];
            }
            unsigned ci = cs;
            unsigned long long wi = ws;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned cu = __shfl_up_sync(0xffffffffu, ci, o);
                const unsigned long long wu = __shfl_up_sync(0xffffffffu, wi, o);
                if (lane >= o) { ci += cu; wi += wu; }
            }
            if (lane == 31) { sm.scan_count[warp] = ci; sm.scan_mass[warp] = wi; }
            if (tid == 0) sm.found = 0;
            __syncthreads();
            unsigned long long all = 0;
            for (int x = 0; x < kFWarps; ++x) {
                if (x < warp) { ci += sm.scan_count[x]; wi += sm.scan_mass[x]; }
                all += sm.scan_mass[x];
            }
            if (level == 0) target = target_share * static_cast<double>(all);
            unsigned cb = above + ci - cs;
            unsigned long long wb = above_mass + wi - ws;
            // by count: the digit with which k is reached; by mass: the last digit before which there is less than the target
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const bool here = by_mass ? static_cast<double>(wb) < target : cb < static_cast<unsigned>(k);
                if (c[x] > 0 && here) atomicMax(&sm.found, 4u * tid + x + 1);
                cb += c[x];
                wb += w[x];
            }
            __syncthreads();
            const int found = static_cast<int>(sm.found) - 1;         // (there is one: the largest key's)
            if (found >= 4 * tid && found < 4 * tid + 4) {
                cb = above + ci - cs;
                wb = above_mass + wi - ws;
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
            const unsigned long long w = fixed(value_of<DT>(key));
            if (w > 0) {
                double i = ceil((target - static_cast<double>(above_mass)) / static_cast<double>(w));
                if (i < 1.0) i = 1.0;
                if (i < static_cast<double>(ties)) some = static_cast<unsigned>(i);
            }
        }
        border = Border{key, kAll};
        if (some == ties) return;
        // the index of the last of them: ties by warp, then in the warp that has it
        unsigned mine = 0;
        each([&](const uint4& v, int) {
#pragma unroll
            for (int x = 0; x < N; ++x) mine += key_of<DT>(R::get(v, x)) == key;
        });
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == 0) sm.warp_count[warp] = mine;
        cluster.sync();
        unsigned before = 0;
        for (int r = 0; r <= rank; ++r) {
            const FilterSmem* o = cluster.map_shared_rank(&sm, r);
            for (int x = 0; x < (r == rank ? warp : kFWarps); ++x) before += o->warp_count[x];
        }
        if (before < some && before + mine >= some) {
            unsigned need = some - before;
            int last = -1;
            each([&](const uint4& v, int i) {
                unsigned n = 0;
#pragma unroll
                for (int x = 0; x < N; ++x) n += key_of<DT>(R::get(v, x)) == key;
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
                        if (key_of<DT>(R::get(v, x)) == key && --left == 0) last = i + x;
                }
                need = need > all ? need - all : 0;                   // (0: found; no later one is)
            });
            if (last >= 0)
                for (int r = 0; r < C; ++r) cluster.map_shared_rank(&sm, r)->index = last;
        }
        cluster.sync();
        border.last = sm.index;
    };
    if (!bad) {
        if (k > 0 && k < a.V) select(false, k, 0.0);
        if (p == 0.f) select(false, 1, 0.0);
        else if (p < 1.f) select(true, 0, static_cast<double>(p));
        if (m > 0.f) {
            // (the lowest value of the type that is not below)
            float low = __double2float_ru(M + static_cast<double>(T) * log(static_cast<double>(m)));
            if constexpr (DT == kBF16) low = __bfloat162float(__float2bfloat16_ru(low));
            const uint32_t least = key_of<DT>(low);
            if (least > border.key) border = Border{least, kAll};
        }
    }

    // ---- the token ----
    if (a.uniforms) {
        double mine = 0.0;
        if (!bad) {
            each([&](const uint4& v, int i) {
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float z = R::get(v, x);
                    const uint32_t key = key_of<DT>(z);
                    if (key > kLowest<DT> && border.keeps(key, i + x)) mine += weight(z);
                }
            });
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (lane == 0) sm.warp_mass[warp] = mine;
        cluster.sync();
        // every warp: the sums of all warps in order, four a lane
        double s[4], inc = 0.0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int w = 4 * lane + x;
            s[x] = w < C * kFWarps ? cluster.map_shared_rank(&sm, w / kFWarps)->warp_mass[w % kFWarps] : 0.0;
            inc += s[x];
        }
        const double own = inc;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        const double W = __shfl_sync(0xffffffffu, inc, 31);
        double before = __shfl_up_sync(0xffffffffu, inc, 1);
        if (lane == 0) before = 0.0;
        (void)own;
        const double t = static_cast<double>(a.uniforms[row]) * W;
        // the first segment with whose end the border is passed; where rounding leaves none, the last that holds anything
        int seg = -1, last = -1;
        double at = 0.0, at_last = 0.0, c = before;
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
        if (hit) {
            const int src = __ffs(hit) - 1;
            seg = __shfl_sync(0xffffffffu, seg, src);
            at = __shfl_sync(0xffffffffu, at, src);
        } else if (some) {
            const int src = 31 - __clz(some);
            seg = __shfl_sync(0xffffffffu, last, src);
            at = __shfl_sync(0xffffffffu, at_last, src);
        }
        if (bad) {
            if (rank == 0 && tid == 0) {
                a.tokens[row] = -1;
                if (a.lse) a.lse[row] = __int_as_float(0x7fc00000);
            }
        } else if (seg == rank * kFWarps + warp) {
            int found = -1, latest = -1;
            double run = at;
            each([&](const uint4& v, int i) {
                double w[N], n = 0.0;
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const float z = R::get(v, x);
                    const uint32_t key = key_of<DT>(z);
                    w[x] = key > kLowest<DT> && border.keeps(key, i + x) ? weight(z) : 0.0;
                    n += w[x];
                }
                double upto = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double u = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += u;
                }
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
                if (found < 0 && h) found = __shfl_sync(0xffffffffu, here, __ffs(h) - 1);
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
    if (a.out) {
        char* const out = a.out + row * a.out_stride;
        each([&](const uint4& v, int i) {
            uint4 w = v;
            if (wrong) {
                w = make_uint4(R::kNaN, R::kNaN, R::kNaN, R::kNaN);
            } else if (!bad) {
                E* e = reinterpret_cast<E*>(&w);
#pragma unroll
                for (int x = 0; x < N; ++x)
                    if (!border.keeps(key_of<DT>(R::get(v, x)), i + x)) e[x] = static_cast<E>(R::kNegInf >> (32 - 8 * sizeof(E)));
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

template <int DT, int NV>
cudaError_t launch(FilterArgs a, int rows, int C, int nv, cudaStream_t stream) {
    a.per_cta = nv * kFThreads * Row<DT>::kN;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = static_cast<unsigned>(C);
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(rows) * C);
    cfg.blockDim = dim3(kFThreads);
    cfg.stream = stream;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, filter_kernel<DT, NV>, a);
}
template <int DT>
cudaError_t pick(const FilterArgs& a, int rows, int sms, cudaStream_t stream) {
    constexpr int N = Row<DT>::kN, kMost = DT == kF32 ? 16 : 8;
    const long long vecs = (static_cast<long long>(a.V) + N - 1) / N, runs = (vecs + kFThreads - 1) / kFThreads;      // vectors a thread of one CTA would have
    // the fewest CTAs that hold the row, and more where rows are fewer than SMs
    int C = 1;
    while (C < 8 && (runs > static_cast<long long>(C) * kMost || (runs > C && 2LL * C * rows <= sms))) C *= 2;
    const int nv = static_cast<int>((runs + C - 1) / C);
    if (nv <= 1) return launch<DT, 1>(a, rows, C, 1, stream);
    if (nv <= 2) return launch<DT, 2>(a, rows, C, 2, stream);
    if (nv <= 4) return launch<DT, 4>(a, rows, C, 4, stream);
    if (nv <= 8) return launch<DT, 8>(a, rows, C, 8, stream);
    if constexpr (kMost == 16)
        if (nv <= 16) return launch<DT, 16>(a, rows, C, 16, stream);
    return launch<DT, 0>(a, rows, C, nv, stream);
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
    a.fixed = 62;
    while (static_cast<long long>(V) >> (62 - a.fixed)) --a.fixed;      // (a row's sum stays below 2^62)
    a.vec_in = on(logits, 16) && (rows == 1 || a.stride % 16 == 0);
    a.vec_out = on(out_logits, 16) && (rows == 1 || a.out_stride % 16 == 0);
    e = dtype == BV_DTYPE_F32 ? bv::pick<bv::kF32>(a, rows, sms, static_cast<cudaStream_t>(stream)) : bv::pick<bv::kBF16>(a, rows, sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return bv::note_cuda_error(e);
    bv::note_launches(1);
    return BV_OK;
}
