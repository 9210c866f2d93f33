// bv_cache_append_rotary: queries and keys of the newest tokens turned by the angles of their positions, keys and values on into their pages.
//
// A pair (x, y) of a head becomes mscale (x cos a - y sin a, y cos a + x sin a), a = position freq[i].  The angle's turns, position freq / 2 pi, are
// formed and cut down to one turn in 64 bits (at position 10^6 a 32-bit angle is off by 0.03), sine and cosine of the rest in 32
// (with the rest's rounding off by 2^-22 at most, a few roundings of a 32-bit result: rows of 32 bits are off by 3.7e-8 where those of 64-bit sines are by 2.9e-8, rows of
// 16 bits by their own rounding either way); a token's angles are those of all its heads, so a CTA forms them once, in shared memory, while the first vectors of its rows are under way.
//
// Each row is read once and written once (keys twice where they are wanted beside): 17500 tokens of 32 heads on 8, D =
// 128, bf16, 506 MB in 105 us, 4.8 TB/s, reads and writes mixed (memory at 51 %, the SMs at 67 %: a unit's place is worked out for its load and again for its stores); 64 blocks of
// 9 tokens, 64 heads on 8, 7.3 us; 7 blocks of 5, 32 bits, 3.4 us, launch and three trips to memory in a row (offsets, length, page).
#include <cmath>

#include "bv_cache.cuh"
#include "bv_launch.h"

namespace bv {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostTokens = kWarps;        // of a CTA: a warp finds a token's place
constexpr int kAhead = 4;                  // units a thread loads before the angles are there (with 2: 17000 tokens of prompts 117 us, with 4: 105)

struct RotaryArgs {
    const char* src[3];       // q, k_new, v_new
    char* out[2];             // queries, keys (null: not wanted)
    char* pool[2];            // keys, values
    long long ss[3][3];       // bytes between sequences, tokens, heads
    long long os[2][3];
    long long ps[2][3];       // bytes between pages, heads, tokens
    const int32_t* table;
    const int32_t* lens;
    const int32_t* n_new;     // [B] or null: n
    const int32_t* offsets;   // [B + 1] or null: [B, n] rows
    const double* freq;
    long long rows;           // B n, or rows of the packed tensors
    int B, n, Hq, Hkv, page, num_pages, width, half, tokens;
    float mscale;
    int turned, units_turned, units_whole;     // of a head: units that turn; with those that do not; of a value's row
    int units;                // of a token
    Divider by_n, by_page, by_turned, by_whole, by_units;
};

// Where a token is and where it goes.
struct Place {
    long long b, t;           // indices of its rows (packed: 0 and the row)
    int pos, page, slot;      // page -1: not stored
    bool counts;
};

// The sequence that row r of the packed tensors belongs to, the last whose offset is not beyond r, by a warp: a look at 32 offsets a round.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int B, int r, int lane) {
    int lo = 0, hi = B;       // offsets[lo] <= r (or lo is 0), offsets[hi] > r (or hi is B)
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const unsigned upto = __ballot_sync(0xffffffffu, at < hi && __ldg(offsets + at) <= r);
        // (lane 0's offset is known not to be beyond r; where offsets are in no order any answer in range will do)
        const int last = upto ? 31 - __clz(upto) : 0, from = lo + last * step;
        hi = from + step < hi ? from + step : hi;
        lo = from;
    }
    return lo;
}
__device__ __forceinline__ Place place_at(const RotaryArgs& a, long long row, int lane) {
    Place p;
    int b, m, t;
    if (a.offsets) {
        const int r = static_cast<int>(row);
        b = sequence_of(a.offsets, a.B, r, lane);
        const int first = __ldg(a.offsets + b), end = __ldg(a.offsets + b + 1);
        p.counts = first >= 0 && first <= r && r < end;
        m = p.counts ? end - first : 0;
        t = p.counts ? r - first : 0;
        p.b = 0;
        p.t = row;
    } else {
        b = row >> 31 ? static_cast<int>(row / a.n) : a.by_n(static_cast<int>(row));
        t = static_cast<int>(row - static_cast<long long>(b) * a.n);
        m = a.n_new ? brought(__ldg(a.n_new + b), a.n) : a.n;
        p.counts = t < m;
        p.b = b;
        p.t = t;
    }
    const int len = __ldg(a.lens + b);
    // (the position as it comes out, whatever the length is: the queries turn by it; unsigned, so that it wraps instead of overflowing)
    p.pos = static_cast<int>(static_cast<unsigned>(len) - static_cast<unsigned>(m) + static_cast<unsigned>(t));
    const int stored = p.counts ? place_of(len, m, t, a.width, a.page) : -1;
    p.page = -1;
    p.slot = 0;
    if (stored >= 0) {
        const int j = a.by_page(stored), page = __ldg(a.table + static_cast<long long>(b) * a.width + j);
        p.slot = stored - j * a.page;
        if (page >= 0 && page < a.num_pages) p.page = page;
    }
    return p;
}

// V: what a thread moves at a time; E: the element.
template <typename V, typename E> struct Lanes {
    static constexpr int kN = sizeof(V) / sizeof(E);
    static __device__ __forceinline__ void get(const V& v, float (&x)[kN]) {
        if constexpr (sizeof(E) == 4) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = __uint_as_float(w[i]);
        } else {
            const uint16_t* w = reinterpret_cast<const uint16_t*>(&v);
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = __uint_as_float(static_cast<uint32_t>(w[i]) << 16);
        }
    }
    static __device__ __forceinline__ V put(const float (&x)[kN]) {
        V v;
        if constexpr (sizeof(E) == 4) {
            uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
            for (int i = 0; i < kN; ++i) w[i] = __float_as_uint(x[i]);
        } else {
            uint16_t* w = reinterpret_cast<uint16_t*>(&v);
#pragma unroll
            for (int i = 0; i < kN; ++i) w[i] = __bfloat16_as_ushort(__float2bfloat16_rn(x[i]));      // (the one rounding of a result)
        }
        return v;
    }
};

// What a thread does at a time.  A unit that turns is two vectors: those of the pairs' first and second elements, or (pairs side by side) one vector
// that holds both, for single elements two neighbours.  Any other unit is one vector.
struct Unit3 {
    int what, token, head, c;      // what: 0 query, 1 key, 2 value
};
template <typename V, typename E, bool SIDE>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryArgs a) {
    using L = Lanes<V, E>;
    constexpr int N = L::kN;
    constexpr bool kOne = SIDE && N > 1;               // a unit that turns is one vector
    extern __shared__ float2 turns[];                  // [tokens][half] cosine and sine
    __shared__ Place places[kMostTokens];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long first = static_cast<long long>(blockIdx.x) * a.tokens;
    const int here = static_cast<int>(a.rows - first < a.tokens ? a.rows - first : a.tokens);

    const int total = here * a.units;
    auto unit_of = [&](int x) {
        Unit3 u;
        u.token = a.by_units(x);
        const int y = x - u.token * a.units, turning = (a.Hq + a.Hkv) * a.units_turned;
        if (y < turning) {
            const int h = a.by_turned(y);
            u.c = y - h * a.units_turned;
            u.what = h >= a.Hq;
            u.head = h - (u.what ? a.Hq : 0);
        } else {
            const int h = a.by_whole(y - turning);
            u.c = y - turning - h * a.units_whole;
            u.what = 2;
            u.head = h;
        }
        return u;
    };
    auto row_of = [&](const Unit3& u, const long long (&st)[3], long long b, long long t) { return b * st[0] + t * st[1] + u.head * st[2]; };
    // byte offsets of a unit's one or two vectors
    auto vectors_of = [&](const Unit3& u, int& one, int& two) {
        one = two = -1;
        if (u.what == 2) {
            one = u.c;
        } else if (u.c >= a.turned) {
            one = u.c - a.turned + (a.units_whole - (a.units_turned - a.turned));
        } else if (kOne) {
            one = u.c;
        } else if (SIDE) {
            one = 2 * u.c;
            two = one + 1;
        } else {
            one = u.c;
            two = u.c + a.turned;
        }
        one *= static_cast<int>(sizeof(V));
        if (two >= 0) two *= static_cast<int>(sizeof(V));
    };
    // (a token's rows lie where its number says, in either form: its place is not needed to load them)
    auto load = [&](const Unit3& u, V& x, V& y) {
        const long long row = first + u.token;
        long long b = 0, t = row;
        if (!a.offsets) {
            b = row >> 31 ? row / a.n : a.by_n(static_cast<int>(row));
            t = row - b * a.n;
        }
        int one, two;
        vectors_of(u, one, two);
        const char* from = a.src[u.what] + row_of(u, a.ss[u.what], b, t);
        x = *reinterpret_cast<const V*>(from + one);
        if (two >= 0) y = *reinterpret_cast<const V*>(from + two);
    };
    auto finish = [&](const Unit3& u, V x, V y) {
        const Place p = places[u.token];
        if (!p.counts) return;
        int one, two;
        vectors_of(u, one, two);
        if (u.what < 2 && u.c < a.turned) {
            float f[N], g[N];
            L::get(x, f);
            const float2* cs = turns + u.token * a.half;
            if constexpr (kOne) {
#pragma unroll
                for (int i = 0; i < N; i += 2) {
                    const float2 r = cs[u.c * (N / 2) + i / 2];
                    const float s = f[i];
                    f[i] = s * r.x - f[i + 1] * r.y;
                    f[i + 1] = f[i + 1] * r.x + s * r.y;
                }
            } else {
                L::get(y, g);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float2 r = cs[u.c * N + i];
                    const float s = f[i];
                    f[i] = s * r.x - g[i] * r.y;
                    g[i] = g[i] * r.x + s * r.y;
                }
                y = L::put(g);
            }
            x = L::put(f);
        }
        if (u.what < 2 && a.out[u.what]) {
            char* to = a.out[u.what] + row_of(u, a.os[u.what], p.b, p.t);
            *reinterpret_cast<V*>(to + one) = x;
            if (two >= 0) *reinterpret_cast<V*>(to + two) = y;
        }
        if (u.what > 0 && p.page >= 0) {
            const long long(&st)[3] = a.ps[u.what - 1];
            char* to = a.pool[u.what - 1] + p.page * st[0] + u.head * st[1] + p.slot * st[2];
            *reinterpret_cast<V*>(to + one) = x;
            if (two >= 0) *reinterpret_cast<V*>(to + two) = y;
        }
    };

    V x[kAhead], y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (tid + i * kThreads < total) load(unit_of(tid + i * kThreads), x[i], y[i]);
    // A warp a token, or several warps one: each finds the place and forms its share of the angles.
    {
        const int each = kWarps / a.tokens, token = warp / each, part = warp - token * each;      // (tokens is a power of two)
        if (token < here) {
            const Place p = place_at(a, first + token, lane);
            if (part == 0 && lane == 0) places[token] = p;
            for (int i = part * 32 + lane; i < a.half; i += each * 32) {
                const double r = static_cast<double>(p.pos) * (__ldg(a.freq + i) * 0.15915494309189533577);
                float s, c;
                sincospif(2.f * static_cast<float>(r - rint(r)), &s, &c);
                turns[token * a.half + i] = make_float2(c * a.mscale, s * a.mscale);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (tid + i * kThreads < total) finish(unit_of(tid + i * kThreads), x[i], y[i]);
    for (int z = tid + kAhead * kThreads; z < total; z += kThreads) {
        const Unit3 u = unit_of(z);
        load(u, x[0], y[0]);
        finish(u, x[0], y[0]);
    }
}

template <typename V, typename E>
cudaError_t launch(RotaryArgs a, int D, bool side, cudaStream_t stream) {
    constexpr int N = sizeof(V) / sizeof(E);
    const int rot = 2 * a.half;
    a.turned = side && N > 1 ? rot / N : a.half / N;
    a.units_whole = D / N;
    a.units_turned = a.turned + (D - rot) / N;
    a.units = (a.Hq + a.Hkv) * a.units_turned + a.Hkv * a.units_whole;
    a.by_n = divider(a.n);
    a.by_page = divider(a.page);
    a.by_turned = divider(a.units_turned);
    a.by_whole = divider(a.units_whole);
    a.by_units = divider(a.units);
    // tokens of a CTA: as many as fill what its threads load ahead, where there are tokens enough for all SMs
    a.tokens = 1;
    while (a.tokens < kMostTokens && 2 * a.tokens * a.units <= kAhead * kThreads && a.rows >= 148LL * 16 * a.tokens) a.tokens *= 2;
    const long long ctas = (a.rows + a.tokens - 1) / a.tokens;
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    const size_t smem = static_cast<size_t>(a.tokens) * a.half * sizeof(float2);
    if (side) rotary_kernel<V, E, true><<<static_cast<unsigned>(ctas), kThreads, smem, stream>>>(a);
    else rotary_kernel<V, E, false><<<static_cast<unsigned>(ctas), kThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool none_negative(const int64_t* s) { return s[0] >= 0 && s[1] >= 0 && s[2] >= 0; }
bool whole(const void* p, const int64_t* s, int es) { return on(p, 16) && s[0] * es % 16 == 0 && s[1] * es % 16 == 0 && s[2] * es % 16 == 0; }

}  // namespace
}  // namespace bv

extern "C" int bv_cache_append_rotary(const bv_cache* c, const bv_rotary* rotary, const void* q, const int64_t* q_stride, int q_heads, const void* k_new,
                                      const int64_t* k_new_stride, const void* v_new, const int64_t* v_new_stride, const int32_t* n_new, const int32_t* offsets,
                                      int n, void* out_q, const int64_t* out_q_stride, void* out_k, const int64_t* out_k_stride, void* stream) {
    using bv::on;
    if (!c || c->num_pages < 1 || c->page_size < 1 || !c->table || !c->lens || !on(c->table, 4) || !on(c->lens, 4) || c->B < 0 || c->width < 1) return BV_ERR_INVALID_ARG;
    if (c->dtype != BV_DTYPE_F32 && c->dtype != BV_DTYPE_BF16) return BV_ERR_INVALID_ARG;
    const int es = c->dtype == BV_DTYPE_F32 ? 4 : 2;
    if (!c->k || !c->v || c->heads < 1 || c->D < 1 || !on(c->k, es) || !on(c->v, es) || !bv::none_negative(c->k_stride) || !bv::none_negative(c->v_stride)) return BV_ERR_INVALID_ARG;
    if (!rotary || !rotary->freq || !on(rotary->freq, 8) || rotary->rot < 2 || rotary->rot % 2 != 0 || rotary->rot > c->D || !std::isfinite(rotary->mscale)) return BV_ERR_INVALID_ARG;
    if (q_heads < 0 || (q_heads > 0 && (!q || !out_q || !q_stride || !out_q_stride || !on(q, es) || !on(out_q, es) || !bv::none_negative(q_stride) || !bv::none_negative(out_q_stride))))
        return BV_ERR_INVALID_ARG;
    if (!k_new || !v_new || !k_new_stride || !v_new_stride || !on(k_new, es) || !on(v_new, es) || !bv::none_negative(k_new_stride) || !bv::none_negative(v_new_stride)) return BV_ERR_INVALID_ARG;
    if (out_k && (!out_k_stride || !on(out_k, es) || !bv::none_negative(out_k_stride))) return BV_ERR_INVALID_ARG;
    if (n < (offsets ? 0 : 1) || (n_new && offsets) || (n_new && !on(n_new, 4)) || (offsets && !on(offsets, 4))) return BV_ERR_INVALID_ARG;
    if (static_cast<long long>(q_heads) + 2LL * c->heads > 65536 || c->D > 4096) return BV_ERR_UNSUPPORTED;      // (a token's units are counted in 32 bits)
    bv::note_launches(0);
    if (c->B == 0 || n == 0) return BV_OK;
    bv::RotaryArgs a{};
    const void* src[3] = {q, k_new, v_new};
    const int64_t* st[3] = {q_stride, k_new_stride, v_new_stride};
    void* out[2] = {q_heads ? out_q : nullptr, out_k};
    const int64_t* ost[2] = {out_q_stride, out_k_stride};
    // a packed tensor has no stride between sequences
    auto taken = [&](const int64_t* s, int64_t (&to)[3]) {
        for (int i = 0; i < 3; ++i) to[i] = offsets && i == 0 ? 0 : s[i];
    };
    bool vec = bv::on(c->k, 16) && bv::on(c->v, 16) && c->D * es % 16 == 0 && (rotary->interleaved ? rotary->rot : rotary->rot / 2) * es % 16 == 0 &&
               bv::whole(c->k, c->k_stride, es) && bv::whole(c->v, c->v_stride, es);
    for (int i = 0; i < 3; ++i) {
        if (i == 0 && !q_heads) continue;
        int64_t s[3];
        taken(st[i], s);
        vec = vec && bv::whole(src[i], s, es);
        a.src[i] = static_cast<const char*>(src[i]);
        for (int x = 0; x < 3; ++x) a.ss[i][x] = s[x] * es;
    }
    for (int i = 0; i < 2; ++i) {
        if (!out[i]) continue;
        int64_t s[3];
        taken(ost[i], s);
        vec = vec && bv::whole(out[i], s, es);
        a.out[i] = static_cast<char*>(out[i]);
        for (int x = 0; x < 3; ++x) a.os[i][x] = s[x] * es;
    }
    a.pool[0] = static_cast<char*>(c->k); a.pool[1] = static_cast<char*>(c->v);
    for (int i = 0; i < 3; ++i) { a.ps[0][i] = c->k_stride[i] * es; a.ps[1][i] = c->v_stride[i] * es; }
    a.table = c->table; a.lens = c->lens; a.n_new = n_new; a.offsets = offsets; a.freq = rotary->freq;
    a.B = c->B; a.n = n; a.Hq = q_heads; a.Hkv = c->heads; a.page = c->page_size; a.num_pages = c->num_pages; a.width = c->width;
    a.half = rotary->rot / 2;
    a.mscale = rotary->mscale;
    a.rows = offsets ? n : static_cast<long long>(c->B) * n;
    if (a.rows > 0x7fffffffLL) return BV_ERR_UNSUPPORTED;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool side = rotary->interleaved != 0;
    const cudaError_t e = c->dtype == BV_DTYPE_F32 ? (vec ? bv::launch<uint4, uint32_t>(a, c->D, side, s) : bv::launch<uint32_t, uint32_t>(a, c->D, side, s))
                                                   : (vec ? bv::launch<uint4, uint16_t>(a, c->D, side, s) : bv::launch<uint16_t, uint16_t>(a, c->D, side, s));
    if (e != cudaSuccess) return bv::note_cuda_error(e);
    bv::note_launches(1);
    return BV_OK;
}
