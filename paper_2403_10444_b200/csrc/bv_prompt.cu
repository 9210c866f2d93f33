// bv_prompt_attend: the entry point, and the kernel for 32 bits and every shape that the tensor cores do not take (bv_prompt_tiles.cu).
//
// Rows of a key-value head (a token's heads of the group one after the other) are cut into tiles of 64 or 128, a CTA takes one over the keys it
// sees, 64 at a time, with a running maximum and sum for each row: scores by 4 x 4 or 8 x 4 values a thread from shared memory, weights through
// shared memory, results in registers.  Bound by the FMAs of both products and what shared memory has to deliver for them (tiles of 128 read a key's
// values half as often: 4 prompts of 2048 tokens, 32 heads on 8, D = 128: 3.8 ms, 36 TFLOP/s; with tiles of 64 5.0 ms), and where tiles are few by
// the longest one's steps in a row: 7 prompts of up to 701 tokens, 10 heads on 2, D = 80: 172 us, 14 TFLOP/s.
#include <cmath>

#include "bv_launch.h"
#include "bv_prompt.cuh"

namespace bv {
namespace {

constexpr int kK = 64, kPThreads = 256;
constexpr int kPStride = kK + 4;
constexpr float kUnseen = -1.f;                // in the place of a weight: the row does not see the key

struct RowsLayout {
    int q_stride, v_stride;                    // floats
    // (an odd number of 16 bytes between rows: eight rows in a column are in eight different places)
    __host__ __device__ explicit RowsLayout(int D) : q_stride(((D + 3) / 4 | 1) * 4), v_stride((D + 63) / 64 * 64) {}
    __host__ __device__ size_t bytes(int R) const { return sizeof(float) * (static_cast<size_t>(R + kK) * q_stride + static_cast<size_t>(kK) * v_stride + static_cast<size_t>(R) * kPStride); }
};

template <typename E> __device__ __forceinline__ float widen(E x);
template <> __device__ __forceinline__ float widen(float x) { return x; }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename E> __device__ __forceinline__ E narrow(float x);
template <> __device__ __forceinline__ float narrow(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

// A vector to shared memory, widened.
template <typename E>
__device__ __forceinline__ void widen_to(float* to, const uint4& v, int c, int width) {
    const E* e = reinterpret_cast<const E*>(&v);
#pragma unroll
    for (int i = 0; i < 16 / static_cast<int>(sizeof(E)); i += 4)
        if (c + i < width) *reinterpret_cast<float4*>(to + c + i) = make_float4(widen<E>(e[i]), widen<E>(e[i + 1]), widen<E>(e[i + 2]), widen<E>(e[i + 3]));
}

// Rows to shared memory, widened; zero beyond D and beyond `count`.  from(row): its first element.  AHEAD: vectors of a thread under way together, with
// their places counted on: 4 where a CTA is alone on its SM (4 prompts of 2048: 3.98 -> 3.79 ms); with two CTAs the plain loop is the faster (6000 tokens, 4 heads on 1: 1.38 and 1.57 ms).
template <typename E, bool VEC, int AHEAD, typename F>
__device__ __forceinline__ void stage(float* to, int stride, int width, int rows, int count, int D, F from) {
    constexpr int N = 16 / sizeof(E);
    if constexpr (VEC && AHEAD == 1) {
        const int per = (width + N - 1) / N;
        for (int x = threadIdx.x; x < rows * per; x += kPThreads) {
            const int r = x / per, c = (x - r * per) * N;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < count && c < D) v = __ldg(reinterpret_cast<const uint4*>(from(r) + c));      // (D is whole vectors)
            widen_to<E>(to + r * stride, v, c, width);
        }
    } else if constexpr (VEC) {
        const int per = (width + N - 1) / N, step_r = kPThreads / per, step_c = kPThreads - step_r * per;
        int r = threadIdx.x / per, c = threadIdx.x - r * per;
        while (r < rows) {
            uint4 v[AHEAD];
            int rs[AHEAD], cs[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                rs[i] = r;
                cs[i] = c * N;
                v[i] = make_uint4(0, 0, 0, 0);
                if (r < count && c * N < D) v[i] = __ldg(reinterpret_cast<const uint4*>(from(r) + c * N));
                r += step_r;
                c += step_c;
                if (c >= per) { c -= per; ++r; }
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (rs[i] < rows) widen_to<E>(to + rs[i] * stride, v[i], cs[i], width);
        }
    } else {
        for (int x = threadIdx.x; x < rows * width; x += kPThreads) {
            const int r = x / width, c = x - r * width;
            to[r * stride + c] = r < count && c < D ? widen<E>(from(r)[c]) : 0.f;
        }
    }
}

// The CTA's sequence and tile of rows: tiles of all sequences in order, a sequence's last ones (they see the most) first.
template <int kR>
__device__ __forceinline__ bool find_rows(const PromptArgs& a, int x, int* b, int* tile, Prompt* prompt) {
    __shared__ int sums[kPThreads / 32], found[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long before = 0;
    if (tid == 0) found[0] = -1;
    for (int base = 0; base < a.B; base += kPThreads) {
        Prompt p{0, 0};
        if (base + tid < a.B) p = prompt_of(a, base + tid);
        const int n = static_cast<int>((static_cast<long long>(p.length) * a.group + kR - 1) / kR);
        int inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = inc;
        __syncthreads();
        long long upto = before + inc, all = before;
        for (int w = 0; w < kPThreads / 32; ++w) {
            if (w < warp) upto += sums[w];
            all += sums[w];
        }
        if (n > 0 && x < upto && x >= upto - n) {
            found[0] = base + tid;
            found[1] = static_cast<int>(upto - 1 - x);
        }
        __syncthreads();
        if (found[0] >= 0) {
            *b = found[0];
            *tile = found[1];
            *prompt = prompt_of(a, *b);
            return true;
        }
        before = all;
    }
    return false;
}

// NC: 64-column parts of D.  RT: rows of a thread.
template <typename E, bool VEC, int NC, int RT>
__global__ void __launch_bounds__(kPThreads, NC <= 2 && RT == 4 ? 2 : 1) prompt_rows_kernel(const PromptArgs a) {
    constexpr int kR = 16 * RT;                             // a tile's
    extern __shared__ __align__(16) float shared[];
    const RowsLayout lay(a.D);
    float* const sq = shared;
    float* const sk = sq + kR * lay.q_stride;
    float* const sv = sk + kK * lay.q_stride;
    float* const sp = sv + kK * lay.v_stride;
    const int tid = threadIdx.x, tr = tid >> 4, tc = tid & 15;
    int b, tile;
    Prompt s;
    if (!find_rows<kR>(a, static_cast<int>(blockIdx.x / a.Hkv), &b, &tile, &s)) return;
    const int h = blockIdx.x % a.Hkv;
    const int r0 = tile * kR;                               // of length * group rows
    const long long all_rows = static_cast<long long>(s.length) * a.group;
    const int count = all_rows - r0 < kR ? static_cast<int>(all_rows - r0) : kR;
    const int wide = (a.D + 3) / 4 * 4;
    {
        const E* q = static_cast<const E*>(a.q) + s.first * a.qs[0] + h * a.group * a.qs[1];
        stage<E, VEC, RT == 8 ? 4 : 1>(sq, lay.q_stride, wide, kR, count, a.D, [&](int r) { const int t = a.by_group(r0 + r); return q + t * a.qs[0] + (r0 + r - t * a.group) * a.qs[1]; });
    }
    int pos[RT], low[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        pos[i] = a.by_group(r0 + tr * RT + i);
        low[i] = low_of(a, pos[i]);
    }
    const int p0 = a.by_group(r0), p1 = a.by_group(r0 + count - 1), low0 = low_of(a, p0), low1 = low_of(a, p1);
    float m[RT], l[RT], o[RT][NC * 4];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < NC * 4; ++c) o[i][c] = 0.f;
    }
    const E* const k = static_cast<const E*>(a.k) + s.first * a.ks[0] + h * a.ks[1];
    const E* const v = static_cast<const E*>(a.v) + s.first * a.vs[0] + h * a.vs[1];
    for (int start = 0; start <= p1; start += kK) {
        // (what lies between the sinks and the windows is passed over)
        if (start + kK <= low0 && start >= a.sinks) start = low0 / kK * kK;
        const int keys = p1 + 1 - start < kK ? p1 + 1 - start : kK;
        const bool whole = start + kK - 1 <= p0 && (start >= low1 || start + kK <= a.sinks);
        __syncthreads();
        stage<E, VEC, RT == 8 ? 4 : 1>(sk, lay.q_stride, wide, kK, keys, a.D, [&](int j) { return k + (start + j) * a.ks[0]; });
        stage<E, VEC, RT == 8 ? 4 : 1>(sv, lay.v_stride, lay.v_stride, kK, keys, a.D, [&](int j) { return v + (start + j) * a.vs[0]; });
        __syncthreads();
        float x[RT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 2
        for (int d = 0; d < wide; d += 4) {
            float4 qv[RT], kv[4];
#pragma unroll
            for (int i = 0; i < RT; ++i) qv[i] = *reinterpret_cast<const float4*>(sq + (tr * RT + i) * lay.q_stride + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(sk + (tc + 16 * j) * lay.q_stride + d);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[i][j] = fmaf(qv[i].w, kv[j].w, fmaf(qv[i].z, kv[j].z, fmaf(qv[i].y, kv[j].y, fmaf(qv[i].x, kv[j].x, x[i][j]))));
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float top = -INFINITY;
            bool sees[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int p = start + tc + 16 * j;
                sees[j] = whole || (p <= pos[i] && (p >= low[i] || p < a.sinks));
                // (the product is rounded before the reference is taken off, so that scores of any size give weights of at most 1)
                x[i][j] = sees[j] ? __fmul_rn(x[i][j], a.kf) : -INFINITY;
                top = fmaxf(top, x[i][j]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float now = fmaxf(m[i], top), ref = now == -INFINITY ? 0.f : now, scale = ex2(m[i] - ref);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float w = ex2(__fsub_rn(x[i][j], ref));
                sum += sees[j] ? w : 0.f;
                sp[(tr * RT + i) * kPStride + tc + 16 * j] = sees[j] ? w : kUnseen;
            }
            l[i] = l[i] * scale + sum;
#pragma unroll
            for (int c = 0; c < NC * 4; ++c) o[i][c] *= scale;
            m[i] = now;
        }
        __syncwarp();                                       // (a row's weights are its half-warp's)
        auto add = [&](auto checked) {
#pragma unroll 2
            for (int j = 0; j < kK; j += 4) {
                float w[RT][4];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float4 f = *reinterpret_cast<const float4*>(sp + (tr * RT + i) * kPStride + j);
                    w[i][0] = f.x; w[i][1] = f.y; w[i][2] = f.z; w[i][3] = f.w;
                }
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const float4 f = *reinterpret_cast<const float4*>(sv + (j + y) * lay.v_stride + c * 64 + tc * 4);
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            if (decltype(checked)::value && w[i][y] == kUnseen) continue;      // (0 times an infinity is not 0)
                            o[i][c * 4] = fmaf(w[i][y], f.x, o[i][c * 4]);
                            o[i][c * 4 + 1] = fmaf(w[i][y], f.y, o[i][c * 4 + 1]);
                            o[i][c * 4 + 2] = fmaf(w[i][y], f.z, o[i][c * 4 + 2]);
                            o[i][c * 4 + 3] = fmaf(w[i][y], f.w, o[i][c * 4 + 3]);
                        }
                    }
            }
        };
        if (whole) add(std::false_type{});
        else add(std::true_type{});
    }
    E* const out = static_cast<E*>(a.out) + s.first * a.os[0] + h * a.group * a.os[1];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        float sum = l[i];
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        const int r = tr * RT + i;
        if (r >= count) continue;
        const float f = 1.f / sum;                          // (a row without weight: 0 / 0)
        E* to = out + pos[i] * a.os[0] + (r0 + r - pos[i] * a.group) * a.os[1];
#pragma unroll
        for (int c = 0; c < NC * 4; ++c) {
            const int d = c / 4 * 64 + tc * 4 + c % 4;
            if (d < a.D) to[d] = narrow<E>(sum == 0.f ? NAN : o[i][c] * f);
        }
    }
}

// As many CTAs as there may be tiles (one more for each sequence than their rows would fill); those that find none leave.
long long rows_ctas(const PromptArgs& a, int R) { return ((static_cast<long long>(a.tokens) * a.group + R - 1) / R + a.B) * a.Hkv; }

template <typename E, bool VEC, int NC, int RT>
cudaError_t launch_rows(const PromptArgs& a, cudaStream_t stream) {
    static std::atomic<unsigned long long> asked{0};
    constexpr int kR = 16 * RT;
    const size_t bytes = RowsLayout(a.D).bytes(kR);
    const cudaError_t e = allow_shared(prompt_rows_kernel<E, VEC, NC, RT>, static_cast<int>(RowsLayout(NC * 64).bytes(kR)), asked);
    if (e != cudaSuccess) return e;
    const long long ctas = rows_ctas(a, kR);
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    prompt_rows_kernel<E, VEC, NC, RT><<<static_cast<unsigned>(ctas), kPThreads, bytes, stream>>>(a);
    return cudaGetLastError();
}
template <typename E, bool VEC>
cudaError_t pick_rows(const PromptArgs& a, int sms, cudaStream_t stream) {
    // Tiles of 128 rows (one CTA an SM) where every SM gets two or more and a row has more than 64 columns: one prompt of 4096 tokens, 16 heads on 4,
    // D = 128: 2.39 ms by 64 rows, 1.89 by 128; 16 of 300, 32 on 8: 650 and 527 us; D = 96: 1003 and 961 us.  With fewer tiles a wave of them is too
    // long (6000 tokens, 4 heads on 1: 1.39 and 1.48 ms; 7 prompts of up to 701, 10 on 2, D = 80: 171 and 182 us; but 4096 tokens, 8 on 2: 1.23 and
    // 1.01 ms), and up to 64 columns the loads take what the FMAs win (620 and 657 us).
    if constexpr (sizeof(E) == 4 && VEC)
        if (a.D > 64 && a.D <= 128 && rows_ctas(a, 128) - static_cast<long long>(a.B) * a.Hkv >= 2 * sms) return launch_rows<E, VEC, 2, 8>(a, stream);
    return a.D <= 64 ? launch_rows<E, VEC, 1, 4>(a, stream) : a.D <= 128 ? launch_rows<E, VEC, 2, 4>(a, stream) : launch_rows<E, VEC, 4, 4>(a, stream);
}

struct PromptCall {
    PromptArgs a;
    int dtype;
    bool aligned, out_vec, tiles;
    cudaStream_t stream;
};
size_t prompt_scratch(int, const void*) { return 0; }
int enqueue_prompt(const StreamWork& work, void* ctx) {
    PromptCall& c = *static_cast<PromptCall*>(ctx);
    c.a.status = work.status;
    c.a.wait_limit = work.wait_limit;
    c.a.never_signal = work.never_signal;
    cudaError_t e = cudaSuccess;
    bool taken = false;
    if (c.tiles) e = launch_prompt_tiles(c.a, c.out_vec, c.stream, &taken);
    if (e == cudaSuccess && !taken) e = launch_prompt_rows(c.a, c.dtype, c.aligned, work.sm_count, c.stream);
    if (e != cudaSuccess) return note_cuda_error(e);
    note_launches(taken ? prompt_tiles_launches(c.a.B) : 1);
    return BV_OK;
}

}  // namespace

cudaError_t launch_prompt_rows(const PromptArgs& a, int dtype, bool aligned, int sms, cudaStream_t stream) {
    if (dtype == BV_DTYPE_F32) return aligned ? pick_rows<float, true>(a, sms, stream) : pick_rows<float, false>(a, sms, stream);
    return aligned ? pick_rows<__nv_bfloat16, true>(a, sms, stream) : pick_rows<__nv_bfloat16, false>(a, sms, stream);
}

}  // namespace bv

extern "C" int bv_prompt_attend(const void* q, const int64_t* q_stride, const void* k, const int64_t* k_stride, const void* v, const int64_t* v_stride,
                                const int32_t* offsets, int B, int tokens, int q_heads, int heads, int D, int dtype, float scale, int window, int sinks,
                                void* out, const int64_t* out_stride, void* stream) {
    if (dtype != BV_DTYPE_F32 && dtype != BV_DTYPE_BF16) return BV_ERR_INVALID_ARG;
    const int es = dtype == BV_DTYPE_F32 ? 4 : 2;
    const double kf = static_cast<double>(scale) * 1.4426950408889634073599246810019;
    auto on = [](const void* p, size_t x) { return reinterpret_cast<uintptr_t>(p) % x == 0; };
    if (!q || !k || !v || !out || !q_stride || !k_stride || !v_stride || !out_stride || !offsets || B < 0 || tokens < 0 || q_heads < 1 || heads < 1 || q_heads % heads != 0 || D < 1 ||
        window < 0 || sinks < 0 || !std::isfinite(static_cast<float>(kf)) || !on(q, es) || !on(k, es) || !on(v, es) || !on(out, es) || !on(offsets, 4)) return BV_ERR_INVALID_ARG;
    const int64_t* strides[4] = {q_stride, k_stride, v_stride, out_stride};
    for (const int64_t* s : strides)
        if (s[0] < 0 || s[1] < 0) return BV_ERR_INVALID_ARG;
    const long long group = q_heads / heads;
    // (a sequence's rows and its tiles are counted in 32 bits)
    if (D > BV_MAX_HEAD_DIM || tokens > (1 << 30) || B > (1 << 20) || tokens * group > (1LL << 30) || (tokens * group / 64 + 1 + B) * heads > 0x7fffffffLL) return BV_ERR_UNSUPPORTED;
    bv::note_launches(0);
    if (B == 0 || tokens == 0) return BV_OK;
    bv::PromptCall call{};
    bv::PromptArgs& a = call.a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    for (int i = 0; i < 2; ++i) { a.qs[i] = q_stride[i]; a.ks[i] = k_stride[i]; a.vs[i] = v_stride[i]; a.os[i] = out_stride[i]; }
    a.offsets = offsets;
    a.B = B; a.tokens = tokens; a.Hkv = heads; a.group = static_cast<int>(group); a.D = D;
    a.by_group = bv::divider(a.group);
    a.kf = static_cast<float>(kf);
    // (a window that no sequence is longer than is none; so sums with either stay below 2^31)
    a.window = window < tokens ? window : 0;
    a.sinks = a.window == 0 ? 0 : sinks < tokens ? sinks : tokens;
    auto vectors = [&](const void* p, const int64_t* s) { return on(p, 16) && D * es % 16 == 0 && s[0] * es % 16 == 0 && s[1] * es % 16 == 0; };
    call.dtype = dtype;
    call.aligned = vectors(q, q_stride) && vectors(k, k_stride) && vectors(v, v_stride);
    call.out_vec = vectors(out, out_stride);
    call.tiles = dtype == BV_DTYPE_BF16 && call.aligned && bv::prompt_tiles_takes(a);
    call.stream = static_cast<cudaStream_t>(stream);
    return bv::with_stream_work(call.stream, bv::prompt_scratch, bv::enqueue_prompt, &call);
}
