// Softmax cross entropy of token rows against a vocabulary matrix, without the logits in memory, and its gradient:
//   z[t][v] = sum_i x[t][i] W[v][i],  lse[t] = log sum_v exp z[t][v],  loss[t] = lse[t] - z[t][target[t]]
//   g[t][v] = dloss[t] (exp(z[t][v] - lse[t]) - [v == target[t]]),  dx = g W,  dW = g^T x
// (the paper trains language models, Section 5; the loss itself has no counterpart in its text).
//
// All three products run on plane_gemm.cuh.  Tokens whose target is ignore_index are taken out first: a preparation kernel copies
// the rows of x that count to the front of a buffer (fp32: split into three bf16 planes; rows whose length is no multiple of 8
// padded, for TMA), so that nothing is computed for the others and what they hold (NaN, say) reaches no sum.
//   forward   logits tile in tensor memory -> per row the maximum and the sum of exponentials of its 128 columns -> one pair per
//             row and half tile in memory -> a warp per row joins them
//   backward  per piece of the vocabulary: logits again, g as bf16 planes in memory, then dW = g^T x and dx += g W from them.
// Parts of g.  fp32: three bf16 planes, all six plane products.  bf16: dx takes one bf16 plane (2^-8 per term, as much as its own
// rounding), of up to kFewTokens tokens two.  dW is a float32 result: two bf16 planes leave 2^-16 of a term (2.7e-6 of dW's norm at
// 2900 tokens), a third costs a quarter of the call's time.  Two FP16 parts leave 2^-22, and x, bf16, fits fp16 once its exponents
// are near 1.  Tokens are what dW sums over, so each may have a power of two of its own: x' = x 2^-a[t] with the row's largest value
// in [1, 2) (2^126 and more: [1, 4)), g' = g 2^(a[t] - E + 13), E the largest a[t] + exponent of dloss[t], so that every |g'| is below
// 2^14 where exp(z - lse) <= 1; dW = 2^(E - 13) sum g' x'.  What fp16 cannot hold of them is 2^-25 of the row's largest x and 2^-39 of the
// largest |dloss| times the largest x of its row.  Up to kFewTokens tokens take three bf16
// planes: the time goes into reading W and writing dW (64 tokens of d 1024, vocabulary 50257: nothing more; 128: 160 -> 182 us, and dx,
// of so few tokens up to 2.5e-3 off with one plane, is as exact as its type, 1.7e-3).
#include <cuda_fp16.h>

#include "plane_gemm.cuh"

namespace monarch {
namespace tc {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kFewTokens = 128, kBias = 1024;
constexpr int kTokenChunk = 32768;              // tokens whose partial sums are in memory at a time (forward)

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float exp_of(float x) { return ex2(x * kLog2e); }
// maximum and sum of exp(z - maximum) -> log of the sum of exponentials
__device__ __forceinline__ float log_sum(float m, float s) { return fmaf(log2f(s), kLn2, m); }

// ------------------------------------------------------------------------------------------------ preparation
struct PrepArgs {
    const void *x;
    const int64_t *targets;
    const float *lse_in, *dloss;      // backward
    float *loss, *lse;                // forward: zeroed for the rows that are left out
    void *dx;                         // backward: likewise
    int *count, *map, *tgt;           // rows that count; compact row -> row; compact row -> target (-1: out of range)
    float *clse, *cdl;                // backward: lse and dloss of the compact rows
    __half *xh;                       // backward, bf16, many tokens: x' [tokens][dp], a[t], and the largest a[t] + exponent of dloss[t]
    int *exponent, *largest;          // (+ kBias, so that zero is below all)
    __nv_bfloat16 *xp;                // planes [planes][tokens][dp]
    int64_t ignore;
    int tokens, d, dp, vocab, rows_per_cta;
    int ctas;                         // CTAs for the tokens; those behind them split the first piece of W
    const void *W;
    __nv_bfloat16 *wp;
    size_t wplane;
    int wrows;
};

// fp32 value -> bf16 planes.  The largest fp32 values round to infinity in bf16: they are cut instead.
template <int PL> __device__ __forceinline__ void split(float v, __nv_bfloat16 (&o)[PL])
{
    const float inf = __int_as_float(0x7f800000);
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        o[i] = __float2bfloat16_rn(v);
        if (PL > 1 && i == 0 && fabsf(__bfloat162float(o[0])) == inf) o[0] = __float2bfloat16_rz(v);
        v -= __bfloat162float(o[i]);
        if (i == 0 && !(fabsf(v) < inf)) v = 0.0f;             // infinite or NaN: all of it is in the first plane
    }
}

// this warp's part of a row, padded to dp columns
template <typename T, int PL>
__device__ __forceinline__ void copy_row(const T *__restrict__ src, __nv_bfloat16 *dst, size_t plane, int d, int dp, int lane, int part = 0, int parts = 1)
{
    if constexpr (sizeof(T) == 2) {
        if (d == dp) {
#pragma unroll 4
            for (int c = (part * 32 + lane) * 8; c < dp; c += parts * 256) *reinterpret_cast<uint4 *>(dst + c) = __ldg(reinterpret_cast<const uint4 *>(src + c));
            return;
        }
    }
    if constexpr (sizeof(T) == 4) {
        if (d % 4 == 0) {                                   // dp - d is 0 or 4
#pragma unroll 4
            for (int c = (part * 32 + lane) * 4; c < dp; c += parts * 128) {
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (c < d) v = __ldg(reinterpret_cast<const float4 *>(src + c));
                __nv_bfloat16 o[4][PL];
                split<PL>(v.x, o[0]); split<PL>(v.y, o[1]); split<PL>(v.z, o[2]); split<PL>(v.w, o[3]);
#pragma unroll
                for (int i = 0; i < PL; ++i) {
                    __nv_bfloat162 w[2] = {__nv_bfloat162(o[0][i], o[1][i]), __nv_bfloat162(o[2][i], o[3][i])};
                    *reinterpret_cast<uint2 *>(dst + i * plane + c) = *reinterpret_cast<const uint2 *>(w);
                }
            }
            return;
        }
    }
#pragma unroll 4
    for (int c = (part * 32 + lane) * 2; c < dp; c += parts * 64) {
        __nv_bfloat16 a[PL], b[PL];
        split<PL>(c < d ? elem<T>::load(src + c) : 0.0f, a);
        split<PL>(c + 1 < d ? elem<T>::load(src + c + 1) : 0.0f, b);
#pragma unroll
        for (int i = 0; i < PL; ++i) *reinterpret_cast<__nv_bfloat162 *>(dst + i * plane + c) = __nv_bfloat162(a[i], b[i]);
    }
}

// exponent of |v| by its bits: -127 for zero and values below the normal range, 128 for infinities
__device__ __forceinline__ int exponent_of(float v) { return (int)(__float_as_uint(v) >> 23) - 127; }
// v 2^e in two steps, of which each is in the normal range where 2^e need not be
__device__ __forceinline__ float scaled(float v, int e)
{
    const int e1 = max(-126, min(127, e / 2)), e2 = max(-126, min(127, e - e / 2));
    return v * __uint_as_float((uint32_t)(127 + e1) << 23) * __uint_as_float((uint32_t)(127 + e2) << 23);
}

// x' of a row (one warp), its exponent, and its part in E
__device__ __forceinline__ void scaled_row(const __nv_bfloat16 *__restrict__ src, __half *to, int d, int dp, float dl, int *exponent, int *largest, int lane)
{
    float top = 0.0f;
    if (d == dp) {
#pragma unroll 4
        for (int c = lane * 8; c < d; c += 256) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src + c));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
        }
    } else {
        for (int c = lane; c < d; c += 32) top = fmaxf(top, fabsf(__bfloat162float(src[c])));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    const int a = max(-126, min(126, exponent_of(top)));       // 2^-a is in the normal range; x' of the largest rows is below 4
    const float down = __uint_as_float((uint32_t)(127 - a) << 23);
    if (d == dp) {
#pragma unroll 4
        for (int c = lane * 8; c < d; c += 256) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src + c));
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half2 h = __floats2half2_rn(__uint_as_float(w[i] << 16) * down, __uint_as_float(w[i] & 0xffff0000u) * down);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            *reinterpret_cast<uint4 *>(to + c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
        for (int c = lane; c < dp; c += 32) to[c] = __float2half_rn(c < d ? __bfloat162float(src[c]) * down : 0.0f);
    }
    if (lane == 0) {
        *exponent = a;
        if (dl > 0.0f) atomicMax(largest, a + exponent_of(dl) + kBias);
    }
}

template <typename T, int PL, bool BWD>
__global__ void __launch_bounds__(256) xent_prep_kernel(const PrepArgs p)
{
    __shared__ int s_part[2][8], s_dst[256];
    depend_wait();
    depend_launch();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((int)blockIdx.x >= p.ctas) {
        for (int r = ((int)blockIdx.x - p.ctas) * 8 + warp; r < p.wrows; r += ((int)gridDim.x - p.ctas) * 8)
            copy_row<T, PL>((const T *)p.W + (size_t)r * p.d, p.wp + (size_t)r * p.dp, p.wplane, p.d, p.dp, lane);
        return;
    }
    const int first = blockIdx.x * p.rows_per_cta, last = min(p.tokens, first + p.rows_per_cta);
    int before = 0, total = 0;
    for (int t = tid; t < p.tokens; t += 256) {
        const int keep = __ldg(p.targets + t) != p.ignore;
        total += keep;
        before += keep & (t < first);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        before += __shfl_xor_sync(~0u, before, o);
        total += __shfl_xor_sync(~0u, total, o);
    }
    if (lane == 0) { s_part[0][warp] = before; s_part[1][warp] = total; }
    __syncthreads();
    before = total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) { before += s_part[0][w]; total += s_part[1][w]; }
    if (blockIdx.x == 0 && tid == 0) *p.count = total;

    const T *x = (const T *)p.x;
    const size_t plane = (size_t)p.tokens * p.dp;
    for (int base = first; base < last; base += 256) {
        const int t = base + tid;
        int64_t y = p.ignore;
        if (t < last) y = __ldg(p.targets + t);
        const bool keep = t < last && y != p.ignore;
        const unsigned mask = __ballot_sync(~0u, keep);
        __syncthreads();                                     // s_part and s_dst of the rows before are read
        if (lane == 0) s_part[0][warp] = __popc(mask);
        __syncthreads();
        int at = before + __popc(mask & ((1u << lane) - 1)), all = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            all += s_part[0][w];
            if (w < warp) at += s_part[0][w];
        }
        before += all;
        s_dst[tid] = keep ? at : -1;
        if (keep) {
            const bool good = y >= 0 && y < p.vocab;
            p.map[at] = t;
            p.tgt[at] = good ? (int)y : -1;
            if (BWD) {
                p.clse[at] = p.lse_in[t];
                p.cdl[at] = good ? p.dloss[t] : __int_as_float(0x7fffffff);
            }
        } else if (t < last && !BWD) {
            p.loss[t] = 0.0f;
            p.lse[t] = 0.0f;
        }
        __syncthreads();
        // fewer rows than warps: several warps a row
        const int here = min(256, last - base), parts = here >= 8 ? 1 : 8 / here;
        for (int i = warp; i < here * parts; i += 8) {
            const int r = i / parts, part = i - r * parts;
            const int dst = s_dst[r];
            if (dst >= 0)
                copy_row<T, PL>(x + (size_t)(base + r) * p.d, p.xp + (size_t)dst * p.dp, plane, p.d, p.dp, lane, part, parts);
            else if (BWD)
                for (int c = part * 32 + lane; c < p.d; c += parts * 32) elem<T>::store((T *)p.dx + (size_t)(base + r) * p.d + c, 0.0f);
            if (BWD && p.xh != nullptr && part == 0 && dst >= 0)
                scaled_row((const __nv_bfloat16 *)p.x + (size_t)(base + r) * p.d, p.xh + (size_t)dst * p.dp, p.d, p.dp, fabsf(p.dloss[base + r]),
                           p.exponent + dst, p.largest, lane);
            if (BWD && p.xh != nullptr && part == 0 && base + r >= total)
                for (int c = lane; c < p.dp; c += 32) p.xh[(size_t)(base + r) * p.dp + c] = __float2half_rn(0.0f);
            if (base + r >= total)                           // rows behind the last one that counts enter sums over tokens as zeros
                for (int j = 0; j < PL; ++j)
                    for (int c = (part * 32 + lane) * 8; c < p.dp; c += parts * 256)
                        *reinterpret_cast<uint4 *>(p.xp + j * plane + (size_t)(base + r) * p.dp + c) = make_uint4(0, 0, 0, 0);
        }
    }
}

// rows [rows][d] -> planes [PL][rows_max][dp]
template <typename T, int PL>
__global__ void __launch_bounds__(256) split_rows_kernel(const T *__restrict__ W, __nv_bfloat16 *wp, int rows, size_t plane, int d, int dp)
{
    depend_wait();
    depend_launch();
    for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8)
        copy_row<T, PL>(W + (size_t)r * d, wp + (size_t)r * dp, plane, d, dp, threadIdx.x & 31);
}

// ------------------------------------------------------------------------------------------------ epilogues
// Per row and half tile: the maximum m and s = sum exp(z - m).  The difference is taken first: it is exact where z is near m, off by
// 2^-24 of itself where it weighs little, and z log2 e leaves fp32 from 2.36e38 on, where masks by the type's lowest value are.
struct EpiStats {
    static constexpr int kStage = 0;
    struct Args {
        float2 *part;              // [rows of the chunk][2 * column tiles]
        float *tlogit;             // logit of the target
        const int *tgt, *count;
        int row0, cols, v0, halves, half0;
    };
    float m, s;
    int y;
    bool live;
    __device__ __forceinline__ void begin(const Args &a, const PgTile &t)
    {
        m = __int_as_float(0xff800000);
        s = 0.0f;
        live = t.row < *a.count;
        y = live ? a.tgt[t.row] : -1;
    }
    __device__ __forceinline__ void start(const Args &a, const PgTile &t) { y -= a.v0 + t.col; }
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32], PgStage<1> &)
    {
        const int left = a.cols - t.col - c;
        if (left <= 0) return;
        if (left < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i >= left) v[i] = __int_as_float(0xff800000);
        }
        float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int i = 4; i < 32; ++i) top[i & 3] = fmaxf(top[i & 3], v[i]);
        const float nm = fmaxf(fmaxf(m, fmaxf(top[0], top[1])), fmaxf(top[2], top[3]));
        const float base = nm == __int_as_float(0xff800000) ? 0.0f : nm;
        float sum[4] = {s * exp_of(m - base), 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 32; ++i) sum[i & 3] += exp_of(v[i] - base);
        s = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        m = nm;
        const int at = y - c;
        if (live && at >= 0 && at < 32) {
            float z = v[0];
#pragma unroll
            for (int i = 1; i < 32; ++i)
                if (at == i) z = v[i];
            a.tlogit[t.row] = z;
        }
    }
    __device__ __forceinline__ void end(const Args &a, const PgTile &t)
    {
        if (live) a.part[(size_t)(t.row - a.row0) * a.halves + a.half0 + t.half] = make_float2(m, s);
    }
};

// g of a piece of the vocabulary; zeros behind the last row and the last column
// HALF: the bf16 plane for dx, then g' in two fp16 parts for dW; else PL bf16 planes
template <int PL, bool HALF> struct EpiGrad {
    static constexpr int kStage = PL;
    struct Args {
        int cols, v0;
        const int *tgt, *count;
        const float *lse, *dl;
        const int *exponent, *largest;
    };
    float l, dl, dlh;               // dlh: dl 2^(a[t] - E + 13)
    int y, e;
    bool live;
    __device__ __forceinline__ void begin(const Args &a, const PgTile &t)
    {
        live = t.row < *a.count;
        l = live ? a.lse[t.row] : 0.0f;
        dl = live ? a.dl[t.row] : 0.0f;
        y = live ? a.tgt[t.row] : -1;
        if (HALF) e = live ? a.exponent[t.row] - *a.largest : 0;
    }
    __device__ __forceinline__ void start(const Args &a, const PgTile &t)
    {
        y -= a.v0 + t.col;
        if (HALF) {
            dlh = scaled(dl, e + kBias + 13);
        }
    }
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32], PgStage<kStage> &st)
    {
        const int left = live ? a.cols - t.col - c : 0, at = y - c;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float e = exp_of(v[i] - l);
            v[i] = i >= left ? 0.0f : (HALF ? 1.0f : dl) * (at == i ? e - 1.0f : e);
        }
        st.begin();
        if constexpr (HALF) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(dl * v[2 * i], dl * v[2 * i + 1]);
            st.row(0, w);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[2 * i] *= dlh;
                v[2 * i + 1] *= dlh;
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                const float2 f = __half22float2(h);
                v[2 * i] -= f.x;
                v[2 * i + 1] -= f.y;
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            st.row(1, w);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            st.row(2, w);
        } else {
#pragma unroll
            for (int q = 0; q < PL; ++q) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                    if (q + 1 < PL) {
                        v[2 * i] -= __uint_as_float(w[i] << 16);
                        v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                    }
                }
                st.row(q, w);
            }
        }
        st.ready();
#pragma unroll
        for (int q = 0; q < PL; ++q) st.send(q, t.col + c, t.row & ~31, q);
        st.close();
    }
    __device__ __forceinline__ void end(const Args &, const PgTile &) {}
};

// rows of float32, stored or added to
struct EpiStoreF32 {
    static constexpr int kStage = 4;
    struct Args {
        float *out;
        int rows, cols, add;
        int y0;                    // of these rows in the map that TMA writes by; -1: none
        const int *largest;        // E of fp16 parts, or null
        size_t part;               // values of a part of the tokens, where there are several
    };
    int e;
    __device__ __forceinline__ void begin(const Args &a, const PgTile &) { e = a.largest != nullptr ? *a.largest - kBias - 13 : 0; }
    __device__ __forceinline__ void start(const Args &, const PgTile &) {}
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32], PgStage<kStage> &st)
    {
        // times 2^(E - 13); without any weights E is far below
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = scaled(v[i], e);
        if (a.y0 >= 0) {
            if ((t.row & ~31) < a.rows && t.col + c < a.cols) st.tile(v, t.col + c, a.y0 + (t.row & ~31), t.z, a.add);
            return;
        }
        const int col = t.col + c + st.lane, row0 = t.row & ~31, rows = col < a.cols ? a.rows - row0 : 0;
        float *out = a.out + t.z * a.part + (size_t)row0 * a.cols + col;
        st.rows(
            v, [&](int r) { return a.add && r < rows ? out[(size_t)r * a.cols] : 0.0f; },
            [&](int r, float x, float w) {
                if (r < rows) out[(size_t)r * a.cols] = x + w;
            });
    }
    __device__ __forceinline__ void end(const Args &, const PgTile &) {}
};

// dx: the sums of the pieces so far in float32 (compact rows), the last one to the caller's rows
template <typename T> struct EpiDx {
    static constexpr int kStage = 2;
    struct Args {
        float *acc;
        T *dx;
        const int *map, *count;
        int d, first, last;
    };
    int n;
    __device__ __forceinline__ void begin(const Args &a, const PgTile &) { n = *a.count; }
    __device__ __forceinline__ void start(const Args &, const PgTile &) {}
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32], PgStage<kStage> &st)
    {
        const int col = t.col + c + st.lane, row0 = t.row & ~31, rows = col < a.d ? n - row0 : 0;
        float *acc = a.acc + (size_t)row0 * a.d + col;
        st.rows(
            v, [&](int r) { return !a.first && r < rows ? acc[(size_t)r * a.d] : 0.0f; },
            [&](int r, float x, float w) {
                if (r >= rows) return;
                if (a.last) elem<T>::store(a.dx + (size_t)a.map[row0 + r] * a.d + col, x + w);
                else acc[(size_t)r * a.d] = x + w;
            });
    }
    __device__ __forceinline__ void end(const Args &, const PgTile &) {}
};

// dx where a few tiles are split along the vocabulary: a sum per part, over the pieces, in float32
struct EpiDxPart {
    static constexpr int kStage = 4;
    struct Args {
        float *acc;                // [parts][tokens][d]
        const int *count;
        size_t part;
        int d, first, tma;
    };
    int n;
    __device__ __forceinline__ void begin(const Args &a, const PgTile &) { n = *a.count; }
    __device__ __forceinline__ void start(const Args &, const PgTile &) {}
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32], PgStage<kStage> &st)
    {
        if (a.tma) {
            if ((t.row & ~31) < n && t.col + c < a.d) st.tile(v, t.col + c, t.row & ~31, t.z, !a.first);
            return;
        }
        const int col = t.col + c + st.lane, row0 = t.row & ~31, rows = col < a.d ? n - row0 : 0;
        float *acc = a.acc + t.z * a.part + (size_t)row0 * a.d + col;
        st.rows(
            v, [&](int r) { return !a.first && r < rows ? acc[(size_t)r * a.d] : 0.0f; },
            [&](int r, float x, float w) {
                if (r < rows) acc[(size_t)r * a.d] = x + w;
            });
    }
    __device__ __forceinline__ void end(const Args &, const PgTile &) {}
};

// the parts of dx, added up, to the caller's rows
template <typename T>
__global__ void __launch_bounds__(256) xent_dx_kernel(const float *__restrict__ acc, size_t part, const int *__restrict__ splits,
                                                      const int *__restrict__ map, const int *__restrict__ count, T *dx, int d)
{
    depend_wait();
    depend_launch();
    const int n = *count, parts = *splits;
    // four columns at a time where rows allow it, a thread each
    const bool four = d % 4 == 0;
    const int per = four ? d / 4 : d;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)n * per; i += (long long)gridDim.x * 256) {
        const int row = (int)(i / per), c = (int)(i - (long long)row * per);
        const float *in = acc + (size_t)row * d;
        T *out = dx + (size_t)map[row] * d;
        if (four) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
            for (int q = 0; q < parts; ++q) {
                const float4 w = *reinterpret_cast<const float4 *>(in + q * part + 4 * c);
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<uint2 *>(out + 4 * c) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
            else
                *reinterpret_cast<float4 *>(out + 4 * c) = v;
        } else {
            float v = 0.0f;
#pragma unroll 8
            for (int q = 0; q < parts; ++q) v += in[q * part + c];
            elem<T>::store(out + c, v);
        }
    }
}

// the parts of dW, added up (and to what is there); n values, V of them a thread
template <int V>
__global__ void __launch_bounds__(256) xent_dw_kernel(const float *__restrict__ acc, size_t part, const int *__restrict__ splits, float *dW, long long n, int add)
{
    depend_wait();
    depend_launch();
    const int parts = *splits;
    for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * V; i < n; i += (long long)gridDim.x * 256 * V) {
        if constexpr (V == 4) {
            float4 v = add ? *reinterpret_cast<const float4 *>(dW + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
            for (int q = 0; q < parts; ++q) {
                const float4 w = *reinterpret_cast<const float4 *>(acc + q * part + i);
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            *reinterpret_cast<float4 *>(dW + i) = v;
        } else {
            float v = add ? dW[i] : 0.0f;
#pragma unroll 8
            for (int q = 0; q < parts; ++q) v += acc[q * part + i];
            dW[i] = v;
        }
    }
}

// ------------------------------------------------------------------------------------------------ joining the parts
__global__ void __launch_bounds__(256) xent_join_kernel(const float2 *__restrict__ part, const float *__restrict__ tlogit,
                                                        const int *__restrict__ tgt, const int *__restrict__ map,
                                                        const int *__restrict__ count, int row0, int rows, int halves, float *loss, float *lse)
{
    depend_wait();
    depend_launch();
    const int lane = threadIdx.x & 31, n = min(row0 + rows, *count);
    for (int row = row0 + blockIdx.x * 8 + (threadIdx.x >> 5); row < n; row += gridDim.x * 8) {
        const float2 *q = part + (size_t)(row - row0) * halves;
        float m = __int_as_float(0xff800000);
        for (int i = lane; i < halves; i += 32) m = fmaxf(m, q[i].x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
        const float base = m == __int_as_float(0xff800000) ? 0.0f : m;
        float s = 0.0f;
        for (int i = lane; i < halves; i += 32) s += q[i].y * exp_of(q[i].x - base);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        if (lane == 0) {
            const float l = log_sum(m, s);
            const int to = map[row];
            lse[to] = l;
            loss[to] = tgt[row] >= 0 ? l - tlogit[row] : __int_as_float(0x7fffffff);
        }
    }
}

// ------------------------------------------------------------------------------------------------ forward of few tokens
// One launch that reads W once.  Rows of W go straight from memory into the first operand of warp MMAs (a lane's 16 bytes are eight
// consecutive k of one row: the order of k within a chunk of 32 is the same for both operands, so it does not matter), the tokens
// (8 per column tile) wait in shared memory.  The eight warps of a team share 16 rows, an eighth of d each: their sums meet in shared
// memory, the warps take turns to turn them into maximum and sum of exponentials while the others go on.  (A warp to itself for 16
// rows: 3142 groups of a vocabulary of 50257 on 2368 warps are two rounds, the second a third full; 26.5 us for one token of d 1024,
// now 23.2.)  Lanes, warps and, in the last CTA to finish, CTAs are joined.  fp32: three planes of both, six products; there several
// launches are taken before the tile kernels, whose planes of W alone cost as much.  bf16: 41 us on tiles, 29 a launch of 16: one only.
constexpr int kFewMost = 16, kFewTeam = 8;
// 24 warps have 96 KB under way, 16 have 64; fp32 and a second column tile need the registers
__host__ __device__ constexpr int few_threads(int planes, int tiles) { return planes == 1 && tiles == 1 ? 768 : 512; }
__host__ __device__ constexpr int few_teams(int planes, int tiles) { return few_threads(planes, tiles) / 32 / kFewTeam; }
constexpr int64_t kPieceBytes = (int64_t)128 << 20;         // planes of W in a piece of the vocabulary (forward)
constexpr size_t kFewSmem = 223 * 1024;         // of 227 KB, 4 of them static
constexpr int kFewTicket = 16;                  // word of the status area, zero between calls

int few_row(int d) { return ((d * 2 + 127) / 128 * 128 + 64) / 2; }             // rows 64 bytes apart in their banks
int few_tiles(int tokens) { return tokens <= 8 ? 1 : 2; }                       // column tiles of 8 tokens: what the kernels are built for
size_t few_x(int tokens, int d, int planes) { return (size_t)tokens * few_row(d) * 2 * planes; }
size_t few_smem(int tokens, int d, int planes) { return few_x(tokens, d, planes) + (size_t)few_teams(planes, few_tiles(tokens)) * 2 * kFewTeam * few_tiles(tokens) * 512; }
// Launches of few tokens that the call takes; 0: tiles.  fp32, us of n launches (on tiles):
//   forward   two always: d 1024, vocabulary 50257 144 (224), 512, 2000 27 (29), 4096, 32768 282 (590), 8192, 16384 306 (565)
//             three where a launch holds up to 8 tokens: 4096, 32768 419 (589), 4096, 2000 91 (98), 8192, 1000 139 (168)
//             or where W is more than one piece of the tile kernels: 1024, 50257 212 (226), 2048, 32768 269 (316), 2560, 20000 245 (278);
//             else not: 1024, 16000 102 (83), 512, 8000 49 (36), 2048, 4000 76 (65)
//             four: 4096, 32768 557 (589), but 4096, 4000 129 (123), 8192, 16384 604 (565), 2048, 32768 342 (314)
//   backward  two: 1024, 50257 381 (473), 512, 2000 42 (60), 4096, 32768 764 (973), 8192, 16384 805 (975)
//             three: 1024, 50257 571 (473), 4096, 32768 1135 (979)
// Rows of other than 16-byte multiples are read value by value, up to 16 tokens (5 tokens, d 1018, 50257: bf16 48 (109) and 188 (322), fp32
// 69 (273) and 157 (554); 3 tokens, d 3661, 57446, fp32: 238 (1410) and 588 (2058))
int few_launches(int64_t tokens, int d, int vocab, int dtype, bool bwd)
{
    const bool f32 = dtype == MONARCH_F32, again = f32 && d % 8 == 0;
    if (tokens > (again ? 3 : 1) * kFewMost) return 0;
    int most = kFewMost;
    while (most > 0 && few_smem(most, d, f32 ? 3 : 1) > kFewSmem) --most;
    if (most == 0) return 0;
    const bool pieces = (int64_t)vocab * d * 6 > kPieceBytes;
    const int n = ((int)tokens + most - 1) / most, limit = !f32 ? 1 : bwd || !again ? 2 : most <= 8 || pieces ? 3 : 2;
    return n <= limit ? n : 0;
}

struct FewArgs {
    const void *x, *W;
    const int64_t *targets;
    float *loss, *lse, *tlogit;
    float2 *part;                               // [tokens][CTAs]
    unsigned *ticket;
    const float *lse_in, *dloss;                // backward: g [vocab][8 or 16] in place of loss and lse
    float *g;
    int64_t ignore;
    int tokens, d, vocab, row;
};

__device__ __forceinline__ void join(float &m, float &s, float m2, float s2)
{
    const float n = fmaxf(m, m2), base = n == __int_as_float(0xff800000) ? 0.0f : n;
    s = s * exp_of(m - base) + s2 * exp_of(m2 - base);
    m = n;
}

// eight consecutive values of a row of W, and the planes of their pairs as MMA operands
template <typename T> struct FewRaw;
template <> struct FewRaw<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool in) { v = in ? __ldcs(reinterpret_cast<const uint4 *>(p)) : make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load_some(const __nv_bfloat16 *p, int n)                       // the first n of them, at any address
    {
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? (uint32_t)__ldg(q + 2 * i) : 0u) | (2 * i + 1 < n ? (uint32_t)__ldg(q + 2 * i + 1) << 16 : 0u);
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void planes(uint32_t (&o)[1][4]) const { o[0][0] = v.x; o[0][1] = v.y; o[0][2] = v.z; o[0][3] = v.w; }
};
template <> struct FewRaw<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p, bool in)
    {
        a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (in) {
            a = __ldcs(reinterpret_cast<const float4 *>(p));
            b = __ldcs(reinterpret_cast<const float4 *>(p + 4));
        }
    }
    __device__ __forceinline__ void load_some(const float *p, int n)
    {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? __ldg(p + i) : 0.0f;
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void planes(uint32_t (&o)[3][4]) const
    {
        const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat16 x[3], y[3];
            split<3>(f[2 * i], x);
            split<3>(f[2 * i + 1], y);
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                const __nv_bfloat162 w(x[q], y[q]);
                o[q][i] = *reinterpret_cast<const uint32_t *>(&w);
            }
        }
    }
};

// ODD: rows of W are not 16-byte multiples
template <typename T, int PL, int NT, bool BWD, bool ODD>
__global__ void __launch_bounds__(few_threads(PL, NT), 1) xent_few_kernel(const FewArgs p)
{
    constexpr int kFewThreads = few_threads(PL, NT), kFewTeams = few_teams(PL, NT);
    extern __shared__ __align__(16) __nv_bfloat16 xs[];                        // [PL][tokens][row], then the sums
    __shared__ float2 s_part[kFewThreads / 32][8 * NT];
    __shared__ int s_tgt[8 * NT], s_last;
    __shared__ float s_lse[8 * NT], s_dl[8 * NT];
    constexpr int kStep = sizeof(T) == 2 ? 4 : 2;                               // chunks of 32 requested ahead
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const size_t xplane = (size_t)p.tokens * p.row;
    const int chunks = (p.d + 31) / 32;
    const int team = warp / kFewTeam, member = warp % kFewTeam;
    // this warp's chunks, in steps of kStep
    const int each = (chunks + kFewTeam - 1) / kFewTeam, k0 = min(member * each, chunks), k1 = min(k0 + each, chunks), steps = (each + kStep - 1) / kStep;
    // this team's rows: as many as every other's, the last group of 16 may be part of one (3142 groups on 296 teams are 10 or 11 each)
    const int teams = gridDim.x * kFewTeams, rows = (p.vocab + teams - 1) / teams;
    const int row0 = min((int)(blockIdx.x * kFewTeams + team) * rows, p.vocab), row1 = min(row0 + rows, p.vocab), groups = (row1 - row0 + 15) / 16;
    FewRaw<T> raw[kStep][2];
    auto fetch = [&](int grp, int step) {
        const int r = row0 + grp * 16 + g;
        const T *w = (const T *)p.W + (size_t)r * p.d;
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
            const int k = k0 + step * kStep + u, at = k * 32 + c * 8;
            const bool in = k < k1 && at < p.d;
            if constexpr (ODD) {
                raw[u][0].load_some(w + at, in && r < row1 ? p.d - at : 0);
                raw[u][1].load_some(w + (size_t)8 * p.d + at, in && r + 8 < row1 ? p.d - at : 0);
            } else {
                raw[u][0].load(w + at, in && r < row1);
                raw[u][1].load(w + (size_t)8 * p.d + at, in && r + 8 < row1);
            }
        }
    };
    depend_wait();
    depend_launch();
    fetch(0, 0);                                                           // on its way while the tokens are prepared
    if (threadIdx.x < 8 * NT && (int)threadIdx.x >= p.tokens) s_tgt[threadIdx.x] = -2;
    const int parts = kFewThreads / 32 / p.tokens;                             // warps a token; tokens <= 16
    if (const int t = warp / parts; t < p.tokens) {
        const int part = warp - t * parts;
        const int64_t y = p.targets[t];
        const bool keep = y != p.ignore;
        if (lane == 0 && part == 0) {
            const bool good = y >= 0 && y < p.vocab;
            s_tgt[t] = !keep ? -2 : good ? (int)y : -1;
            if (BWD) {
                s_lse[t] = p.lse_in[t];
                s_dl[t] = good ? p.dloss[t] : __int_as_float(0x7fffffff);
            }
        }
#pragma unroll 4
        for (int k = (part * 32 + lane) * 2; k < p.row; k += parts * 64) {
            __nv_bfloat16 a[PL], b[PL];
            const T *src = (const T *)p.x + (size_t)t * p.d + k;
            const float v0 = k < p.d ? elem<T>::load(src) : 0.0f, v1 = k + 1 < p.d ? elem<T>::load(src + 1) : 0.0f;
            split<PL>(keep ? v0 : 0.0f, a);
            split<PL>(keep ? v1 : 0.0f, b);
#pragma unroll
            for (int q = 0; q < PL; ++q) *reinterpret_cast<__nv_bfloat162 *>(xs + q * xplane + (size_t)t * p.row + k) = __nv_bfloat162(a[q], b[q]);
        }
    }
    __syncthreads();
    int tgt[NT][2];
    float m[NT][2], s[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            tgt[n][e] = s_tgt[n * 8 + 2 * c + e];
            m[n][e] = __int_as_float(0xff800000);
            s[n][e] = 0.0f;
        }
    const __nv_bfloat16 *xl = xs + (size_t)g * p.row + c * 8;
    float *sums = reinterpret_cast<float *>(xs + PL * xplane) + team * 2 * kFewTeam * NT * 128;      // [2][team][NT][4][32 lanes]
    int turn = 0;
    for (int grp = 0; grp < groups; ++grp, ++turn) {
        float z[NT][4] = {}, low[NT][4] = {}, sum[NT][4] = {};          // low: the products of other than the first planes (fp32)
        for (int step = 0; step < steps; ++step) {
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                const int k = k0 + step * kStep + u;
                if (k >= k1) break;
                uint32_t a0[PL][4], a1[PL][4];
                raw[u][0].planes(a0);
                raw[u][1].planes(a1);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 b[PL];
#pragma unroll
                    for (int q = 0; q < PL; ++q)                                   // columns without a token: zeros
                        b[q] = n * 8 + g < p.tokens ? *reinterpret_cast<const uint4 *>(xl + q * xplane + (size_t)n * 8 * p.row + k * 32) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int o = PL - 1; o >= 0; --o)
#pragma unroll
                        for (int q = o; q >= 0; --q) {
                            const uint32_t f0[4] = {a0[q][0], a1[q][0], a0[q][1], a1[q][1]}, f1[4] = {a0[q][2], a1[q][2], a0[q][3], a1[q][3]};
                            float(&to)[4] = o > 0 ? low[n] : z[n];
                            mma(to, f0, b[o - q].x, b[o - q].y);
                            mma(to, f1, b[o - q].z, b[o - q].w);
                        }
                }
            }
            fetch(step + 1 < steps ? grp : grp + 1, step + 1 < steps ? step + 1 : 0);
            if (step % 4 == 3)                                                    // runs of at most 32 products (plane_gemm.cuh)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { sum[n][e] += z[n][e]; z[n][e] = 0.0f; }
        }
        float *mine = sums + (turn & 1) * kFewTeam * NT * 128;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[((member * NT + n) * 4 + e) * 32 + lane] = sum[n][e] + z[n][e] + low[n][e];
        asm volatile("bar.sync %0, 256;" ::"r"(team + 1) : "memory");
        // this buffer is written again two groups on, behind the next barrier, which its reader reaches when it has read
        if (turn % kFewTeam != member) continue;
        const int r0 = row0 + grp * 16 + g, r1 = r0 + 8;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float t[4] = {};
#pragma unroll
            for (int w = 0; w < kFewTeam; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] += mine[((w * NT + n) * 4 + e) * 32 + lane];
#pragma unroll
            for (int e = 0; e < 2 && BWD; ++e) {
                const int at = n * 8 + 2 * c + e;
                const float l = s_lse[at], dl = s_dl[at];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float x = exp_of(t[e + 2 * h] - l);
                    t[e + 2 * h] = tgt[n][e] == -2 ? 0.0f : dl * (tgt[n][e] == r0 + 8 * h ? x - 1.0f : x);
                }
            }
            if (BWD) {
                float *to = p.g + (size_t)r0 * (8 * NT) + n * 8 + 2 * c;
                if (r0 < row1) *reinterpret_cast<float2 *>(to) = make_float2(t[0], t[1]);
                if (r1 < row1) *reinterpret_cast<float2 *>(to + 64 * NT) = make_float2(t[2], t[3]);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float z0 = t[e], z1 = t[e + 2];
                if (r0 == tgt[n][e] && r0 < row1) p.tlogit[n * 8 + 2 * c + e] = z0;
                if (r1 == tgt[n][e] && r1 < row1) p.tlogit[n * 8 + 2 * c + e] = z1;
                const float v0 = r0 < row1 ? z0 : __int_as_float(0xff800000), v1 = r1 < row1 ? z1 : __int_as_float(0xff800000);
                const float top = fmaxf(m[n][e], fmaxf(v0, v1)), base = top == __int_as_float(0xff800000) ? 0.0f : top;
                s[n][e] = s[n][e] * exp_of(m[n][e] - base) + exp_of(v0 - base) + exp_of(v1 - base);
                m[n][e] = top;
            }
        }
    }
    if (BWD) return;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) join(m[n][e], s[n][e], __shfl_xor_sync(~0u, m[n][e], o), __shfl_xor_sync(~0u, s[n][e], o));
            if (g == 0) s_part[warp][n * 8 + 2 * c + e] = make_float2(m[n][e], s[n][e]);
        }
    __syncthreads();
    if (threadIdx.x < (unsigned)p.tokens) {
        float2 v = s_part[0][threadIdx.x];
        for (int w = 1; w < kFewThreads / 32; ++w) join(v.x, v.y, s_part[w][threadIdx.x].x, s_part[w][threadIdx.x].y);
        p.part[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = v;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
        if (s_last) *p.ticket = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    for (int t = warp; t < p.tokens; t += kFewThreads / 32) {
        float mm = __int_as_float(0xff800000), ss = 0.0f;
        for (int i = lane; i < (int)gridDim.x; i += 32) {
            const float2 v = __ldcg(p.part + (size_t)t * gridDim.x + i);
            join(mm, ss, v.x, v.y);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) join(mm, ss, __shfl_xor_sync(~0u, mm, o), __shfl_xor_sync(~0u, ss, o));
        if (lane == 0) {
            const int y = s_tgt[t];
            const float l = log_sum(mm, ss);
            p.lse[t] = y == -2 ? 0.0f : l;
            p.loss[t] = y == -2 ? 0.0f : y >= 0 ? l - __ldcg(p.tlogit + t) : __int_as_float(0x7fffffff);
        }
    }
}

// ------------------------------------------------------------------------------------------------ gradients of few tokens
// With g [vocab][8 or 16] from the kernel above: dW = g^T x and dx = g W in one pass over W and dW, in fp32 FMAs packed over pairs of
// tokens (dW takes (g, g') (x, x') and adds the halves at the end, dx (g, g') (w, w)).  A lane keeps x and the sums of dx for its columns
// (4, of 16 tokens 2) in registers; a warp takes eight rows at a time (fp32: 4, for the registers: 186 -> 141 us of a call), asks for the
// next as it goes, and its values of g wait in shared memory.  The eight warps' and then the CTAs' sums of dx are added in a fixed order.
// d 1024, a vocabulary of 50257, us of this kernel (of the call; on tiles): 8 tokens bf16 65 (93; 153) = 309 MB at 4.7 TB/s, fp32 76
// (142; 452) = 412 MB at 5.4 TB/s, both bound by memory; 16 tokens bf16 110 (140; 153), fp32 122 (184; 454), bound by the FMAs.
template <typename T> constexpr int kFewRows = sizeof(T) == 2 ? 8 : 4;           // of a warp's step

struct FewGradArgs {
    const void *x, *W;
    const int64_t *targets;
    const float *g;
    float *dW, *part;                           // part: [parts][tokens][d]
    int64_t ignore;
    int tokens, d, vocab, rows, accumulate;     // rows of W per CTA
};

// C consecutive values
template <typename T, int C> struct FewCols;
template <int C> struct FewCols<__nv_bfloat16, C> {
    uint32_t v[C / 2];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool in)
    {
        if constexpr (C == 4) {
            const uint2 w = in ? __ldcs(reinterpret_cast<const uint2 *>(p)) : make_uint2(0, 0);
            v[0] = w.x; v[1] = w.y;
        } else {
            v[0] = in ? __ldcs(reinterpret_cast<const uint32_t *>(p)) : 0u;
        }
    }
    __device__ __forceinline__ void load_apart(const __nv_bfloat16 *p, int n)          // value i at p + 32 i, where that is below n
    {
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < C; i += 2) v[i / 2] = (32 * i < n ? (uint32_t)__ldg(q + 32 * i) : 0u) | (32 * (i + 1) < n ? (uint32_t)__ldg(q + 32 * (i + 1)) << 16 : 0u);
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16); }
};
template <int C> struct FewCols<float, C> {
    float2 v[C / 2];
    __device__ __forceinline__ void load(const float *p, bool in)
    {
        if constexpr (C == 4) {
            const float4 w = in ? __ldcs(reinterpret_cast<const float4 *>(p)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            v[0] = make_float2(w.x, w.y); v[1] = make_float2(w.z, w.w);
        } else {
            v[0] = in ? __ldcs(reinterpret_cast<const float2 *>(p)) : make_float2(0.0f, 0.0f);
        }
    }
    __device__ __forceinline__ void load_apart(const float *p, int n)
    {
#pragma unroll
        for (int i = 0; i < C; i += 2) v[i / 2] = make_float2(32 * i < n ? __ldg(p + 32 * i) : 0.0f, 32 * (i + 1) < n ? __ldg(p + 32 * (i + 1)) : 0.0f);
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? v[i / 2].y : v[i / 2].x; }
};

// ODD: rows are not 16-byte multiples; a lane's columns are 32 apart, its loads and stores single values
template <typename T, int TP, bool ODD>
__global__ void __launch_bounds__(256, 2) xent_few_grad_kernel(const FewGradArgs p)
{
    constexpr int R = kFewRows<T>, C = 32 / TP, G = R * TP / 32;               // columns of a lane, values of g it fetches
    __shared__ __align__(16) float s_g[8][R][TP];
    __shared__ float s_dx[TP][32 * C];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, apart = ODD ? 32 : 1, at0 = ODD ? lane : lane * C;
    const int col = blockIdx.x * 32 * C + at0;                                 // this lane's first column, the others `apart`
    const bool live = col < p.d;                                               // not ODD: d % 8 == 0
    const int row0 = blockIdx.y * p.rows, row1 = min(row0 + p.rows, p.vocab);
    depend_wait();
    depend_launch();
    FewCols<T, C> w[R];
    float g[G];
    const int r_g = lane * G / TP;                                             // the row of this lane's values of g
    auto fetch_g = [&](int r) {
        const float *from = p.g + (size_t)r * TP + lane * G;
        const bool in = r + r_g < row1;
        if constexpr (G == 4) {
            const float4 v = in ? *reinterpret_cast<const float4 *>(from) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            g[0] = v.x; g[1] = v.y; g[2] = v.z; g[3] = v.w;
        } else if constexpr (G == 1) {
            g[0] = in ? *from : 0.0f;
        } else {
            const float2 v = in ? *reinterpret_cast<const float2 *>(from) : make_float2(0.0f, 0.0f);
            g[0] = v.x; g[1] = v.y;
        }
    };
    auto fetch = [&](FewCols<T, C> &v, const T *row, bool in) {
        if constexpr (ODD) v.load_apart(row + col, in ? p.d - col : 0);
        else v.load(row + col, in && live);
    };
    auto fetch_w = [&](int r, int u) { fetch(w[u], (const T *)p.W + (size_t)(r + u) * p.d, r + u < row1); };
    int r = row0 + warp * R;
#pragma unroll
    for (int u = 0; u < R; ++u) fetch_w(r, u);
    fetch_g(r);
    f32x2 x[TP / 2][C], dx[TP / 2][C];                                         // pairs of tokens
#pragma unroll
    for (int t = 0; t < TP; t += 2) {
        FewCols<T, C> v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            fetch(v[k], (const T *)p.x + (size_t)(t + k) * p.d, t + k < p.tokens && p.targets[t + k < p.tokens ? t + k : 0] != p.ignore);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[t / 2][c] = pack2(v[0].at(c), v[1].at(c));
            dx[t / 2][c] = pack2(0.0f, 0.0f);
        }
    }
    for (; r < row1; r += 8 * R) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < G; ++i) s_g[warp][r_g][lane * G % TP + i] = g[i];
        __syncwarp();
        fetch_g(r + 8 * R);
#pragma unroll
        for (int u = 0; u < R; ++u) {
            f32x2 v[C], o[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float f = w[u].at(c);
                v[c] = pack2(f, f);
                o[c] = pack2(0.0f, 0.0f);
            }
            fetch_w(r + 8 * R, u);
#pragma unroll
            for (int t = 0; t < TP / 2; t += 2) {
                const ulonglong2 gg = *reinterpret_cast<const ulonglong2 *>(&s_g[warp][u][2 * t]);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    o[c] = fma2(gg.x, x[t][c], o[c]);
                    dx[t][c] = fma2(gg.x, v[c], dx[t][c]);
                    o[c] = fma2(gg.y, x[t + 1][c], o[c]);
                    dx[t + 1][c] = fma2(gg.y, v[c], dx[t + 1][c]);
                }
            }
            if (live && r + u < row1) {
                float *to = p.dW + (size_t)(r + u) * p.d + col;
                float f[C];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const float2 h = unpack2(o[c]);
                    f[c] = h.x + h.y;
                }
                if constexpr (ODD) {
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        if (col + 32 * c < p.d) {
                            if (p.accumulate) atomicAdd(to + 32 * c, f[c]);
                            else __stcs(to + 32 * c, f[c]);
                        }
                } else if (p.accumulate) {                                     // one addition of one thread to each value; nothing waits for it
                    if constexpr (C == 4)
                        asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(to), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
                    else
                        asm volatile("red.relaxed.gpu.global.add.v2.f32 [%0], {%1, %2};" ::"l"(to), "f"(f[0]), "f"(f[1]) : "memory");
                } else if constexpr (C == 4) {
                    __stcs(reinterpret_cast<float4 *>(to), make_float4(f[0], f[1], f[2], f[3]));
                } else {
                    __stcs(reinterpret_cast<float2 *>(to), make_float2(f[0], f[1]));
                }
            }
        }
    }
    for (int q = 0; q < 8; ++q) {
        if (warp == q)
#pragma unroll
            for (int t = 0; t < TP; t += 2)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float2 v = unpack2(dx[t / 2][c]);
                    float *to = &s_dx[t][at0 + apart * c];
                    if (q > 0) { v.x += to[0]; v.y += to[32 * C]; }
                    to[0] = v.x;
                    to[32 * C] = v.y;
                }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < p.tokens * 32 * C; i += 256) {
        const int t = i / (32 * C), c = blockIdx.x * 32 * C + i % (32 * C);
        if (c < p.d) p.part[((size_t)blockIdx.y * p.tokens + t) * p.d + c] = s_dx[t][i % (32 * C)];
    }
}

// the CTAs' sums: a CTA per 32 columns of a token, eight warps an eighth of the parts each
template <typename T>
__global__ void __launch_bounds__(256) xent_few_dx_kernel(const float *part, const int64_t *targets, int64_t ignore, T *dx, int tokens, int d, int parts)
{
    __shared__ float s[8][32];
    depend_wait();
    depend_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane, t = blockIdx.y;
    const size_t step = (size_t)tokens * d;
    const float *in = part + (size_t)t * d + c;
    float v = 0.0f;
    if (c < d)
#pragma unroll 8
        for (int q = warp; q < parts; q += 8) v += in[q * step];
    s[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || c >= d) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) v += s[q][lane];
    elem<T>::store(dx + (size_t)t * d + c, targets[t] == ignore ? 0.0f : v);
}

// ------------------------------------------------------------------------------------------------ host side
size_t up(size_t v) { return (v + 255) & ~(size_t)255; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

constexpr size_t kHead = MONARCH_STATUS_BYTES + 65536;      // the status area and the counters of kernels that may share the workspace
constexpr int kPairs = kPgPairs;

struct Layout {
    bool direct;                                // W is read where it is (bf16 rows of 16-byte multiples)
    int planes, gplanes, dp, piece;             // planes of x and W, of g; padded row; vocabulary entries per piece
    int chunk, halves, trows;
    int tn, tn_dw, tn_dx;                       // columns of a tile: logits, dW, dx
    int dx_parts, dw_parts;                     // most parts of the vocabulary in dx, of the tokens in dW; 1: no parts
    bool half;                                  // dW from fp16 parts
    size_t count, splits, largest, exponent, xh, map, tgt, lse, dl, tlogit, x, w, part, g, dx, dw_splits, dw, total;
};

// Vocabulary entries per piece of the backward pass: whole 256-entry tiles, a plane of g within 160 MB, and
// as few rounds of the pairs over the tiles of the three products as can be had.
int bwd_piece(int64_t tokens, int d, int vocab)
{
    const int mt = tokens > 0 ? ceil_div(tokens, 256) : 1, nt = ceil_div(d, 256), vt = ceil_div(vocab, 256);
    int most = (int)(((size_t)160 << 20) / ((size_t)mt * 256 * 256 * 2));
    most = most < 1 ? 1 : most > vt ? vt : most;
    int best = most;
    double best_cost = 1e300;
    const int fewest = ceil_div(vt, most);
    for (int pieces = fewest; pieces < fewest + 16 && pieces <= vt; ++pieces) {
        const int k = ceil_div(vt, pieces);
        double cost = 0.0;
        for (int left = vt, n = 0; left > 0 && n < 2; ++n) {                  // the full pieces, then the last one
            const int now = left < k ? left : k, times = left < k ? 1 : left / k;
            const double z = (double)ceil_div((int64_t)mt * now, kPairs) * nt, w = (double)ceil_div((int64_t)now * nt, kPairs) * mt * 2,
                         x = (double)ceil_div((int64_t)mt * nt, kPairs) * now;
            cost += times * (z + w + x + 24.0);                               // in tiles of 256 of K; a piece costs some 10 us
            left -= times * now;
        }
        if (cost < best_cost) { best_cost = cost; best = k; }
    }
    return best * 256;
}

// Where everything stands, by the choices in `l`
void place(Layout &l, int64_t tokens, int d, int vocab, bool bwd)
{
    // half tiles of all pieces
    l.halves = 2 * (vocab / l.piece * ceil_div(l.piece, l.tn) + ceil_div(vocab % l.piece, l.tn));
    size_t at = kHead;
    auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes); return o; };
    const size_t t = (size_t)tokens;
    l.count = take(4);
    l.splits = take(4);
    l.largest = take(4);
    l.exponent = l.xh = 0;
    if (l.half) {
        l.exponent = take(t * 4);
        l.xh = take(t * l.dp * 2);
    }
    l.map = take(t * 4);
    l.tgt = take(t * 4);
    l.lse = l.dl = l.tlogit = l.part = l.g = l.dx = 0;
    if (bwd) { l.lse = take(t * 4); l.dl = take(t * 4); }
    else l.tlogit = take(t * 4);
    l.x = take(t * l.dp * 2 * l.planes);
    l.w = l.direct ? 0 : take((size_t)l.piece * l.dp * 2 * l.planes);
    if (bwd) {
        l.g = take((size_t)l.trows * l.piece * 2 * l.gplanes);
        l.dx = take(t * d * 4 * l.dx_parts);
        l.dw_splits = take(4);
        l.dw = l.dw_parts > 1 ? take((size_t)l.piece * d * 4 * l.dw_parts) : 0;
    } else {
        l.part = take((size_t)l.chunk * l.halves * sizeof(float2));
    }
    l.total = at;
}

// What takes the least time
Layout layout(int64_t tokens, int d, int vocab, int dtype, bool bwd)
{
    Layout l;
    l.direct = dtype == MONARCH_BF16 && d % 8 == 0;
    l.planes = dtype == MONARCH_F32 ? 3 : 1;
    l.gplanes = 3;
    l.half = bwd && dtype == MONARCH_BF16 && tokens > kFewTokens;
    l.dp = (d + 7) / 8 * 8;
    l.chunk = (int)(tokens < kTokenChunk ? tokens : kTokenChunk);
    l.trows = ceil_div(tokens, 64) * 64;                                      // what dW's K chunks read; stores and loads behind it are clipped
    if (bwd) {
        l.piece = bwd_piece(tokens, d, vocab);
    } else {
        l.piece = vocab;
        if (!l.direct) {
            // planes of W within 128 MB, or whole rounds of the pairs over tiles of 128 columns, one at least, where that takes fewer
            // column rounds for an entry (fp32, 128 tokens: d 1024, vocabulary 50257: 249 -> 218 us; d 4096, 32768: 840 -> 597)
            const int mt = ceil_div(tokens > 0 ? tokens : 1, 256), half = kPgPairs / mt / 2, unit = (half > 0 ? half : 1) * 256;
            const int64_t most = kPieceBytes / ((int64_t)l.dp * 2 * l.planes);
            auto cost = [&](int piece) {
                const int tn = pg_tile(mt, piece, true);
                return (double)ceil_div((int64_t)mt * ceil_div(piece, tn), kPgPairs) * tn * (tn == 256 ? 10 : tn == 192 ? 11 : 12) / piece;
            };
            if (most < vocab) {
                const int near = most < 256 ? 256 : (int)(most / 256 * 256), whole = most < unit ? unit : (int)(most / unit * unit);
                l.piece = cost(whole) < cost(near) ? whole : near;
                if (l.piece > vocab) l.piece = vocab;
            }
        }
    }
    const int64_t mt = ceil_div(tokens, 256);
    l.tn = pg_tile(mt, l.piece, !bwd);
    l.tn_dw = pg_tile(ceil_div(l.piece, 256), d, false);
    // dx of few tiles is split along the vocabulary, as far as the parts stay within L2; narrow tiles where there would be many parts
    l.tn_dx = mt * ceil_div(d, 256) >= 8 ? 256 : 128;
    const int64_t tiles = mt * ceil_div(d, l.tn_dx), part = tokens * d * 4;
    int64_t parts = part > 0 ? ((int64_t)64 << 20) / part : 1;
    if (parts > l.piece / 256) parts = l.piece / 256;
    if (parts > kPgPairs) parts = kPgPairs;
    l.dx_parts = tiles >= 4 * kPgPairs || parts < 1 ? 1 : (int)parts;
    // dW of a small vocabulary is a few tiles, long ones: split along the tokens, 512 at least (whole calls, fp32 / bf16: 16384 tokens, d 512,
    // vocabulary 100: 457 -> 150 / 178 -> 103 us; 9065, 220, 451: 238 -> 88 / 104 -> 68)
    l.dw_parts = 1;
    if (bwd && 2 * (int64_t)ceil_div(l.piece, 256) * ceil_div(d, l.tn_dw) <= kPgPairs) {
        int64_t n = ((int64_t)64 << 20) / ((int64_t)l.piece * d * 4);
        if (n > tokens / 512) n = tokens / 512;
        if (n > kPgPairs) n = kPgPairs;
        if (n > 1) l.dw_parts = (int)n;
    }
    place(l, tokens, d, vocab, bwd);
    return l;
}

// The same in pieces of `units` 256 vocabulary entries, without parts (parts: dx keeps its own).  With widest tiles in the forward pass: fewest
// sums in memory.  Everything here grows with the tokens and the units.
Layout smaller(const Layout &best, int64_t tokens, int d, int vocab, bool bwd, int units, bool parts)
{
    Layout l = best;
    l.piece = units * 256 < best.piece ? units * 256 : best.piece;
    if (!bwd) l.tn = 256;
    l.tn_dw = pg_tile(ceil_div(l.piece, 256), d, false);
    l.dw_parts = 1;
    l.dx_parts = !parts ? 1 : best.dx_parts < units ? best.dx_parts : units;
    place(l, tokens, d, vocab, bwd);
    return l;
}

// What takes the least time within `bytes`.  Pieces and parts are chosen by the tokens, and fewer tokens may take more memory (gradient, bf16, d 1024,
// vocabulary 50257: 4096 tokens 499 MB, 5000 tokens 470): a workspace that was asked for with more tokens serves fewer in smaller pieces.
Layout layout_within(size_t bytes, int64_t tokens, int d, int vocab, int dtype, bool bwd)
{
    const Layout best = layout(tokens, d, vocab, dtype, bwd);
    if (best.total <= bytes) return best;
    const int most = ceil_div(best.piece, 256);
    for (int parts = 1; parts >= 0; --parts) {
        int units = 0;                                                        // the most that fit
        for (int lo = 1, hi = most; lo <= hi;) {
            const int mid = lo + (hi - lo) / 2;
            if (smaller(best, tokens, d, vocab, bwd, mid, parts != 0).total <= bytes) { units = mid; lo = mid + 1; }
            else hi = mid - 1;
        }
        // dx in parts only where they leave room for pieces of some size: each is four launches and its last round of tiles
        if (units >= (parts ? (most < 8 ? most : 8) : 1)) return smaller(best, tokens, d, vocab, bwd, units, parts != 0);
    }
    return best;
}
// the least that a call takes
size_t least_bytes(int64_t tokens, int d, int vocab, int dtype, bool bwd)
{
    return smaller(layout(tokens, d, vocab, dtype, bwd), tokens, d, vocab, bwd, 1, false).total;
}

template <typename T, int PL, bool BWD> int prep(PrepArgs a, cudaStream_t s)
{
    // few rows per CTA while there are SMs without one; every CTA reads all targets
    const int rows = ceil_div(a.tokens, 4 * 148);
    a.rows_per_cta = rows;
    a.ctas = ceil_div(a.tokens, rows);
    const int extra = ceil_div(a.wrows, 8);
    return launch_serialized(xent_prep_kernel<T, PL, BWD>, dim3((unsigned)(a.ctas + (extra < 148 * 6 ? extra : 148 * 6))), 256, 0, s, a);
}

template <bool BWD> int prep_any(const PrepArgs &a, int dtype, cudaStream_t s)
{
    return dtype == MONARCH_F32 ? prep<float, 3, BWD>(a, s) : prep<__nv_bfloat16, 1, BWD>(a, s);
}

int split_w(const void *W, void *wp, int v0, int rows, int piece, int d, int dp, int dtype, cudaStream_t s)
{
    const dim3 grid((unsigned)(ceil_div(rows, 8) < 148 * 8 ? ceil_div(rows, 8) : 148 * 8));
    const size_t plane = (size_t)piece * dp;
    if (dtype == MONARCH_F32)
        return launch_serialized(split_rows_kernel<float, 3>, grid, 256, 0, s, (const float *)W + (size_t)v0 * d, (__nv_bfloat16 *)wp, rows, plane, d, dp);
    return launch_serialized(split_rows_kernel<__nv_bfloat16, 1>, grid, 256, 0, s, (const __nv_bfloat16 *)W + (size_t)v0 * d, (__nv_bfloat16 *)wp, rows, plane, d, dp);
}

PlaneGemm gemm(unsigned *status)
{
    PlaneGemm g = {};
    g.status = status;
    g.splits = 1;
    return g;
}

// Sums in tensor memory.  An error of z is a relative error of g, so the logits' sums end there after 64 (bf16) or 24 (fp32) steps
// (pg_seg).  Of few tokens or a small vocabulary, where time is not the matter, they end after 16 and those of dW after 32: 3857 tokens,
// d 824, vocabulary 220: dW 2.2e-6 -> below 1e-6 off.  Up to 512 tokens the logits' end after 32 (100 tokens: 1.01e-6 -> 5.8e-7; of 1000 on
// dW's own sums weigh as much, and 4096 tokens would take 4 % longer).  The loss takes less harm: 96 (64 steps: 3.4e-7 of lse; 241: 2e-6).
constexpr int kSmallVocab = 16384;
bool short_runs(int64_t tokens, int vocab) { return tokens <= kFewTokens || vocab <= kSmallVocab; }

template <int SCHEME, class Epi>
int logits(const CUtensorMap &ma, const CUtensorMap &mb, const CUtensorMap &mc, PlaneGemm p, const typename Epi::Args &e, int seg, bool exact, cudaStream_t s)
{
    p.seg = seg < pg_seg(SCHEME) ? seg : pg_seg(SCHEME);
    if (exact && p.kdim > p.seg * kPgChunk) return launch_plane_gemm<0, 0, SCHEME, true, Epi>(ma, mb, mc, p, e, s);
    return launch_plane_gemm<0, 0, SCHEME, false, Epi>(ma, mb, mc, p, e, s);
}

}  // namespace
}  // namespace tc

namespace tc {
namespace {

constexpr int kFewCtas = 148;

template <typename T, int PL, int NT, bool BWD> int few_launch(const FewArgs &a, cudaStream_t s)
{
    return launch_serialized_up_to((int)kFewSmem, a.d % 8 == 0 ? xent_few_kernel<T, PL, NT, BWD, false> : xent_few_kernel<T, PL, NT, BWD, true>, dim3(kFewCtas),
                                   few_threads(PL, NT), (int)few_smem(a.tokens, a.d, PL), s, a);
}
template <typename T, int PL, bool BWD> int few_any(const FewArgs &a, cudaStream_t s)
{
    return few_tiles(a.tokens) == 1 ? few_launch<T, PL, 1, BWD>(a, s) : few_launch<T, PL, 2, BWD>(a, s);
}

int few(int launches, const void *x, const void *W, const int64_t *targets, float *loss, float *lse, int tokens, int d, int vocab, int64_t ignore, int dtype,
        void *ws, cudaStream_t s)
{
    FewArgs a = {};
    a.W = W;
    a.tlogit = (float *)((char *)ws + kHead);
    a.part = (float2 *)(a.tlogit + kFewMost);
    a.ticket = (unsigned *)ws + kFewTicket;
    a.ignore = ignore; a.d = d; a.vocab = vocab; a.row = few_row(d);
    const int each = (tokens + launches - 1) / launches;
    for (int t0 = 0; t0 < tokens; t0 += each) {
        a.x = (const char *)x + (size_t)t0 * d * (dtype == MONARCH_F32 ? 4 : 2);
        a.targets = targets + t0; a.loss = loss + t0; a.lse = lse + t0;
        a.tokens = tokens - t0 < each ? tokens - t0 : each;
        const int rc = dtype == MONARCH_F32 ? few_any<float, 3, false>(a, s) : few_any<__nv_bfloat16, 1, false>(a, s);
        MONARCH_TRY(rc);
    }
    return MONARCH_OK;
}

// CTAs along the vocabulary for two per SM
int few_parts(int d, int vocab, int tiles)
{
    const int wide = ceil_div(d, 128 / tiles), most = ceil_div(vocab, 64), want = 2 * kFewCtas / wide;
    return want < 1 ? 1 : want < most ? want : most;
}
size_t few_bwd_bytes(int d, int vocab) { return kHead + up((size_t)vocab * kFewMost * 4) + (size_t)few_parts(d, vocab, 1) * kFewMost * d * 4; }

template <typename T, int TP> int few_grad_launch(FewGradArgs a, T *dx, cudaStream_t s)
{
    const int parts = few_parts(a.d, a.vocab, TP / 8);
    a.rows = ceil_div(a.vocab, parts);
    const int used = ceil_div(a.vocab, a.rows);
    MONARCH_TRY(launch_serialized(a.d % 8 == 0 ? xent_few_grad_kernel<T, TP, false> : xent_few_grad_kernel<T, TP, true>, dim3(ceil_div(a.d, 1024 / TP), used), 256, 0, s, a));
    return launch_serialized(xent_few_dx_kernel<T>, dim3(ceil_div(a.d, 32), a.tokens), 256, 0, s, a.part, a.targets, a.ignore, dx, a.tokens, a.d, used);
}

template <typename T, int PL>
int few_bwd(int launches, const T *x, const T *W, const int64_t *targets, const float *lse, const float *dloss, T *dx, float *dW, int accumulate, int tokens,
            int d, int vocab, int64_t ignore, void *ws, cudaStream_t s)
{
    FewArgs a = {};
    a.W = W;
    a.g = (float *)((char *)ws + kHead);
    a.ignore = ignore; a.d = d; a.vocab = vocab; a.row = few_row(d);
    FewGradArgs b = {};
    b.W = W; b.g = a.g; b.dW = dW; b.part = (float *)((char *)ws + kHead + up((size_t)vocab * kFewMost * 4));
    b.ignore = ignore; b.d = d; b.vocab = vocab;
    const int each = (tokens + launches - 1) / launches;
    for (int t0 = 0; t0 < tokens; t0 += each) {
        b.x = a.x = x + (size_t)t0 * d;
        b.targets = a.targets = targets + t0; a.lse_in = lse + t0; a.dloss = dloss + t0;
        b.tokens = a.tokens = tokens - t0 < each ? tokens - t0 : each;
        b.accumulate = accumulate || t0 > 0;
        int rc = few_any<T, PL, true>(a, s);
        MONARCH_TRY(rc);
        rc = few_tiles(a.tokens) == 1 ? few_grad_launch<T, 8>(b, dx + (size_t)t0 * d, s) : few_grad_launch<T, 16>(b, dx + (size_t)t0 * d, s);
        MONARCH_TRY(rc);
    }
    return MONARCH_OK;
}

}  // namespace
}  // namespace tc

// A workspace sized for a batch serves every smaller one, on whichever kernels: also the few tokens' parts, whose size is the same for all.
// `least`: what a call needs, else what it runs best with.
size_t xent_workspace_bytes(int64_t tokens, int32_t d, int32_t vocab, int dtype, int bwd, bool least)
{
    const size_t few = bwd ? tc::few_bwd_bytes(d, vocab) : tc::kHead + tc::kFewMost * (4 + 8 * tc::kFewCtas);
    const size_t need = least ? tc::least_bytes(tokens, d, vocab, dtype, bwd != 0) : tc::layout(tokens, d, vocab, dtype, bwd != 0).total;
    return need > few ? need : few;
}

int xent_fwd(const void *x, const void *W, const int64_t *targets, float *loss, float *lse, int64_t tokens, int32_t d, int32_t vocab,
             int64_t ignore_index, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    using namespace tc;
    if (tokens == 0) return MONARCH_OK;
    if (const int launches = few_launches(tokens, d, vocab, dtype, false)) return few(launches, x, W, targets, loss, lse, (int)tokens, d, vocab, ignore_index, dtype, ws, s);
    const Layout l = layout_within(ws_bytes, tokens, d, vocab, dtype, false);
    char *base = (char *)ws;
    unsigned *status = (unsigned *)ws;
    int *count = (int *)(base + l.count), *map = (int *)(base + l.map), *tgt = (int *)(base + l.tgt);
    float *tlogit = (float *)(base + l.tlogit);
    float2 *part = (float2 *)(base + l.part);
    __nv_bfloat16 *xp = (__nv_bfloat16 *)(base + l.x);

    PrepArgs a = {};
    a.x = x; a.targets = targets; a.loss = loss; a.lse = lse;
    a.count = count; a.map = map; a.tgt = tgt; a.xp = xp;
    a.ignore = ignore_index; a.tokens = (int)tokens; a.d = d; a.dp = l.dp; a.vocab = vocab;
    const int wfirst = vocab < l.piece ? vocab : l.piece;
    if (!l.direct) { a.W = W; a.wp = (__nv_bfloat16 *)(base + l.w); a.wplane = (size_t)l.piece * l.dp; a.wrows = wfirst; }
    MONARCH_TRY(prep_any<false>(a, dtype, s));

    CUtensorMap ma, mb;
    MONARCH_TRY(plane_map(&ma, xp, 0, tokens, l.dp, l.dp, tokens * l.dp, l.planes));
    for (int64_t row0 = 0; row0 < tokens; row0 += l.chunk) {
        int half0 = 0;
        const int rows = (int)(tokens - row0 < l.chunk ? tokens - row0 : l.chunk);
        for (int v0 = 0; v0 < vocab; v0 += l.piece) {
            const int cols = vocab - v0 < l.piece ? vocab - v0 : l.piece;
            PlaneGemm p = gemm(status);
            p.count = count; p.row0 = (int)row0; p.rows = rows; p.cols = cols; p.kdim = d; p.tn = l.tn;
            if (l.direct) {
                MONARCH_TRY(plane_map(&mb, W, 0, vocab, d, d, (int64_t)vocab * d, 1, l.tn / 2));
                p.b_n0 = v0;
            } else {
                // the preparation has split the first piece; where there are more, another chunk of tokens splits it again
                if (v0 > 0 || (row0 > 0 && l.piece < vocab)) MONARCH_TRY(split_w(W, base + l.w, v0, cols, l.piece, d, l.dp, dtype, s));
                MONARCH_TRY(plane_map(&mb, base + l.w, 0, cols, l.dp, l.dp, (int64_t)l.piece * l.dp, l.planes, l.tn / 2));
            }
            const EpiStats::Args e = {part, tlogit, tgt, count, (int)row0, cols, v0, l.halves, half0};
            half0 += 2 * ceil_div(cols, l.tn);
            if (dtype == MONARCH_F32) MONARCH_TRY((logits<kP3x3, EpiStats>(ma, mb, mb, p, e, 16, true, s)));
            else MONARCH_TRY((logits<kP1, EpiStats>(ma, mb, mb, p, e, 16, d > 1536, s)));
        }
        const int ctas = ceil_div(rows, 8) < 148 * 8 ? ceil_div(rows, 8) : 148 * 8;
        MONARCH_TRY(launch_serialized(xent_join_kernel, dim3((unsigned)ctas), 256, 0, s, (const float2 *)part, (const float *)tlogit,
                                      (const int *)tgt, (const int *)map, (const int *)count, (int)row0, rows, l.halves, loss, lse));
    }
    return MONARCH_OK;
}

namespace tc {
namespace {

template <typename T, bool HALF, int LOGITS, int DW, int DX>
int bwd_pieces(const Layout &l, const void *W, T *dx, float *dW, int accumulate, int64_t tokens, int32_t d, int32_t vocab, int dtype, char *base, cudaStream_t s)
{
    unsigned *status = (unsigned *)base;
    const int *count = (const int *)(base + l.count), *map = (const int *)(base + l.map), *tgt = (const int *)(base + l.tgt);
    const float *clse = (const float *)(base + l.lse), *cdl = (const float *)(base + l.dl);
    __nv_bfloat16 *xp = (__nv_bfloat16 *)(base + l.x), *g = (__nv_bfloat16 *)(base + l.g);
    float *acc = (float *)(base + l.dx);
    int *splits = (int *)(base + l.splits);
    const size_t gplane = (size_t)l.trows * l.piece;
    const int *largest = (const int *)(base + l.largest), *exponent = (const int *)(base + l.exponent);
    constexpr int GP = 3;

    CUtensorMap x_k, x_n, w_k, w_n, g_m, g_k, g_to, dw_to, dx_to, x_h;
    if (d % 4 == 0) {
        if (l.dw_parts > 1) MONARCH_TRY(tile_target(&dw_to, base + l.dw, l.piece, d, (int64_t)l.piece * d, l.dw_parts));
        else MONARCH_TRY(tile_target(&dw_to, dW, vocab, d, (int64_t)vocab * d, 1));
        MONARCH_TRY(tile_target(&dx_to, acc, tokens, d, tokens * d, l.dx_parts));
    } else {
        MONARCH_TRY(plane_map(&dw_to, xp, 0, tokens, l.dp, l.dp, tokens * l.dp, l.planes));                    // not used
        dx_to = dw_to;
    }
    MONARCH_TRY(plane_target(&g_to, g, l.trows, l.piece, l.piece, (int64_t)gplane, l.gplanes));
    MONARCH_TRY(plane_map(&x_k, xp, 0, tokens, l.dp, l.dp, tokens * l.dp, l.planes));
    MONARCH_TRY(plane_map(&x_n, xp, 1, tokens, l.dp, l.dp, tokens * l.dp, l.planes));
    MONARCH_TRY(plane_map(&g_k, g, 0, l.trows, l.piece, l.piece, (int64_t)gplane, l.gplanes));
    // dW: all planes, or the two fp16 parts behind the bf16 one
    MONARCH_TRY(plane_map(&g_m, g + (HALF ? gplane : 0), 1, l.trows, l.piece, l.piece, (int64_t)gplane, HALF ? 2 : l.gplanes));
    if (HALF) MONARCH_TRY(plane_map(&x_h, base + l.xh, 1, tokens, l.dp, l.dp, tokens * l.dp, 1));
    else x_h = x_n;
    if (l.direct) {
        MONARCH_TRY(plane_map(&w_k, W, 0, vocab, d, d, (int64_t)vocab * d, 1, l.tn / 2));
        MONARCH_TRY(plane_map(&w_n, W, 1, vocab, d, d, (int64_t)vocab * d, 1));
    }
    for (int v0 = 0; v0 < vocab; v0 += l.piece) {
        const int cols = vocab - v0 < l.piece ? vocab - v0 : l.piece;
        if (!l.direct) {
            if (v0 > 0) MONARCH_TRY(split_w(W, base + l.w, v0, cols, l.piece, d, l.dp, dtype, s));
            MONARCH_TRY(plane_map(&w_k, base + l.w, 0, cols, l.dp, l.dp, (int64_t)l.piece * l.dp, l.planes, l.tn / 2));
            MONARCH_TRY(plane_map(&w_n, base + l.w, 1, cols, l.dp, l.dp, (int64_t)l.piece * l.dp, l.planes));
        }
        // g
        PlaneGemm p = gemm(status);
        p.count = count; p.rows = (int)tokens; p.cols = cols; p.kdim = d; p.tn = l.tn;
        p.b_n0 = l.direct ? v0 : 0;
        const typename EpiGrad<GP, HALF>::Args eg = {cols, v0, tgt, count, clse, cdl, exponent, largest};
        MONARCH_TRY((logits<LOGITS, EpiGrad<GP, HALF>>(x_k, w_k, g_to, p, eg, short_runs(tokens, vocab) ? 4 : tokens <= 512 ? 8 : 16, true, s)));
        // dW = g^T x
        p = gemm(status);
        p.count = count; p.count_is_k = 1; p.rows = cols; p.cols = d; p.kdim = (int)tokens; p.tn = l.tn_dw;
        p.n_fastest = 1;
        p.seg = short_runs(tokens, vocab) && pg_seg(DW) > 4 ? 4 : pg_seg(DW);
        p.half = HALF;
        float *to = dW + (size_t)v0 * d, *parts = (float *)(base + l.dw);
        int *dw_splits = (int *)(base + l.dw_splits);
        const size_t part = (size_t)l.piece * d;
        const bool tma = d % 4 == 0;
        EpiStoreF32::Args ew = {to, cols, d, accumulate, tma ? v0 : -1, HALF ? largest : nullptr, 0};
        if (l.dw_parts > 1) {
            p.splits = l.dw_parts;
            p.splits_out = dw_splits;
            ew.out = parts; ew.add = 0; ew.y0 = tma ? 0 : -1; ew.part = part;
        }
        MONARCH_TRY((launch_plane_gemm<1, 1, DW, true, EpiStoreF32>(g_m, x_h, dw_to, p, ew, s)));
        if (l.dw_parts > 1) {
            const long long n = (long long)cols * d, want = (n / (tma ? 4 : 1) + 255) / 256;
            MONARCH_TRY(launch_serialized(tma ? xent_dw_kernel<4> : xent_dw_kernel<1>, dim3((unsigned)(want < 148 * 8 ? want : 148 * 8)), 256, 0, s, (const float *)parts, part,
                                          (const int *)dw_splits, to, n, accumulate));
        }
        // dx += g W
        p = gemm(status);
        p.count = count; p.rows = (int)tokens; p.cols = d; p.kdim = cols; p.tn = l.tn_dx;
        p.b_k0 = l.direct ? v0 : 0;
        p.n_fastest = 1;
        p.seg = pg_seg(DX);
        if (l.dx_parts == 1) {
            const typename EpiDx<T>::Args ex = {acc, dx, map, count, d, v0 == 0, v0 + cols == vocab};
            MONARCH_TRY((launch_plane_gemm<0, 1, DX, DX != kP1, EpiDx<T>>(g_k, w_n, w_n, p, ex, s)));
        } else {
            // the last piece may be smaller: every piece has as many parts as the first found best
            p.splits = l.dx_parts;
            p.splits_out = v0 == 0 ? splits : nullptr;
            p.splits_in = v0 == 0 ? nullptr : splits;
            const EpiDxPart::Args ex = {acc, count, (size_t)tokens * d, d, v0 == 0, d % 4 == 0};
            MONARCH_TRY((launch_plane_gemm<0, 1, DX, DX != kP1, EpiDxPart>(g_k, w_n, dx_to, p, ex, s)));
        }
    }
    if (l.dx_parts > 1) {
        const int64_t want = (tokens * d / (d % 4 == 0 ? 4 : 1) + 255) / 256;
        const int ctas = (int)(want < 148 * 8 ? want : 148 * 8);
        return launch_serialized(xent_dx_kernel<T>, dim3((unsigned)ctas), 256, 0, s, (const float *)acc, (size_t)tokens * d, (const int *)splits, map, count, dx, d);
    }
    return MONARCH_OK;
}

}  // namespace
}  // namespace tc

int xent_bwd(const void *x, const void *W, const int64_t *targets, const float *lse, const float *dloss, void *dx, float *dW, int accumulate,
             int64_t tokens, int32_t d, int32_t vocab, int64_t ignore_index, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    using namespace tc;
    if (tokens == 0) {
        if (!accumulate) MONARCH_CUDA_TRY(cudaMemsetAsync(dW, 0, (size_t)vocab * d * sizeof(float), s));
        return MONARCH_OK;
    }
    if (const int launches = few_launches(tokens, d, vocab, dtype, true)) {
        if (dtype == MONARCH_F32)
            return few_bwd<float, 3>(launches, (const float *)x, (const float *)W, targets, lse, dloss, (float *)dx, dW, accumulate, (int)tokens, d, vocab, ignore_index, ws, s);
        return few_bwd<__nv_bfloat16, 1>(launches, (const __nv_bfloat16 *)x, (const __nv_bfloat16 *)W, targets, lse, dloss, (__nv_bfloat16 *)dx, dW, accumulate, (int)tokens, d, vocab,
                                         ignore_index, ws, s);
    }
    const Layout l = layout_within(ws_bytes, tokens, d, vocab, dtype, true);
    char *base = (char *)ws;
    PrepArgs a = {};
    a.x = x; a.targets = targets; a.lse_in = lse; a.dloss = dloss; a.dx = dx;
    a.count = (int *)(base + l.count); a.map = (int *)(base + l.map); a.tgt = (int *)(base + l.tgt);
    a.clse = (float *)(base + l.lse); a.cdl = (float *)(base + l.dl);
    a.xp = (__nv_bfloat16 *)(base + l.x);
    a.ignore = ignore_index; a.tokens = (int)tokens; a.d = d; a.dp = l.dp; a.vocab = vocab;
    if (!l.direct) { a.W = W; a.wp = (__nv_bfloat16 *)(base + l.w); a.wplane = (size_t)l.piece * l.dp; a.wrows = vocab < l.piece ? vocab : l.piece; }
    if (l.half) {
        a.xh = (__half *)(base + l.xh); a.exponent = (int *)(base + l.exponent); a.largest = (int *)(base + l.largest);
        MONARCH_CUDA_TRY(cudaMemsetAsync(a.largest, 0, 4, s));
    }
    MONARCH_TRY(prep_any<true>(a, dtype, s));
    if (dtype == MONARCH_F32)
        return bwd_pieces<float, false, kP3x3, kP3x3, kP3x3>(l, W, (float *)dx, dW, accumulate, tokens, d, vocab, dtype, base, s);
    if (!l.half)
        return bwd_pieces<__nv_bfloat16, false, kP1, kP3x1, kP2x1>(l, W, (__nv_bfloat16 *)dx, dW, accumulate, tokens, d, vocab, dtype, base, s);
    return bwd_pieces<__nv_bfloat16, true, kP1, kP2x1, kP1>(l, W, (__nv_bfloat16 *)dx, dW, accumulate, tokens, d, vocab, dtype, base, s);
}

}  // namespace monarch
