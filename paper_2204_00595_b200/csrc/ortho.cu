// Orthogonalisation of every block of a stack by Newton-Schulz products, and the optimiser step that uses it:
//   X0 = U / (||U||_F + 1e-7);  steps times: S = X X^T (X^T X where rows > cols), X <- a X + (b S + c S^2) X
// for the gradients of the factors L, R (each block is a matrix of its own: with orthogonal blocks M = P L P^T R is orthogonal).
#include "plane_gemm.cuh"

namespace monarch {
namespace tc {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kEps = 1e-7f;

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// What a call reads and writes: orthogonalize (V == null: U = in, out = O) or the optimiser step (in = dW, out = W).
template <typename T> struct Io {
    const void *in;            // T, or float (dW)
    float *V;
    T *out;
    float keep, step, beta;    // W <- keep W - step O
    int nesterov;
    // U of element i; the momentum is updated where `update` says so (once per call), else read as updated
    __device__ __forceinline__ float u(size_t i, bool update) const
    {
        if (V == nullptr) return elem<T>::load((const T *)in + i);
        const float g = ((const float *)in)[i];
        float v = V[i];
        if (update) {
            v = fmaf(beta, v, g);
            V[i] = v;
        }
        return nesterov ? fmaf(beta, v, g) : v;
    }
    __device__ __forceinline__ void write(size_t i, float o) const
    {
        if (V == nullptr) elem<T>::store(out + i, o);
        else elem<T>::store(out + i, keep * elem<T>::load(out + i) - step * o);
    }
};

// ------------------------------------------------------------------------------------------------ blocks that fit one SM
// X (k x n, the smaller side first) twice and one k x k matrix in shared memory; S lives in the buffer of the next X.
constexpr int kSmallThreads = 256;

__host__ __device__ constexpr int pad4(int v) { return (v + 3) / 4 * 4; }
// floats: X, Y (also S), P; rows padded to four and 4 words apart in their banks
__host__ __device__ inline size_t small_floats(int k, int n)
{
    const int kp = pad4(k), ldn = pad4(n) + 4, ldk = kp + 4;
    return (size_t)kp * (2 * ldn) + (size_t)kp * ldk;
}
constexpr size_t kSmallMax = 220 * 1024;
bool fits_small(int k, int n) { return small_floats(k, n) * 4 <= kSmallMax; }

template <typename T>
__global__ void __launch_bounds__(kSmallThreads) ortho_small_kernel(const Io<T> io, int rows, int cols, int steps)
{
    extern __shared__ __align__(16) float sm[];
    __shared__ double s_norm[kSmallThreads / 32];
    const bool wide = rows <= cols;
    const int k = wide ? rows : cols, n = wide ? cols : rows;
    const int kp = pad4(k), np = pad4(n), ldn = np + 4, ldk = kp + 4;
    float *X = sm, *Y = X + (size_t)kp * ldn, *P = Y + (size_t)kp * ldn;
    const int tid = threadIdx.x, size = rows * cols;
    const size_t base = (size_t)blockIdx.x * size;
    depend_wait();
    depend_launch();
    for (int i = tid; i < kp * ldn; i += kSmallThreads) X[i] = 0.0f;
    __syncthreads();
    double q = 0.0;
    for (int i = tid; i < size; i += kSmallThreads) {
        const int r = i / cols, c = i - r * cols;
        const float u = io.u(base + i, true);
        q += (double)u * u;
        X[wide ? r * ldn + c : c * ldn + r] = u;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if ((tid & 31) == 0) s_norm[tid >> 5] = q;
    __syncthreads();
    q = 0.0;
#pragma unroll
    for (int w = 0; w < kSmallThreads / 32; ++w) q += s_norm[w];
    const double inv = 1.0 / (sqrt(q) + (double)kEps);               // fp64: norms beyond the fp32 range
    for (int i = tid; i < kp * ldn; i += kSmallThreads) X[i] = (float)((double)X[i] * inv);
    __syncthreads();
    const int tk = kp / 4, tn = np / 4;
    for (int it = 0; it < steps; ++it) {
        float *S = Y;                                                  // k x k, row length ldk
        for (int t = tid; t < tk * tk; t += kSmallThreads) {
            const int i = t / tk * 4, j = t % tk * 4;
            float a[4][4] = {};
            for (int c = 0; c < np; c += 4) {
                float4 x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = *reinterpret_cast<const float4 *>(X + (i + e) * ldn + c);
                    y[e] = *reinterpret_cast<const float4 *>(X + (j + e) * ldn + c);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        a[e][f] = fmaf(x[e].x, y[f].x, fmaf(x[e].y, y[f].y, fmaf(x[e].z, y[f].z, fmaf(x[e].w, y[f].w, a[e][f]))));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) *reinterpret_cast<float4 *>(S + (i + e) * ldk + j) = make_float4(a[e][0], a[e][1], a[e][2], a[e][3]);
        }
        __syncthreads();
        for (int t = tid; t < tk * tk; t += kSmallThreads) {
            const int i = t / tk * 4, j = t % tk * 4;
            float a[4][4] = {};
            for (int c = 0; c < kp; c += 4) {
                float4 x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = *reinterpret_cast<const float4 *>(S + (i + e) * ldk + c);
                    y[e] = *reinterpret_cast<const float4 *>(S + (j + e) * ldk + c);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        a[e][f] = fmaf(x[e].x, y[f].x, fmaf(x[e].y, y[f].y, fmaf(x[e].z, y[f].z, fmaf(x[e].w, y[f].w, a[e][f]))));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int f = 0; f < 4; ++f) P[(i + e) * ldk + j + f] = fmaf(kB, S[(i + e) * ldk + j + f], kC * a[e][f]);
        }
        __syncthreads();
        for (int t = tid; t < tk * tn; t += kSmallThreads) {
            const int i = t / tn * 4, j = t % tn * 4;
            float a[4][4] = {};
            for (int c = 0; c < kp; ++c) {
                const float4 y = *reinterpret_cast<const float4 *>(X + c * ldn + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = P[(i + e) * ldk + c];
                    a[e][0] = fmaf(x, y.x, a[e][0]);
                    a[e][1] = fmaf(x, y.y, a[e][1]);
                    a[e][2] = fmaf(x, y.z, a[e][2]);
                    a[e][3] = fmaf(x, y.w, a[e][3]);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 y = *reinterpret_cast<const float4 *>(X + (i + e) * ldn + j);
                *reinterpret_cast<float4 *>(Y + (i + e) * ldn + j) =
                    make_float4(fmaf(kA, y.x, a[e][0]), fmaf(kA, y.y, a[e][1]), fmaf(kA, y.z, a[e][2]), fmaf(kA, y.w, a[e][3]));
            }
        }
        __syncthreads();
        float *t = X;
        X = Y;
        Y = t;
    }
    for (int i = tid; i < size; i += kSmallThreads) {
        const int r = i / cols, c = i - r * cols;
        io.write(base + i, X[wide ? r * ldn + c : c * ldn + r]);
    }
}

// ------------------------------------------------------------------------------------------------ larger blocks
constexpr int kNormParts = 64;

// sums of squares of kNormParts parts of each block (and the new momentum)
template <typename T>
__global__ void __launch_bounds__(256) norm_kernel(const Io<T> io, double *part, int64_t size)
{
    __shared__ double s_part[8];
    depend_wait();
    depend_launch();
    const int64_t per = (size + kNormParts - 1) / kNormParts, first = blockIdx.x * per, last = min(size, first + per);
    const size_t base = (size_t)blockIdx.y * size;
    double q = 0.0;
    for (int64_t i = first + threadIdx.x; i < last; i += 256) {
        const float u = io.u(base + i, true);
        q += (double)u * u;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = q;
    __syncthreads();
    if (threadIdx.x == 0) {
        q = 0.0;
        for (int w = 0; w < 8; ++w) q += s_part[w];
        part[(size_t)blockIdx.y * kNormParts + blockIdx.x] = q;
    }
}

// one value into PL planes
template <int PL> __device__ __forceinline__ void put_planes(__nv_bfloat16 *to, size_t plane, float v)
{
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v);
        to[i * plane] = h;
        v -= __bfloat162float(h);
    }
}

struct Finish {
    const float *part;            // [blocks][splits][rows][cols]
    int splits;
    int rows, cols, ld;           // ld: row of a plane
    float *f32;                   // S or X, [blocks][rows][cols]
    __nv_bfloat16 *planes;        // [blocks][PL][rows][ld]
};

// MODE 0: X = U / |U|;  1: S = sum of the parts;  2: P = b S + c sum;  3: X = a X + sum;  4: the last X, to the caller
template <typename T, int PL, int MODE>
__global__ void __launch_bounds__(256) finish_kernel(const Finish f, const Io<T> io, const double *norm)
{
    depend_wait();
    depend_launch();
    const int64_t size = (int64_t)f.rows * f.cols;
    const size_t base = (size_t)blockIdx.y * size;
    const size_t plane = (size_t)f.rows * f.ld;
    double inv = 0.0;
    if (MODE == 0) {
        double q = 0.0;
        for (int i = 0; i < kNormParts; ++i) q += norm[(size_t)blockIdx.y * kNormParts + i];
        inv = 1.0 / (sqrt(q) + (double)kEps);
    }
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)gridDim.x * 256) {
        float v;
        if (MODE == 0) {
            v = (float)((double)io.u(base + i, false) * inv);
        } else {
            const float *p = f.part + ((size_t)blockIdx.y * f.splits) * size + i;
            v = 0.0f;
            for (int s = 0; s < f.splits; ++s) v += p[(size_t)s * size];
            if (MODE == 2) v = fmaf(kB, f.f32[base + i], kC * v);
            if (MODE == 3 || MODE == 4) v = fmaf(kA, f.f32[base + i], v);
        }
        if (MODE == 4) {
            io.write(base + i, v);
            continue;
        }
        if (MODE != 2) f.f32[base + i] = v;
        const int64_t r = i / f.cols, c = i - r * f.cols;
        put_planes<PL>(f.planes + (size_t)blockIdx.y * PL * plane + (size_t)r * f.ld + c, plane, v);
    }
}

struct EpiPart {
    struct Args {
        float *out;
        int rows, cols;
    };
    __device__ __forceinline__ void begin(const Args &, const PgTile &) {}
    __device__ __forceinline__ void chunk(const Args &a, const PgTile &t, int c, float (&v)[32])
    {
        if (t.row >= a.rows) return;
        const int left = a.cols - t.col - c;
        float *out = a.out + ((size_t)t.z * a.rows + t.row) * a.cols + t.col + c;
        if ((a.cols & 3) == 0) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
                if (i < left) *reinterpret_cast<float4 *>(out + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < left) out[i] = v[i];
        }
    }
    __device__ __forceinline__ void end(const Args &, const PgTile &) {}
};

struct Large {
    int k, n, ldx, ldk, planes, split_s, split_p, split_x;
    size_t norm, x, xp, s, sp, pp, part, total;
};

int split_for(int64_t blocks, int m, int n, int kdim)
{
    const int64_t tiles = blocks * ceil_div(m, kPgTile) * ceil_div(n, kPgTile), chunks = ceil_div(kdim, kPgChunk);
    int64_t s = tiles > 0 ? 74 / tiles : 1;
    if (s > chunks / 4) s = chunks / 4;
    return s < 1 ? 1 : (int)s;
}

Large large_layout(int64_t blocks, int rows, int cols, int dtype)
{
    Large l;
    l.k = rows < cols ? rows : cols;
    l.n = rows < cols ? cols : rows;
    l.ldx = (cols + 7) / 8 * 8;
    l.ldk = (l.k + 7) / 8 * 8;
    l.planes = dtype == MONARCH_F32 ? 3 : 2;
    l.split_s = split_for(blocks, l.k, l.k, l.n);
    l.split_p = split_for(blocks, l.k, l.k, l.k);
    l.split_x = split_for(blocks, rows, cols, l.k);
    const size_t kk = (size_t)l.k * l.k, rc = (size_t)rows * cols, b = (size_t)blocks;
    size_t at = MONARCH_STATUS_BYTES;
    auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes); return o; };
    l.norm = take(b * kNormParts * 8);
    l.x = take(b * rc * 4);
    l.xp = take(b * l.planes * rows * l.ldx * 2);
    l.s = take(b * kk * 4);
    l.sp = take(b * l.planes * l.k * l.ldk * 2);
    l.pp = take(b * l.planes * l.k * l.ldk * 2);
    size_t part = kk * (l.split_s > l.split_p ? l.split_s : l.split_p);
    if (rc * l.split_x > part) part = rc * l.split_x;
    l.part = take(b * part * 4);
    l.total = at;
    return l;
}

template <typename T, int PL, int SCHEME>
int ortho_large(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, int dtype, void *ws, cudaStream_t s)
{
    const Large l = large_layout(blocks, rows, cols, dtype);
    char *base = (char *)ws;
    const bool wide = rows <= cols;
    double *norm = (double *)(base + l.norm);
    float *X = (float *)(base + l.x), *S = (float *)(base + l.s), *part = (float *)(base + l.part);
    __nv_bfloat16 *xp = (__nv_bfloat16 *)(base + l.xp), *sp = (__nv_bfloat16 *)(base + l.sp), *pp = (__nv_bfloat16 *)(base + l.pp);
    const int64_t size = (int64_t)rows * cols;
    if (blocks > 65535) return MONARCH_ERR_UNSUPPORTED;

    CUtensorMap x_k, x_n, s_k, p_k;
    MONARCH_TRY(plane_map(&x_k, xp, 0, rows, cols, l.ldx, (int64_t)rows * l.ldx, blocks * PL));
    MONARCH_TRY(plane_map(&x_n, xp, 1, rows, cols, l.ldx, (int64_t)rows * l.ldx, blocks * PL));
    MONARCH_TRY(plane_map(&s_k, sp, 0, l.k, l.k, l.ldk, (int64_t)l.k * l.ldk, blocks * PL));
    MONARCH_TRY(plane_map(&p_k, pp, 0, l.k, l.k, l.ldk, (int64_t)l.k * l.ldk, blocks * PL));
    const Finish fx = {part, l.split_x, rows, cols, l.ldx, X, xp}, fs = {part, l.split_s, l.k, l.k, l.ldk, S, sp},
                 fp = {part, l.split_p, l.k, l.k, l.ldk, S, pp};
    auto grid = [&](int64_t n) {
        int64_t g = (n + 1023) / 1024, most = 148 * 8 / blocks + 1;
        return dim3((unsigned)(g < most ? g : most), (unsigned)blocks);
    };
    MONARCH_TRY(launch_serialized(norm_kernel<T>, dim3(kNormParts, (unsigned)blocks), 256, 0, s, io, norm, size));
    MONARCH_TRY(launch_serialized(finish_kernel<T, PL, 0>, grid(size), 256, 0, s, fx, io, (const double *)norm));
    PlaneGemm p = {};
    p.status = (unsigned *)ws;
    p.batches = (int)blocks;
    p.a_zstep = p.b_zstep = PL;
    p.seg = SCHEME == kP3x3 ? pg_seg(SCHEME) : 16;         // bf16 results: 192 steps
    for (int i = 0; i < steps; ++i) {
        p.rows = p.cols = l.k;
        p.kdim = l.n;
        p.splits = l.split_s;
        const EpiPart::Args ek = {part, l.k, l.k}, ex = {part, rows, cols};
        if (wide) MONARCH_TRY((launch_plane_gemm<0, 0, SCHEME, true, EpiPart>(x_k, x_k, p, ek, s)));
        else MONARCH_TRY((launch_plane_gemm<1, 1, SCHEME, true, EpiPart>(x_n, x_n, p, ek, s)));
        MONARCH_TRY(launch_serialized(finish_kernel<T, PL, 1>, grid((int64_t)l.k * l.k), 256, 0, s, fs, io, (const double *)norm));
        p.kdim = l.k;
        p.splits = l.split_p;
        MONARCH_TRY((launch_plane_gemm<0, 0, SCHEME, true, EpiPart>(s_k, s_k, p, ek, s)));
        MONARCH_TRY(launch_serialized(finish_kernel<T, PL, 2>, grid((int64_t)l.k * l.k), 256, 0, s, fp, io, (const double *)norm));
        p.rows = rows;
        p.cols = cols;
        p.splits = l.split_x;
        if (wide) MONARCH_TRY((launch_plane_gemm<0, 1, SCHEME, true, EpiPart>(p_k, x_n, p, ex, s)));
        else MONARCH_TRY((launch_plane_gemm<0, 0, SCHEME, true, EpiPart>(x_k, p_k, p, ex, s)));
        if (i + 1 < steps)
            MONARCH_TRY(launch_serialized(finish_kernel<T, PL, 3>, grid(size), 256, 0, s, fx, io, (const double *)norm));
        else
            MONARCH_TRY(launch_serialized(finish_kernel<T, PL, 4>, grid(size), 256, 0, s, fx, io, (const double *)norm));
    }
    return MONARCH_OK;
}

template <typename T, int PL, int SCHEME>
int ortho_any(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, int dtype, void *ws, cudaStream_t s)
{
    if (blocks == 0) return MONARCH_OK;
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (!fits_small(k, n)) return ortho_large<T, PL, SCHEME>(io, blocks, rows, cols, steps, dtype, ws, s);
    return launch_serialized(ortho_small_kernel<T>, dim3((unsigned)blocks), kSmallThreads, (int)(small_floats(k, n) * 4), s, io, rows, cols, steps);
}

}  // namespace
}  // namespace tc

size_t ortho_workspace_bytes(int64_t blocks, int32_t rows, int32_t cols, int dtype)
{
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return tc::fits_small(k, n) ? (size_t)MONARCH_STATUS_BYTES : tc::large_layout(blocks, rows, cols, dtype).total;
}

int orthogonalize(const void *G, void *O, int64_t blocks, int32_t rows, int32_t cols, int32_t steps, int dtype, void *ws, cudaStream_t s)
{
    if (dtype == MONARCH_F32) {
        const tc::Io<float> io = {G, nullptr, (float *)O, 0.0f, 0.0f, 0.0f, 0};
        return tc::ortho_any<float, 3, tc::kP3x3>(io, blocks, rows, cols, steps, dtype, ws, s);
    }
    const tc::Io<__nv_bfloat16> io = {G, nullptr, (__nv_bfloat16 *)O, 0.0f, 0.0f, 0.0f, 0};
    return tc::ortho_any<__nv_bfloat16, 2, tc::kP2x2>(io, blocks, rows, cols, steps, dtype, ws, s);
}

int muon_step(void *W, const float *dW, float *V, int64_t blocks, int32_t rows, int32_t cols, float keep, float step, float beta, int nesterov,
              int32_t steps, int dtype, void *ws, cudaStream_t s)
{
    if (dtype == MONARCH_F32) {
        const tc::Io<float> io = {dW, V, (float *)W, keep, step, beta, nesterov};
        return tc::ortho_any<float, 3, tc::kP3x3>(io, blocks, rows, cols, steps, dtype, ws, s);
    }
    const tc::Io<__nv_bfloat16> io = {dW, V, (__nv_bfloat16 *)W, keep, step, beta, nesterov};
    return tc::ortho_any<__nv_bfloat16, 2, tc::kP2x2>(io, blocks, rows, cols, steps, dtype, ws, s);
}

}  // namespace monarch
