// Orthogonalisation of every block of a stack by Newton-Schulz products, and the optimiser step that uses it:
//   X0 = U / (||U||_F + 1e-7);  steps times: S = X X^T (X^T X where rows > cols), X <- a X + (b S + c S^2) X
// for the gradients of the factors L, R (each block is a matrix of its own: with orthogonal blocks M = P L P^T R is orthogonal).
#include <type_traits>

#include "plane_gemm.cuh"

namespace monarch {
namespace tc {
namespace {

// published with the Muon optimiser (K. Jordan and others, 2024)
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
    // Reads and writes are separate steps, so that a thread can have all its reads under way before its first write.
    struct In {
        float g, v;
    };
    __device__ __forceinline__ In fetch(size_t i) const
    {
        if (V == nullptr) return {elem<T>::load((const T *)in + i), 0.0f};
        return {((const float *)in)[i], V[i]};
    }
    // U of element i; the momentum is updated where `update` says so (once per call), else `f.v` is the updated one
    __device__ __forceinline__ float u(size_t i, In f, bool update) const
    {
        if (V == nullptr) return f.g;
        if (update) {
            f.v = fmaf(beta, f.v, f.g);
            V[i] = f.v;
        }
        return nesterov ? fmaf(beta, f.v, f.g) : f.v;
    }
    // the same for four consecutive elements, i a multiple of 4
    struct In4 {
        float g[4], v[4];
    };
    static __device__ __forceinline__ void load4(const float *p, float (&o)[4])
    {
        const float4 t = *reinterpret_cast<const float4 *>(p);
        o[0] = t.x; o[1] = t.y; o[2] = t.z; o[3] = t.w;
    }
    static __device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&o)[4])
    {
        const uint2 t = *reinterpret_cast<const uint2 *>(p);
        o[0] = __uint_as_float(t.x << 16); o[1] = __uint_as_float(t.x & 0xffff0000u);
        o[2] = __uint_as_float(t.y << 16); o[3] = __uint_as_float(t.y & 0xffff0000u);
    }
    static __device__ __forceinline__ void store4(float *p, const float (&o)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(o[0], o[1], o[2], o[3]); }
    static __device__ __forceinline__ void store4(__nv_bfloat16 *p, const float (&o)[4])
    {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
    }
    __device__ __forceinline__ In4 fetch4(size_t i) const
    {
        In4 f = {};
        if (V == nullptr) {
            load4((const T *)in + i, f.g);
        } else {
            load4((const float *)in + i, f.g);
            load4(V + i, f.v);
        }
        return f;
    }
    __device__ __forceinline__ void u4(size_t i, In4 &f, float (&o)[4]) const
    {
        if (V == nullptr) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = f.g[e];
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f.v[e] = fmaf(beta, f.v[e], f.g[e]);
            o[e] = nesterov ? fmaf(beta, f.v[e], f.g[e]) : f.v[e];
        }
        store4(V + i, f.v);
    }
    __device__ __forceinline__ void old4(size_t i, float (&w)[4]) const
    {
        if (V != nullptr) load4(out + i, w);
    }
    __device__ __forceinline__ void write4(size_t i, float (&o)[4], const float (&w)[4]) const
    {
        if (V != nullptr) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(keep, w[e], -step * o[e]);
        }
        store4(out + i, o);
    }
    __device__ __forceinline__ float old(size_t i) const { return V == nullptr ? 0.0f : elem<T>::load(out + i); }
    __device__ __forceinline__ void write(size_t i, float o, float w) const
    {
        elem<T>::store(out + i, V == nullptr ? o : fmaf(keep, w, -step * o));
    }
};

// Element e = thread, thread + threads, .. of a row-major block as (row, column), without a division per element
struct Walk {
    int r, c, dr, dc, cols;
    __device__ __forceinline__ Walk(int first, int stride, int cols_) : cols(cols_)
    {
        r = first / cols;
        c = first - r * cols;
        dr = stride / cols;
        dc = stride - dr * cols;
    }
    __device__ __forceinline__ void next()
    {
        r += dr;
        c += dc;
        if (c >= cols) { c -= cols; ++r; }
    }
};

// ------------------------------------------------------------------------------------------------ long, narrow blocks
// k up to 32, n over 256: X (k x n, the smaller side first) twice and one k x k matrix in shared memory in fp32, plain FMA; S lives in
// the buffer of the next X.  A few MACs per value: tensor core tiles of 128 or 256 rows would be nearly empty.
constexpr int kSmallThreads = 256;

__host__ __device__ constexpr int pad4(int v) { return (v + 3) / 4 * 4; }
// floats: X, Y (also S), P; rows padded to four and 4 words apart in their banks
__host__ __device__ inline size_t small_floats(int k, int n)
{
    const int kp = pad4(k), ldn = pad4(n) + 4, ldk = kp + 4;
    return (size_t)kp * (2 * ldn) + (size_t)kp * ldk;
}
constexpr size_t kSmallMax = 220 * 1024;
bool fits_small(int k, int n) { return k <= 32 && small_floats(k, n) * 4 <= kSmallMax; }

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
        const float u = io.u(base + i, io.fetch(base + i), true);
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
        io.write(base + i, X[wide ? r * ldn + c : c * ldn + r], io.old(base + i));
    }
}

// ------------------------------------------------------------------------------------------------ blocks up to 64 x 256
// One CTA per block, everything on chip: X, S and P = b S + c S^2 are bf16 planes in shared memory (PL = 2 for bf16 results, 3 for
// fp32), their fp32 values stay in the registers of the thread that holds them as an accumulator, warp-level MMAs (m16n8k16).
// S is symmetric, so S and P serve as either operand as stored; only P X needs X transposed (ldmatrix.trans).  For k up to 32, and for
// n of 129 to 256 with k up to 64, where X does not fit what the kernel below has.  64 blocks of 32 x 32, five steps: bf16 4.8 us, fp32 5.9, of which 3.5 is the launch.
// KP, NP: k and n rounded up; warps: KP / 16 rows of tiles times two column halves.
template <int KP, int NP, int PL> struct BlockCfg {
    static constexpr int kRows = KP / 16, kThreads = kRows * 2 * 32;
    static constexpr int kLdX = NP + 8, kLdS = KP + 8;                       // rows 16 bytes apart in their banks
    static constexpr int kXPlane = KP * kLdX, kSPlane = KP * kLdS;           // elements
    static constexpr int kXBufs = NP > 128 ? 1 : 2;                          // the next X beside the one it is made of, or over it
    static constexpr int kSmem = (kXBufs * PL * kXPlane + 2 * PL * kSPlane) * 2;
    static constexpr int kS = KP / 16, kX = NP / 16;                         // 8-column tiles of a warp in S and in X
};

// acc[t] += A B for T column tiles of 8.  A: planes at `a` (row-major, 16 rows of this warp), B: planes at `b`, TRANS: stored [k][n].
// An MMA adds without rounding to nearest, so what a sum loses goes by the number of its products when it is large.  kApart: those of the
// first planes have a sum of their own, which takes a sixth of them (fp32; bf16: a third), and the small ones are added to it at the end;
// kTwice (no registers for that): all the small ones come first, then K once more for the first planes.
enum Sums { kOne, kApart, kTwice };
template <int PL, int KSTEPS, int T, bool TRANS, Sums SUMS = kOne>
__device__ __forceinline__ void plane_mma(float (&acc)[T][4], uint32_t a, uint32_t aplane, int lda, uint32_t b, uint32_t bplane, int ldb)
{
    const int lane = threadIdx.x & 31, mtx = lane >> 3, r = lane & 7;
    // A: matrices (rows 0-7, k 0-7), (rows 8-15, k 0-7), (rows 0-7, k 8-15), (rows 8-15, k 8-15)
    const uint32_t a_at = a + ((mtx & 1) * 8 + r) * lda * 2 + (mtx >> 1) * 16;
    // B, two column tiles at a time: (n 0-7, k 0-7), (n 0-7, k 8-15), (n 8-15, k 0-7), (n 8-15, k 8-15); of an odd T the last one
    // alone, twice: what would be the other one's rows may lie behind the planes
    const uint32_t b_at = TRANS ? b + ((mtx & 1) * 8 + r) * ldb * 2 : b + r * ldb * 2 + (mtx & 1) * 16;
    const uint32_t second = TRANS ? (mtx >> 1) * 16 : (mtx >> 1) * 8 * ldb * 2;
    constexpr bool APART = SUMS == kApart;
    float low[APART ? T : 1][4] = {};
#pragma unroll
    for (int i = 0; i < (SUMS == kTwice ? 2 : 1) * KSTEPS; ++i) {
        const int k = i % KSTEPS, first = SUMS == kTwice && i < KSTEPS ? 1 : 0, last = SUMS == kTwice && i >= KSTEPS ? 0 : PL - 1;      // of these orders
        uint32_t fa[PL][4];
#pragma unroll
        for (int q = 0; q <= last; ++q) ldm4(fa[q], a_at + q * aplane + k * 32);
#pragma unroll
        for (int t = 0; t < T; t += 2) {
            const uint32_t at = b_at + (t + 1 < T ? second : 0);
            uint32_t fb[PL][4];
#pragma unroll
            for (int q = 0; q <= last; ++q) {
                if constexpr (TRANS) ldm4t(fb[q], at + q * bplane + k * 16 * ldb * 2 + t * 16);
                else ldm4(fb[q], at + q * bplane + t * 8 * ldb * 2 + k * 32);
            }
            // the small products first
#pragma unroll
            for (int o = last; o >= first; --o)
#pragma unroll
                for (int q = o; q >= 0; --q) {
                    float (*to)[4] = APART && o > 0 ? low : acc;
                    mma(to[t], fa[q], fb[o - q][0], fb[o - q][1]);
                    if (t + 1 < T) mma(to[t + 1], fa[q], fb[o - q][2], fb[o - q][3]);
                }
        }
    }
    if constexpr (APART)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] += low[t][e];
}

// this thread's values of T column tiles as planes: rows row, row + 8
template <int PL, int T> __device__ __forceinline__ void put_tiles(const float (&v)[T][4], __nv_bfloat16 *to, int plane, int ld)
{
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x = v[t][2 * h], y = v[t][2 * h + 1];
#pragma unroll
            for (int q = 0; q < PL; ++q) {
                const uint32_t w = pack_bf16(x, y);
                *reinterpret_cast<uint32_t *>(to + q * plane + h * 8 * ld + t * 8) = w;
                x -= __uint_as_float(w << 16);
                y -= __uint_as_float(w & 0xffff0000u);
            }
        }
}

template <typename T, int KP, int NP, int PL>
__global__ void __launch_bounds__(BlockCfg<KP, NP, PL>::kThreads) ortho_block_kernel(const Io<T> io, int rows, int cols, int steps)
{
    using C = BlockCfg<KP, NP, PL>;
    extern __shared__ __align__(16) __nv_bfloat16 smb[];
    __shared__ double s_norm[C::kThreads / 32];
    __nv_bfloat16 *Xs = smb, *Ss = smb + C::kXBufs * PL * C::kXPlane, *Ps = Ss + PL * C::kSPlane;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row0 = (warp >> 1) * 16, half = warp & 1;
    const int r = lane >> 2, c2 = (lane & 3) * 2;
    const bool wide = rows <= cols;
    const int k = wide ? rows : cols, n = wide ? cols : rows;
    const int sr = wide ? cols : 1, sc = wide ? 1 : cols;                    // X[i][j] = G[i sr + j sc]
    const size_t base = (size_t)blockIdx.x * rows * cols;
    depend_wait();
    depend_launch();

    float x[C::kX][4];
    typename Io<T>::In f[C::kX][4];
    double q = 0.0;
#pragma unroll
    for (int t = 0; t < C::kX; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = row0 + r + (e >> 1) * 8, j = half * (NP / 2) + t * 8 + c2 + (e & 1);
            f[t][e] = {0.0f, 0.0f};
            if (i < k && j < n) f[t][e] = io.fetch(base + (size_t)(i * sr + j * sc));
        }
#pragma unroll
    for (int t = 0; t < C::kX; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = row0 + r + (e >> 1) * 8, j = half * (NP / 2) + t * 8 + c2 + (e & 1);
            const float u = i < k && j < n ? io.u(base + (size_t)(i * sr + j * sc), f[t][e], true) : 0.0f;
            x[t][e] = u;
            q += (double)u * u;
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if (lane == 0) s_norm[warp] = q;
    __syncthreads();
    q = 0.0;
#pragma unroll
    for (int w = 0; w < C::kThreads / 32; ++w) q += s_norm[w];
    const double inv = 1.0 / (sqrt(q) + (double)kEps);                       // fp64: norms beyond the fp32 range
#pragma unroll
    for (int t = 0; t < C::kX; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][e] = (float)((double)x[t][e] * inv);

    const int x_at = (row0 + r) * C::kLdX + half * (NP / 2) + c2, s_at = (row0 + r) * C::kLdS + half * (KP / 2) + c2;
    put_tiles<PL>(x, Xs + x_at, C::kXPlane, C::kLdX);
    const uint32_t s_a = smem_u32(Ss) + row0 * C::kLdS * 2, s_b = smem_u32(Ss) + half * (KP / 2) * C::kLdS * 2;
    const uint32_t p_a = smem_u32(Ps) + row0 * C::kLdS * 2;
    for (int it = 0; it < steps; ++it) {
        __syncthreads();
        const uint32_t X = smem_u32(Xs) + (C::kXBufs > 1 ? it & 1 : 0) * (PL * C::kXPlane * 2);
        float s[C::kS][4] = {}, p[C::kS][4] = {};
        plane_mma<PL, NP / 16, C::kS, false, kApart>(s, X + row0 * C::kLdX * 2, C::kXPlane * 2, C::kLdX, X + half * (KP / 2) * C::kLdX * 2, C::kXPlane * 2, C::kLdX);
        put_tiles<PL>(s, Ss + s_at, C::kSPlane, C::kLdS);
        __syncthreads();
        plane_mma<PL, KP / 16, C::kS, false, kApart>(p, s_a, C::kSPlane * 2, C::kLdS, s_b, C::kSPlane * 2, C::kLdS);
#pragma unroll
        for (int t = 0; t < C::kS; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[t][e] = fmaf(kB, s[t][e], kC * p[t][e]);
        put_tiles<PL>(p, Ps + s_at, C::kSPlane, C::kLdS);
        __syncthreads();
        float y[C::kX][4] = {};
        plane_mma<PL, KP / 16, C::kX, true, (KP > 32 && PL > 2 ? kTwice : kOne)>(y, p_a, C::kSPlane * 2, C::kLdS, X + half * NP, C::kXPlane * 2, C::kLdX);
#pragma unroll
        for (int t = 0; t < C::kX; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][e] = fmaf(kA, x[t][e], y[t][e]);
        if (it + 1 < steps) {
            if (C::kXBufs == 1) __syncthreads();
            put_tiles<PL>(x, Xs + (C::kXBufs > 1 ? (it + 1) & 1 : 0) * PL * C::kXPlane + x_at, C::kXPlane, C::kLdX);
        }
    }
    float w[C::kX][4];
#pragma unroll
    for (int t = 0; t < C::kX; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = row0 + r + (e >> 1) * 8, j = half * (NP / 2) + t * 8 + c2 + (e & 1);
            w[t][e] = i < k && j < n ? io.old(base + (size_t)(i * sr + j * sc)) : 0.0f;
        }
#pragma unroll
    for (int t = 0; t < C::kX; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = row0 + r + (e >> 1) * 8, j = half * (NP / 2) + t * 8 + c2 + (e & 1);
            if (i < k && j < n) io.write(base + (size_t)(i * sr + j * sc), x[t][e], w[t][e]);
        }
}

template <typename T, int KP, int NP, int PL> int launch_block(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, cudaStream_t s)
{
    using C = BlockCfg<KP, NP, PL>;
    return launch_serialized(ortho_block_kernel<T, KP, NP, PL>, dim3((unsigned)blocks), C::kThreads, C::kSmem, s, io, rows, cols, steps);
}

bool fits_block(int k, int n) { return k <= 64 && n <= 256; }

template <typename T, int PL> int ortho_block(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, cudaStream_t s)
{
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (k <= 16) {
        if (n <= 16) return launch_block<T, 16, 16, PL>(io, blocks, rows, cols, steps, s);
        if (n <= 32) return launch_block<T, 16, 32, PL>(io, blocks, rows, cols, steps, s);
        if (n <= 64) return launch_block<T, 16, 64, PL>(io, blocks, rows, cols, steps, s);
        if (n <= 128) return launch_block<T, 16, 128, PL>(io, blocks, rows, cols, steps, s);
        return launch_block<T, 16, 256, PL>(io, blocks, rows, cols, steps, s);
    }
    if (k <= 32) {
        if (n <= 32) return launch_block<T, 32, 32, PL>(io, blocks, rows, cols, steps, s);
        if (n <= 64) return launch_block<T, 32, 64, PL>(io, blocks, rows, cols, steps, s);
        if (n <= 128) return launch_block<T, 32, 128, PL>(io, blocks, rows, cols, steps, s);
        return launch_block<T, 32, 256, PL>(io, blocks, rows, cols, steps, s);
    }
    return launch_block<T, 64, 256, PL>(io, blocks, rows, cols, steps, s);
}

// ------------------------------------------------------------------------------------------------ blocks up to 128 x 128
// One CTA per block on the tcgen05 tensor cores, everything on chip: X and S in registers (thread = row and a quarter of either
// column half), accumulators in tensor memory, operands as planes: the second one in shared memory as slabs of 64 columns in the
// 128-byte swizzle (K-major as stored; MN-major for the X of P X, whose rows are K), the first one in tensor memory, whose rows are
// the threads' (both from shared memory take 8 KB for the 64 cycles of an MMA of 128 x 128 x 16: all that an SM can read).  There is
// room there for two planes; of three, the third is read from shared memory.  KP x NP: k and n rounded up to 64 or 128; all of it is
// computed, what stands behind the block is zeros.  (KP = 64: the MMAs have 128 rows all the same, nobody reads the others.)
//
// After a product: tensor memory -> fp32 -> planes of the next operand.  Products and conversions overlap by column halves: the K
// steps that read the first half of an operand are issued as soon as it is written, the others finish the first half of a result of
// 128 columns before the second, so that its values are converted meanwhile.  What a conversion overwrites (P over S, X over X) is the
// half that no MMA still under way reads.
// Measured, 128 blocks of 128 x 128, optimiser step: bf16 27.6 us (3.7 a step: 2360 cycles a product, 1536 of them MMAs of three
// plane products), fp32 43.0 (6.6 a step); with fp32 FMA 525.  128 of 64 x 64: 14.2 and 19.4 us (1.9 and 2.9 a step; on warp MMAs
// 15.1 and 22.1): a product is 384 (768) cycles of MMAs and some 800 of hand-over, two barriers and two waits.  The one thread that issues has to keep its operands in uniform
// registers (elect_one): picked as thread 0 it took 60 cycles per MMA, 33.3 and 51.1 us.
constexpr int kTcThreads = 512;
template <int KP, int NP, int PL> struct TcCfg {
    static constexpr int kSlab = KP * 128;                                   // KP rows of 64 columns
    static constexpr int kXPlane = KP * NP * 2, kSPlane = KP * KP * 2;
    // MMAs that take the first operand's third plane from shared memory read 128 rows: with 64, what stands behind as well
    static constexpr int kSmem = PL * (kXPlane + kSPlane) + (PL > 2 && KP < 128 ? kSlab : 0) + 1024;
    static constexpr int kCs = KP / 8, kCx = NP / 8;                         // columns of a thread in a half of S, of X
};

struct KMajor { static constexpr bool value = false; };
struct NMajor { static constexpr bool value = true; };

// D[tmem] (+)= A[tmem] B[smem desc]
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
template <int C> __device__ __forceinline__ void tmem_put(uint32_t taddr, const uint32_t (&r)[C])
{
    static_assert(C == 4 || C == 8, "8 or 16 columns of packed values");
    if constexpr (C == 8)
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                     "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                     : "memory");
    else
        asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// C columns of this thread's lane
template <int C> __device__ __forceinline__ void tmem_get(uint32_t taddr, float (&f)[C])
{
    static_assert(C == 8 || C == 16, "8 or 16 columns");
    if constexpr (C == 16) {
        tmem_ask16(taddr, f);
        tmem_ready(f);
    } else {
        tmem_ld8(taddr, reinterpret_cast<uint32_t (&)[8]>(f));
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7])::"memory");
    }
}

// K columns k0 .. k0 + 16 STEPS of A B for columns n0 .. n0 + N of B, all plane products, the small ones first.  A: planes 0 and 1 in
// tensor memory (64 columns each), plane 2 in shared memory at `a2`; planes of A there `aplane` bytes apart, of B `bplane`.
template <int PL, bool BMN, int N, int STEPS, int SLAB>
__device__ __forceinline__ void tc_part(uint32_t d, uint32_t a, uint32_t a2, uint32_t aplane, uint32_t b, uint32_t bplane, int k0, int n0, uint32_t more)
{
    constexpr uint32_t idesc = make_idesc_bf16(128, N, 0, BMN);
    a += k0 / 2;
    a2 += 2 * aplane + (k0 >> 6) * SLAB + (k0 & 63) * 2;
    b += BMN ? (n0 >> 6) * SLAB + k0 * 128 : (k0 >> 6) * SLAB + (k0 & 63) * 2 + n0 * 128;
#pragma unroll
    for (int o = PL - 1; o >= 0; --o)
#pragma unroll
        for (int q = o; q >= 0; --q) {
            const uint64_t bd = BMN ? make_smem_desc(b + (o - q) * bplane, SLAB, 1024, kSwizzle128) : make_smem_desc(b + (o - q) * bplane, 16, 1024, kSwizzle128);
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                if (q < 2) mma_f16_ts(d + n0, a + q * 64 + k * 8, bd + (BMN ? 128 : 2) * k, idesc, more);
                else mma_f16_ss(d + n0, make_smem_desc(a2, 16, 1024, kSwizzle128) + 2 * k, bd + (BMN ? 128 : 2) * k, idesc, more);
                more = 1;
            }
        }
}

// C values of a row from column `col` as planes: the first operand (tensor memory at `a`, the third plane in shared memory), and if
// BOTH the second one (shared memory)
template <int PL, bool BOTH, int SLAB, int C> __device__ __forceinline__ void tc_put(uint32_t planes, uint32_t plane, uint32_t a, int row, int col, float (&v)[C])
{
#pragma unroll
    for (int q = 0; q < PL; ++q) {
        uint32_t w[C / 2];
#pragma unroll
        for (int e = 0; e < C / 2; ++e) {
            w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
            v[2 * e] -= __uint_as_float(w[e] << 16);
            v[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
        }
        if (q < 2) tmem_put(a + q * 64 + col / 2, w);
        if (BOTH || q >= 2) {
            const uint32_t at = planes + q * plane + (col >> 6) * SLAB + row * 128;
#pragma unroll
            for (int j = 0; j < C / 8; ++j)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((((col & 63) >> 3) + j) ^ (row & 7)) << 4)), "r"(w[4 * j]), "r"(w[4 * j + 1]),
                             "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                             : "memory");
        }
    }
}

template <typename T, int PL, int KP, int NP>
__global__ void __launch_bounds__(kTcThreads, 1) ortho_tc_kernel(const Io<T> io, int rows, int cols, int steps, unsigned *status)
{
    using C = TcCfg<KP, NP, PL>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_s[2];
    __shared__ double s_norm[kTcThreads / 32];
    __shared__ uint32_t tmem_base_s;
    __shared__ int dead_s;
    const uint32_t X = (smem_u32(smem_raw) + 1023u) & ~1023u, S = X + PL * C::kXPlane, bar = smem_u32(bar_s);
    float *stage = reinterpret_cast<float *>(smem_raw + (X - smem_u32(smem_raw)));       // KP x NP floats over the planes of X
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;     // the same in all lanes, for the compiler too
    const int row = (warp & 3) * 32 + lane, cs = (warp >> 2) * C::kCs, cx = (warp >> 2) * C::kCx;
    const bool holds = KP == 128 || (warp & 3) < KP / 32;                                 // this warp has rows
    const bool wide = rows <= cols;
    const int size = rows * cols;
    const size_t base = (size_t)blockIdx.x * size;
    volatile int *dead = &dead_s;

    if (tid == 0) {
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        fence_mbar_init();
        dead_s = 0;
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_base_s), 512);
        tmem_relinquish();
    }
    if (size < KP * NP)
        for (int i = tid * 4; i < KP * NP; i += kTcThreads * 4) *reinterpret_cast<float4 *>(stage + i) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(~0u, tmem_base_s, 0);
    depend_wait();
    depend_launch();

    // X[i][j] at stage[i * NP + (j ^ (i & 31))]: consecutive values of G and one column of all rows are both in different banks
    double q = 0.0;
    const bool four = cols % 4 == 0;           // four values of a row at a time
    Walk at(four ? 4 * tid : tid, four ? 4 * kTcThreads : kTcThreads, cols);
    if (four) {
        constexpr int kMost = KP * NP / 4 / kTcThreads;
        typename Io<T>::In4 f[kMost];
#pragma unroll
        for (int a = 0; a < kMost; ++a)
            if ((tid + a * kTcThreads) * 4 < size) f[a] = io.fetch4(base + (tid + a * kTcThreads) * 4);
#pragma unroll
        for (int a = 0; a < kMost; ++a) {
            if ((tid + a * kTcThreads) * 4 >= size) break;
            float u[4];
            io.u4(base + (tid + a * kTcThreads) * 4, f[a], u);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int i = wide ? at.r : at.c + b, j = wide ? at.c + b : at.r;
                q += (double)u[b] * u[b];
                stage[i * NP + (j ^ (i & 31))] = u[b];
            }
            at.next();
        }
    } else
    for (int e0 = tid; e0 < size; e0 += 8 * kTcThreads) {
        typename Io<T>::In f[8];
#pragma unroll
        for (int a = 0; a < 8; ++a)
            if (e0 + a * kTcThreads < size) f[a] = io.fetch(base + e0 + a * kTcThreads);
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            if (e0 + a * kTcThreads >= size) break;
            const int i = wide ? at.r : at.c, j = wide ? at.c : at.r;
            const float u = io.u(base + e0 + a * kTcThreads, f[a], true);
            q += (double)u * u;
            stage[i * NP + (j ^ (i & 31))] = u;
            at.next();
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if (lane == 0) s_norm[warp] = q;
    __syncthreads();
    q = 0.0;
#pragma unroll
    for (int w = 0; w < kTcThreads / 32; ++w) q += s_norm[w];
    const double inv = 1.0 / (sqrt(q) + (double)kEps);                       // fp64: norms beyond the fp32 range
    float x[2][C::kCx];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < C::kCx; ++j) x[h][j] = holds ? (float)((double)stage[row * NP + ((h * (NP / 2) + cx + j) ^ lane)] * inv) : 0.0f;
    __syncthreads();

    // the first operand of P X (and of S S) beside that of X X^T where their halves are not the same columns: X is written while P is read
    const uint32_t d_s = tmem, d_t = tmem + KP, d_x = tmem + 256, a_x = tmem + 384, a_s = KP == NP ? a_x : tmem + 128;
    static_assert(KP == NP || KP == 64, "room for a second first operand");
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    uint32_t phase = 0;
    bool ok = true, stop = false;               // stop: some thread's wait ran out, the same in all threads
    auto written = [&]() {                     // this half of the operands is written, and its accumulators are read
        tmem_st_wait();
        fence_proxy_async_smem();
        tc_fence_before();
        stop = __syncthreads_or(!ok);
        tc_fence_after();
    };
    auto arrived = [&](int h) {
        if (!mbar_wait(bar + h * 8, phase, status, dead, kErrMmaWait)) ok = false;
        tc_fence_after();
    };
    // the MMAs of a product of N columns over K: what the first half of the operands allows (h = 0), or the rest
    auto issue = [&](auto bmn, auto n, auto k, int h, uint32_t d, uint32_t A, uint32_t a2, uint32_t aplane, uint32_t b, uint32_t bplane) {
        if (warp != 0 || !elect_one()) return;
        constexpr bool kBmn = decltype(bmn)::value;
        constexpr int N = decltype(n)::value, K = decltype(k)::value, kSteps = K / 32;
        if (h == 0) {
            tc_part<PL, kBmn, N, kSteps, C::kSlab>(d, A, a2, aplane, b, bplane, 0, 0, 0);
        } else if (N == 128) {
            tc_part<PL, kBmn, 64, kSteps, C::kSlab>(d, A, a2, aplane, b, bplane, K / 2, 0, 1);
            mma_commit(bar);
            tc_part<PL, kBmn, 64, kSteps, C::kSlab>(d, A, a2, aplane, b, bplane, K / 2, 64, 1);
            mma_commit(bar + 8);
        } else {
            tc_part<PL, kBmn, N, kSteps, C::kSlab>(d, A, a2, aplane, b, bplane, K / 2, 0, 1);
            mma_commit(bar);
            mma_commit(bar + 8);
        }
    };
    using Kp = std::integral_constant<int, KP>;
    using Np = std::integral_constant<int, NP>;
    auto gram = [&](int h) { issue(KMajor(), Kp(), Np(), h, d_s, a_x, X, C::kXPlane, X, C::kXPlane); };
    auto square = [&](int h) { issue(KMajor(), Kp(), Kp(), h, d_t, a_s, S, C::kSPlane, S, C::kSPlane); };
    auto update = [&](int h) { issue(NMajor(), Np(), Kp(), h, d_x, a_s, S, C::kSPlane, X, C::kXPlane); };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float v[C::kCx];
#pragma unroll
        for (int j = 0; j < C::kCx; ++j) v[j] = x[h][j];
        if (holds) tc_put<PL, true, C::kSlab>(X, C::kXPlane, a_x + lanes, row, h * (NP / 2) + cx, v);
    }
    written();
    gram(0);
    gram(1);
    for (int it = 0; it < steps; ++it) {
        float s[2][C::kCs];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            arrived(h);
            if (holds) {
                float v[C::kCs];
                tmem_get(d_s + lanes + h * (KP / 2) + cs, v);
#pragma unroll
                for (int j = 0; j < C::kCs; ++j) s[h][j] = v[j];
                tc_put<PL, true, C::kSlab>(S, C::kSPlane, a_s + lanes, row, h * (KP / 2) + cs, v);
            }
            written();
            square(h);
        }
        phase ^= 1;
        // P = b S + c S^2
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            arrived(h);
            if (holds) {
                float v[C::kCs];
                tmem_get(d_t + lanes + h * (KP / 2) + cs, v);
#pragma unroll
                for (int j = 0; j < C::kCs; ++j) v[j] = fmaf(kB, s[h][j], kC * v[j]);
                tc_put<PL, false, C::kSlab>(S, C::kSPlane, a_s + lanes, row, h * (KP / 2) + cs, v);
            }
            written();
            update(h);
        }
        phase ^= 1;
        // X = a X + P X
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            arrived(h);
            if (holds) {
                float v[C::kCx];
                tmem_get(d_x + lanes + h * (NP / 2) + cx, v);
#pragma unroll
                for (int j = 0; j < C::kCx; ++j) x[h][j] = v[j] = fmaf(kA, x[h][j], v[j]);
                if (it + 1 < steps) tc_put<PL, true, C::kSlab>(X, C::kXPlane, a_x + lanes, row, h * (NP / 2) + cx, v);
            }
            if (it + 1 < steps) {
                written();
                gram(h);
            }
        }
        phase ^= 1;
        if (stop) break;
    }
    tc_fence_before();
    if (__syncthreads_or(!ok)) let_copies_land(dead);      // nor do MMAs outlive their shared and tensor memory, the last product's among them
    if (warp == 0) tmem_dealloc(tmem, 512);
    if (holds)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < C::kCx; ++j) stage[row * NP + ((h * (NP / 2) + cx + j) ^ lane)] = x[h][j];
    __syncthreads();
    at = Walk(four ? 4 * tid : tid, four ? 4 * kTcThreads : kTcThreads, cols);
    if (four) {
        constexpr int kMost = KP * NP / 4 / kTcThreads;
        float w[kMost][4];
#pragma unroll
        for (int a = 0; a < kMost; ++a)
            if ((tid + a * kTcThreads) * 4 < size) io.old4(base + (tid + a * kTcThreads) * 4, w[a]);
#pragma unroll
        for (int a = 0; a < kMost; ++a) {
            if ((tid + a * kTcThreads) * 4 >= size) break;
            float o[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int i = wide ? at.r : at.c + b, j = wide ? at.c + b : at.r;
                o[b] = stage[i * NP + (j ^ (i & 31))];
            }
            io.write4(base + (tid + a * kTcThreads) * 4, o, w[a]);
            at.next();
        }
    } else
    for (int e0 = tid; e0 < size; e0 += 8 * kTcThreads) {
        float w[8];
#pragma unroll
        for (int a = 0; a < 8; ++a)
            if (e0 + a * kTcThreads < size) w[a] = io.old(base + e0 + a * kTcThreads);
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            if (e0 + a * kTcThreads >= size) break;
            const int i = wide ? at.r : at.c, j = wide ? at.c : at.r;
            io.write(base + e0 + a * kTcThreads, stage[i * NP + (j ^ (i & 31))], w[a]);
            at.next();
        }
    }
}

template <typename T, int PL, int KP, int NP>
int launch_tc(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, void *ws, cudaStream_t s)
{
    return launch_serialized(ortho_tc_kernel<T, PL, KP, NP>, dim3((unsigned)blocks), kTcThreads, TcCfg<KP, NP, PL>::kSmem, s, io, rows, cols, steps, (unsigned *)ws);
}

// ------------------------------------------------------------------------------------------------ larger blocks
// Three products a step, with the square completed so that each needs its operands alone:
//   S~ = X X^T + beta I,   P = c S~ S~^T + (a - c beta^2) I = a I + b S + c S^2,   X <- P X,      beta = b / 2c
// (X^T X and X P where rows > cols).  An error of P counts against its eigenvalues, 0.64 to 3.44; that b S comes out of a difference
// costs nothing there.  S~, P and X exist only as bf16 planes in memory.  S~ and P are symmetric: only the blocks of 256 columns up
// to the diagonal are computed, each tile below it is written transposed as well.
//
// ONE launch does all products of all steps on the CTA pairs of plane_gemm.cuh (256 x tn tiles, a ring of operand tiles, two
// accumulators, the epilogue in eight warps).  The tiles of all products form one list, step by step, product by product, block by
// block; pair i takes tiles i, i + pairs, ..  A tile's loader waits until the product before it in its block is complete (a counter
// per block that every epilogue warp adds to when its stores have landed); the tiles of other blocks fill the time.  The launch is
// cooperative: all CTAs are resident, and a tile only ever waits for tiles before it in the list.  As fifteen launches each product
// cost 8 to 11 us beside its MMAs: code and tensor maps fetched anew, the pipeline filled and drained (4 blocks of 1024 x 1024, bf16:
// 446 us).
// A product of fewer tiles than there are pairs is cut along K as well: the parts' sums go to memory, and when all parts of a tile
// are there, each pair that made one adds up some of its columns, always in the same order (all of them added up by the last to
// finish: 112 us a step for one 1024 x 1024 block in bf16).
constexpr float kBeta = kB / (2.0f * kC), kGamma = kA - kC * kBeta * kBeta;
constexpr int kNormParts = 256;

template <int PL> __device__ __forceinline__ void put_planes(__nv_bfloat16 *to, size_t plane, float v)
{
#pragma unroll
    for (int q = 0; q < PL; ++q) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v);
        to[q * plane] = h;
        v -= __bfloat162float(h);
    }
}
// four consecutive values, the first at a multiple of four
template <int PL> __device__ __forceinline__ void put_planes4(__nv_bfloat16 *to, size_t plane, const float (&from)[4])
{
    float u[4] = {from[0], from[1], from[2], from[3]};
#pragma unroll
    for (int q = 0; q < PL; ++q) {
        const uint32_t w0 = pack_bf16(u[0], u[1]), w1 = pack_bf16(u[2], u[3]);
        *reinterpret_cast<uint2 *>(to + q * plane) = make_uint2(w0, w1);
        u[0] -= __uint_as_float(w0 << 16); u[1] -= __uint_as_float(w0 & 0xffff0000u);
        u[2] -= __uint_as_float(w1 << 16); u[3] -= __uint_as_float(w1 & 0xffff0000u);
    }
}

// A stack of matrices as planes: [blocks][PL][rows][ld], ld a multiple of 16 (what stands behind the columns is never read)
struct Planes {
    __nv_bfloat16 *at;
    int rows, cols, ld;
    __device__ __forceinline__ size_t plane() const { return (size_t)rows * ld; }
    template <int PL> __device__ __forceinline__ __nv_bfloat16 *element(int64_t block, int r, int c) const
    {
        return at + (block * PL * rows + r) * ld + c;
    }
};

// ---- the products
struct Product {
    int rows, cols, kchunks;
    int a_mn, b_mn;                // operands stored with K along their rows
    int tn, sub, lower;            // columns of a tile; tiles in 256 columns; symmetric result
    int ntiles, tiles;             // of a block
    int splits, per_split;         // parts of K, chunks in one
    int publishers;                // warps that publish something of a tile
    float scale, diagonal;         // of the result
    unsigned *parts_done;          // [blocks][tiles][16 warps], where splits > 1
};

struct alignas(64) OrthoMaps {
    CUtensorMap s_a[2], s_b[2], p_a, p_b, x_a[2], x_b[2], s_to, p_to, x_to[2];            // [2]: by the X that is read (s, x_a, x_b), written (x_to)
};

struct OrthoRun {
    unsigned *status, *done;       // done: [blocks]
    Product prod[3];
    int blocks, steps;
    int rows, cols;                // of a block
    float *part;                   // [blocks][part_units: tiles, splits][16 warps][128][32 lanes]; a block's place serves its products in turn
    int64_t part_units;
};

constexpr int kRunStage = 3, kRunSlots = pg_slots(kRunStage), kRunSmem = pg_smem(kRunStage);

__device__ __forceinline__ unsigned ld_acquire(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// bounded wait until *ctr >= need; what its writers published may then be loaded by TMA
__device__ __noinline__ bool wait_published(const unsigned *ctr, unsigned need, unsigned *status, volatile int *dead)
{
    if (ld_acquire(ctr) < need) {
        const unsigned long long t0 = global_timer_ns(), limit = wait_limit_ns(status);
        while (ld_acquire(ctr) < need) {
            if (*dead || global_timer_ns() - t0 > limit) {
                *dead = 1;
                atomicCAS(status, 0u, (unsigned)kErrPeerWait);
                return false;
            }
            __nanosleep(32);
        }
    }
    asm volatile("fence.proxy.async.global;" ::: "memory");
    return true;
}

struct Tile {
    int step, ph, block, tile, split, mt, nt, c0, c1, mirror;
};

template <typename T, int PL, int SCHEME>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPgThreads, 1)
ortho_run_kernel(const __grid_constant__ OrthoMaps maps, const __grid_constant__ OrthoRun p, const Io<T> io)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) PgBars bars;
    __shared__ uint32_t tmem_base_s;
    __shared__ int dead_s;

    const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    volatile int *dead = &dead_s;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kRunSlots; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 1);
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&bars.acc_full[a]), 1);
            mbar_init(smem_u32(&bars.acc_empty[a]), 2 * kPgEpiWarps);
        }
        fence_mbar_init();
        dead_s = 0;
    }
    if (warp == 0) {
        tmem_alloc_pair(smem_u32(&tmem_base_s), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive_release();
    cluster_wait_acquire();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(~0u, tmem_base_s, 0);
    const uint32_t full0 = smem_u32(bars.full), empty0 = smem_u32(bars.empty);
    const uint32_t accf0 = smem_u32(bars.acc_full), acce0 = smem_u32(bars.acc_empty);
    constexpr int kLoads = pg_loads(SCHEME), kSeg = SCHEME == kP3x3 ? pg_seg(SCHEME) : 16;            // bf16 results: 192 steps

    const int u0 = p.prod[0].tiles * p.prod[0].splits, u1 = p.prod[1].tiles * p.prod[1].splits, u2 = p.prod[2].tiles * p.prod[2].splits;
    const int per_step = p.blocks * (u0 + u1 + u2), total = per_step * p.steps;
    auto locate = [&](int g) {
        Tile t;
        t.step = g / per_step;
        int r = g - t.step * per_step;
        t.ph = 0;
        int u = u0;
        if (r >= p.blocks * u0) { r -= p.blocks * u0; t.ph = 1; u = u1; }
        if (t.ph == 1 && r >= p.blocks * u1) { r -= p.blocks * u1; t.ph = 2; u = u2; }
        const Product &q = p.prod[t.ph];
        t.block = r / u;
        const int v = r - t.block * u;
        t.tile = v / q.splits;
        t.split = v - t.tile * q.splits;
        t.mirror = 0;
        if (q.lower) {
            const int w = t.tile / q.sub;
            int m = (int)((sqrtf(8.0f * (float)w + 1.0f) - 1.0f) * 0.5f);
            while (m * (m + 1) / 2 > w) --m;
            while ((m + 1) * (m + 2) / 2 <= w) ++m;
            const int n = w - m * (m + 1) / 2;
            t.mt = m;
            t.nt = n * q.sub + t.tile % q.sub;
            t.mirror = n < m;
        } else {
            t.mt = t.tile / q.ntiles;
            t.nt = t.tile - t.mt * q.ntiles;
        }
        t.c0 = min(t.split * q.per_split, q.kchunks);
        t.c1 = min(t.c0 + q.per_split, q.kchunks);
        return t;
    };

    if (warp == 8) {
        // ------------------------------------------------------------ loader (both CTAs)
        if (elect_one()) {
            uint32_t slot = 0, phase = 1;
            bool ok = true;
            for (int g = pair; ok && g < total; g += npairs) {
                const Tile t = locate(g);
                const Product &q = p.prod[t.ph];
                // what the products before this one in its block have published
                const unsigned of_s = p.prod[0].tiles * p.prod[0].publishers, of_p = p.prod[1].tiles * p.prod[1].publishers, of_x = p.prod[2].tiles * p.prod[2].publishers;
                const unsigned need = (unsigned)t.step * (of_s + of_p + of_x) + (t.ph > 0 ? of_s : 0) + (t.ph > 1 ? of_p : 0);
                if (!wait_published(p.done + t.block, need, p.status, dead)) break;
                const int at = t.step & 1, m0 = t.mt * kPgTile + (int)rank * 128, n0 = t.nt * q.tn + (int)rank * (q.tn / 2);
                const CUtensorMap *ma = t.ph == 0 ? &maps.s_a[at] : t.ph == 1 ? &maps.p_a : &maps.x_a[at];
                const CUtensorMap *mb = t.ph == 0 ? &maps.s_b[at] : t.ph == 1 ? &maps.p_b : &maps.x_b[at];
                for (int c = t.c0; ok && c < t.c1; ++c) {
                    const int k0 = c * kPgChunk;
#pragma unroll
                    for (int l = 0; l < kLoads; ++l) {
                        if (!pg_wait(empty0 + slot * 8, phase, p.status, dead, kErrSlotWait)) { ok = false; break; }
                        const uint32_t dst = ring0 + slot * kPgSlotBytes, full = full0 + slot * 8;
                        constexpr int tag[6] = {pg_load(SCHEME, 0), pg_load(SCHEME, 1), pg_load(SCHEME, 2), pg_load(SCHEME, 3),
                                                pg_load(SCHEME, 4), pg_load(SCHEME, 5)};
                        const bool second = tag[l] & 4;
                        const int z = t.block * PL + (tag[l] & 3), mn = second ? q.b_mn : q.a_mn, r0 = second ? n0 : m0;
                        const CUtensorMap *m = second ? mb : ma;
                        if (rank == 0) mbar_expect_tx(full, second ? q.tn * (kPgChunk * 2) : 2 * kPgSlotBytes);
                        tma_load_3d_pair(dst, m, mn ? r0 : k0, mn ? k0 : r0, z, full);
                        if (mn && (!second || q.tn == 256)) tma_load_3d_pair(dst + 8192, m, r0 + 64, k0, z, full);
                        if (++slot == kRunSlots) { slot = 0; phase ^= 1; }
                    }
                }
            }
        }
    } else if (warp == 9) {
        if (rank == 0 && elect_one()) {
            // ------------------------------------------------------------ even CTA: MMA issuer for the pair
            uint32_t slot = 0, phase = 0, it = 0;
            bool ok = true;
            for (int g = pair; ok && g < total; g += npairs) {
                const Tile t = locate(g);
                const Product &q = p.prod[t.ph];
                const uint32_t idesc = make_idesc_bf16(256, q.tn, q.a_mn, q.b_mn), astep = q.a_mn ? 128 : 2, bstep = q.b_mn ? 128 : 2;
                const uint64_t adesc = make_smem_desc(0, q.a_mn ? 8192 : 16, 1024, kSwizzle128), bdesc = make_smem_desc(0, q.b_mn ? 8192 : 16, 1024, kSwizzle128);
                for (int c0 = t.c0; ok && c0 < t.c1; c0 += kSeg, ++it) {
                    const int c1 = min(c0 + kSeg, t.c1);
                    const uint32_t buf = it & 1;
                    if (!pg_wait(acce0 + buf * 8, ((it >> 1) & 1) ^ 1, p.status, dead, kErrTmemWait)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem_base + buf * 256;
                    for (int c = c0; ok && c < c1; ++c) {
                        uint32_t at_slot[kLoads];
#pragma unroll
                        for (int l = 0; l < kLoads; ++l) {
                            at_slot[l] = slot;
                            if (!pg_wait(full0 + slot * 8, phase, p.status, dead, kErrTmaWait)) { ok = false; break; }
                            if (++slot == kRunSlots) { slot = 0; phase ^= 1; }
                            tc_fence_after();
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int w = pg_mma(SCHEME, l, i);
                                if (w == 0xff) continue;
                                const uint64_t ad = adesc | (uint64_t)((ring0 + at_slot[w & 15] * kPgSlotBytes) >> 4);
                                const uint64_t bd = bdesc | (uint64_t)((ring0 + at_slot[w >> 4] * kPgSlotBytes) >> 4);
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk)
                                    mma_f16_ss_pair(d, ad + astep * kk, bd + bstep * kk, idesc, (uint32_t)(c != c0 || l != 1 || kk != 0));
                            }
#pragma unroll
                            for (int j = 0; j < kLoads; ++j)
                                if ((pg_done(SCHEME, l) >> j) & 1) mma_commit_pair(empty0 + at_slot[j] * 8, 3);
                        }
                    }
                    if (ok) mma_commit_pair(accf0 + buf * 8, 3);
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue (both CTAs; own 128 rows)
        const uint32_t acce_leader = map_to_cta(acce0, 0);
        uint32_t it = 0;
        bool ok = true;
        PgStage<kRunStage> st = {nullptr, ring0 + kRunSlots * kPgSlotBytes + warp * kRunStage * kPgStageBytes, lane, 0};
        for (int g = pair; ok && g < total; g += npairs) {
            const Tile t = locate(g);
            const Product &q = p.prod[t.ph];
            const int tn = q.tn;
            const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * (tn / 2));
            float acc[4][32];
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[h][i] = 0.0f;
            for (int c0 = t.c0; c0 < t.c1; c0 += kSeg, ++it) {
                const uint32_t buf = it & 1;
                if (!pg_wait_warp(accf0 + buf * 8, (it >> 1) & 1, p.status, dead, kErrMmaWait)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    if (h * 64 >= tn) break;
#pragma unroll
                    for (int j = 0; j < 32; j += 16) {
                        float v[16];
                        tmem_ask16(lane_base + buf * 256 + h * 32 + j, v);
                        tmem_ready(v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[h][j + i] += v[i];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(acce_leader + buf * 8);
            }
            if (!ok) break;
            const int mine = (int)rank * 8 + warp;
            const float *part = p.part + (((size_t)t.block * p.part_units + (size_t)t.tile * q.splits) * 16 + mine) * 4096 + lane;
            if (q.splits > 1) {
                float *to = const_cast<float *>(part) + (size_t)t.split * 16 * 4096;
                unsigned *ctr = q.parts_done + ((size_t)t.block * q.tiles + t.tile) * 16 + mine;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    if (h * 64 >= tn) break;
#pragma unroll
                    for (int i = 0; i < 32; ++i) __stcg(to + (h * 32 + i) * 32, acc[h][i]);
                }
                __threadfence();
                __syncwarp();
                if (lane == 0) atomicAdd(ctr, 1u);
                if (t.split * 64 >= tn) continue;                              // more parts than groups of columns
                if (lane == 0) ok = wait_published(ctr, (unsigned)q.splits * (unsigned)(t.step + 1), p.status, dead);
                ok = __shfl_sync(~0u, ok, 0);
                if (!ok) break;
                __threadfence();
            }
            const int row0 = t.mt * kPgTile + (int)rank * 128 + (warp & 3) * 32, col0 = t.nt * tn + (warp >> 2) * (tn / 2);
            const bool last = t.ph == 2 && t.step + 1 == p.steps;
            st.map = t.ph == 0 ? &maps.s_to : t.ph == 1 ? &maps.p_to : &maps.x_to[(t.step & 1) ^ 1];
            // one copy of the conversion, the columns moved up to it
#pragma unroll 1
            for (int h = q.splits > 1 ? t.split : 0; h * 64 < tn; h += q.splits) {
                const int col = col0 + h * 32;
                if (q.splits > 1) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[0][i] = 0.0f;
#pragma unroll 1
                    for (int s = 0; s < q.splits; ++s)
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[0][i] += __ldcg(part + (size_t)s * 16 * 4096 + (h * 32 + i) * 32);
                }
                if (row0 < q.rows && col < q.cols) {                           // the same in all lanes; TMA clips the rest
                    float (&v)[32] = acc[0];
                    if (last) {
                        const size_t at = ((size_t)t.block * p.rows + row0) * p.cols + col + lane;
                        const int rows = col + lane < p.cols ? p.rows - row0 : 0;
                        st.rows(
                            v, [&](int r) { return r < rows ? io.old(at + (size_t)r * p.cols) : 0.0f; },
                            [&](int r, float x, float w) {
                                if (r < rows) io.write(at + (size_t)r * p.cols, x, w);
                            });
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = row0 + lane == col + i ? fmaf(q.scale, v[i], q.diagonal) : q.scale * v[i];
                        // all planes behind one fence, or a plane and its transpose at a time: there are three pieces (a fourth would
                        // be a slot less for the operands: fp32 4096 x 4096 7 % slower)
                        if (!t.mirror) st.begin();
#pragma unroll
                        for (int b = 0; b < PL; ++b) {
                            uint32_t w[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                                v[2 * i] -= __uint_as_float(w[i] << 16);
                                v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                            }
                            if (!t.mirror) {
                                st.row(b, w);
                            } else {
                                st.begin();
                                st.row(0, w);
                                __syncwarp();
                                st.transpose(0, 1);
                                st.ready();
                                st.send(0, col, row0, t.block * PL + b);
                                st.send(1, row0, col, t.block * PL + b);
                                st.close();
                            }
                        }
                        if (!t.mirror) {
                            st.ready();
#pragma unroll
                            for (int b = 0; b < PL; ++b) st.send(b, col, row0, t.block * PL + b);
                            st.close();
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) { acc[0][i] = acc[1][i]; acc[1][i] = acc[2][i]; acc[2][i] = acc[3][i]; }
            }
            if (lane == 0 && !last) {
                tma_store_wait_all<0>();                                       // landed, and visible to this thread
                __threadfence();
                atomicAdd(p.done + t.block, 1u);
            }
            __syncwarp();
        }
    }

    tc_fence_before();
    __syncthreads();
    let_copies_land(dead);                                                     // as in plane_gemm.cuh
    cluster_arrive_release();
    cluster_wait_acquire();
    if (warp == 0) tmem_dealloc_pair(tmem_base, 512);
}

// sums of squares of `parts` parts of each block, and the new momentum; the counters of the products at zero
template <typename T>
__global__ void __launch_bounds__(256) norm_kernel(const Io<T> io, double *part, int parts, int64_t size, unsigned *zero, int64_t zeros)
{
    __shared__ double s_part[8];
    depend_wait();
    depend_launch();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < zeros; i += (int64_t)gridDim.x * 256) zero[i] = 0;
    const int block = blockIdx.x / parts, p = blockIdx.x % parts;
    const int64_t per = ((size + parts - 1) / parts + 3) / 4 * 4, first = p * per, last = min(size, first + per);
    const size_t base = (size_t)block * size;
    double q = 0.0;
    if (size % 4 == 0) {
        for (int64_t i = first + threadIdx.x * 4; i < last; i += 4096) {
            typename Io<T>::In4 f[4];
#pragma unroll
            for (int a = 0; a < 4; ++a)
                if (i + a * 1024 < last) f[a] = io.fetch4(base + i + a * 1024);
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                if (i + a * 1024 >= last) break;
                float u[4];
                io.u4(base + i + a * 1024, f[a], u);
                // four squares in fp64 as well: their fp32 range ends at 1.8e19
#pragma unroll
                for (int e = 0; e < 4; ++e) q += (double)u[e] * u[e];
            }
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < last; i += 256) {
            const float u = io.u(base + i, io.fetch(base + i), true);
            q += (double)u * u;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = q;
    __syncthreads();
    if (threadIdx.x == 0) {
        q = 0.0;
        for (int w = 0; w < 8; ++w) q += s_part[w];
        part[(size_t)block * parts + p] = q;
    }
}

// X0 = U / (|U| + 1e-7) as planes: `ctas` CTAs per block
template <typename T, int PL>
__global__ void __launch_bounds__(256) start_kernel(const Planes x, const Io<T> io, const double *norm, int parts, int ctas)
{
    __shared__ double s_part[8];
    depend_wait();
    depend_launch();
    const int block = blockIdx.x / ctas, p = blockIdx.x % ctas;
    double q = threadIdx.x < parts ? norm[(size_t)block * parts + threadIdx.x] : 0.0;                // kNormParts <= 256
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(~0u, q, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = q;
    __syncthreads();
    q = 0.0;
    for (int w = 0; w < 8; ++w) q += s_part[w];
    const double inv = 1.0 / (sqrt(q) + (double)kEps);
    const int64_t size = (int64_t)x.rows * x.cols;
    const size_t base = (size_t)block * size;
    if (x.cols % 4 == 0) {
        const int per_row = x.cols / 4;
        for (int64_t i = (int64_t)p * 256 + threadIdx.x; i < size / 4; i += (int64_t)ctas * 256) {
            const int r = (int)(i / per_row), c = (int)(i - (int64_t)r * per_row) * 4;
            typename Io<T>::In4 f = io.fetch4(base + i * 4);
            __nv_bfloat16 *to = x.template element<PL>(block, r, c);
            float u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = (float)((double)io.u(0, {f.g[e], f.v[e]}, false) * inv);
            put_planes4<PL>(to, x.plane(), u);
        }
    } else {
        for (int64_t i = (int64_t)p * 256 + threadIdx.x; i < size; i += (int64_t)ctas * 256) {
            const int r = (int)(i / x.cols), c = (int)(i - (int64_t)r * x.cols);
            put_planes<PL>(x.template element<PL>(block, r, c), x.plane(), (float)((double)io.u(base + i, io.fetch(base + i), false) * inv));
        }
    }
}

// Tiles and parts of a product by the time they take on a block's share of the CTA pairs, in cycles: `products` MMAs of 512 cycles per
// K chunk (narrow tiles load more per MMA), 4000 for a tile's start and end, 6000 and 1000 each for parts, `most` of them.
Product cut(int64_t blocks, int m, int n, int kdim, int products, bool lower, int most)
{
    Product best = {};
    double best_cost = 1e300;
    const int64_t mt = ceil_div(m, 256), chunks = ceil_div(kdim, kPgChunk), share = blocks >= kPgPairs ? 1 : kPgPairs / (blocks > 0 ? blocks : 1);
    for (int tn = 256; tn >= 128; tn /= 2) {
        const int64_t tiles = lower ? mt * (mt + 1) / 2 * (256 / tn) : mt * ceil_div(n, tn);
        for (int s = 1; s <= most && s <= chunks; ++s) {
            if (s > 1 && tiles * s > share) break;
            const int64_t rounds = (tiles * s + share - 1) / share, per = (chunks + s - 1) / s;
            const double chunk = 512.0 * products * tn / 256 * (tn == 128 ? 1.2 : 1.0);
            const double cost = rounds * (per * chunk + 4000.0) + (s > 1 ? 6000.0 + 1000.0 * s : 0.0);
            if (cost < best_cost) {
                best_cost = cost;
                best.tn = tn;
                best.splits = s;
                best.tiles = (int)tiles;
            }
        }
    }
    best.rows = m;
    best.cols = n;
    best.kchunks = (int)chunks;
    best.per_split = ceil_div(chunks, best.splits);
    best.publishers = best.splits == 1 ? 16 : 16 * (best.splits < best.tn / 64 ? best.splits : best.tn / 64);
    best.sub = 256 / best.tn;
    best.lower = lower;
    best.ntiles = ceil_div(n, best.tn);
    best.scale = 1.0f;
    return best;
}

struct Large {
    int k, n, ldx, ldk, planes, parts;
    Product prod[3];               // S~, P, X
    int64_t counters, part_units;
    size_t norm, count, xp[2], sp, pp, part, total;
};

constexpr int kMostParts = 16;

Large large_layout(int64_t blocks, int rows, int cols, int dtype, int most = kMostParts)
{
    Large l;
    l.k = rows < cols ? rows : cols;
    l.n = rows < cols ? cols : rows;
    l.ldx = (cols + 15) / 16 * 16;
    l.ldk = (l.k + 15) / 16 * 16;
    l.planes = dtype == MONARCH_F32 ? 3 : 2;
    const int products = dtype == MONARCH_F32 ? 6 : 3;
    const bool wide = rows <= cols;
    l.prod[0] = cut(blocks, l.k, l.k, l.n, products, true, most);
    l.prod[1] = cut(blocks, l.k, l.k, l.k, products, true, most);
    l.prod[2] = cut(blocks, rows, cols, l.k, products, false, most);
    l.prod[0].a_mn = l.prod[0].b_mn = !wide;
    l.prod[2].b_mn = wide;
    l.prod[0].diagonal = kBeta;
    l.prod[1].scale = kC;
    l.prod[1].diagonal = kGamma;
    const size_t rc = (size_t)rows * cols, b = (size_t)blocks;
    const int64_t want = (int64_t)((rc + 8191) / 8192);
    l.parts = (int)(want < kNormParts ? want : kNormParts);
    size_t at = MONARCH_STATUS_BYTES + 65536;          // the status area and the counters of kernels that may share the workspace
    auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes); return o; };
    l.norm = take(b * l.parts * 8);
    l.counters = blocks;
    for (const Product &q : l.prod)
        if (q.splits > 1) l.counters += blocks * q.tiles * 16;
    l.count = take((size_t)l.counters * 4);
    // two X: the last product of a step reads the one and writes the other
    l.xp[0] = take(b * l.planes * rows * l.ldx * 2);
    l.xp[1] = take(b * l.planes * rows * l.ldx * 2);
    l.sp = take(b * l.planes * l.k * l.ldk * 2);
    l.pp = take(b * l.planes * l.k * l.ldk * 2);
    l.part_units = 0;
    for (const Product &q : l.prod)
        if (q.splits > 1 && (int64_t)q.tiles * q.splits > l.part_units) l.part_units = (int64_t)q.tiles * q.splits;
    l.part = take(b * l.part_units * 16 * 4096 * 4);
    l.total = at;
    return l;
}

// Fewer blocks are cut into more parts and may take more memory (512 x 512, fp32: 4 blocks 42 MB, 5 blocks 30): a workspace that was asked for
// with more blocks serves fewer in as many parts as it has room for.
Large large_within(size_t bytes, int64_t blocks, int rows, int cols, int dtype)
{
    Large l = large_layout(blocks, rows, cols, dtype);
    for (int most = kMostParts - 1; l.total > bytes && most >= 1; --most) l = large_layout(blocks, rows, cols, dtype, most);
    return l;
}

template <typename T, int PL, int SCHEME>
int ortho_large(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    const Large l = large_within(ws_bytes, blocks, rows, cols, dtype);
    char *base = (char *)ws;
    const bool wide = rows <= cols;
    double *norm = (double *)(base + l.norm);
    unsigned *count = (unsigned *)(base + l.count);
    const Planes sp = {(__nv_bfloat16 *)(base + l.sp), l.k, l.k, l.ldk}, pp = {(__nv_bfloat16 *)(base + l.pp), l.k, l.k, l.ldk};
    Planes x[2];
    OrthoMaps m;
    const int64_t xz = (int64_t)rows * l.ldx, kz = (int64_t)l.k * l.ldk, z = blocks * PL;
    const int ts = l.prod[0].tn / 2, tp = l.prod[1].tn / 2, tx = l.prod[2].tn / 2;
    for (int i = 0; i < 2; ++i) {
        x[i] = {(__nv_bfloat16 *)(base + l.xp[i]), rows, cols, l.ldx};
        MONARCH_TRY(plane_map(&m.s_a[i], x[i].at, !wide, rows, cols, l.ldx, xz, z));
        MONARCH_TRY(plane_map(&m.s_b[i], x[i].at, !wide, rows, cols, l.ldx, xz, z, ts));
        if (wide) {
            MONARCH_TRY(plane_map(&m.x_a[i], pp.at, 0, l.k, l.k, l.ldk, kz, z));
            MONARCH_TRY(plane_map(&m.x_b[i], x[i].at, 1, rows, cols, l.ldx, xz, z));
        } else {
            MONARCH_TRY(plane_map(&m.x_a[i], x[i].at, 0, rows, cols, l.ldx, xz, z));
            MONARCH_TRY(plane_map(&m.x_b[i], pp.at, 0, l.k, l.k, l.ldk, kz, z, tx));
        }
        MONARCH_TRY(plane_target(&m.x_to[i], x[i].at, rows, cols, l.ldx, xz, z));
    }
    MONARCH_TRY(plane_map(&m.p_a, sp.at, 0, l.k, l.k, l.ldk, kz, z));
    MONARCH_TRY(plane_map(&m.p_b, sp.at, 0, l.k, l.k, l.ldk, kz, z, tp));
    MONARCH_TRY(plane_target(&m.s_to, sp.at, l.k, l.k, l.ldk, kz, z));
    MONARCH_TRY(plane_target(&m.p_to, pp.at, l.k, l.k, l.ldk, kz, z));

    int64_t units = 0, all = 0;
    for (const Product &q : l.prod) {
        const int64_t u = blocks * q.tiles * q.splits;
        if (u > units) units = u;
        all += u * steps;
    }
    if (all > 0x7ffffff0) return MONARCH_ERR_UNSUPPORTED;               // tile numbers are 32 bits
    MONARCH_TRY(launch_serialized(norm_kernel<T>, dim3((unsigned)(blocks * l.parts)), 256, 0, s, io, norm, l.parts, (int64_t)rows * cols, count, l.counters));
    int64_t ctas = ceil_div((int64_t)rows * cols, 4096), most = 148 * 8 / blocks + 1;
    if (ctas > most) ctas = most;
    MONARCH_TRY(launch_serialized(start_kernel<T, PL>, dim3((unsigned)(blocks * ctas)), 256, 0, s, x[0], io, (const double *)norm, l.parts, (int)ctas));

    OrthoRun p = {};
    p.status = (unsigned *)ws;
    p.done = count;
    p.blocks = (int)blocks;
    p.steps = steps;
    p.rows = rows;
    p.cols = cols;
    p.part = (float *)(base + l.part);
    p.part_units = l.part_units;
    unsigned *next = count + blocks;
    for (int i = 0; i < 3; ++i) {
        p.prod[i] = l.prod[i];
        if (l.prod[i].splits > 1) {
            p.prod[i].parts_done = next;
            next += blocks * l.prod[i].tiles * 16;
        }
    }
    const auto kern = ortho_run_kernel<T, PL, SCHEME>;
    static PerDeviceCache cache;
    int pairs = cache.get();
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kPgThreads);
    cfg.dynamicSmemBytes = kRunSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeCooperative;            // all CTAs resident at once: tiles wait for one another
    attr[1].val.cooperative = 1;
    cfg.attrs = attr;
    if (pairs < 0) {
        MONARCH_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRunSmem));
        cfg.gridDim = dim3(2);
        cfg.numAttrs = 1;
        MONARCH_CUDA_TRY(cudaOccupancyMaxActiveClusters(&pairs, kern, &cfg));
        cache.set(pairs);
    }
    if (pairs < 1) return MONARCH_ERR_CUDA;
    cfg.gridDim = dim3((unsigned)(2 * (units < pairs ? units : pairs)));
    cfg.numAttrs = 2;
    MONARCH_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, m, p, io));
    note_launch();
    return MONARCH_OK;
}

// Which kernel serves blocks whose smaller side is k and larger side n; not by their number, so that a workspace for many blocks
// serves fewer (large_within).
enum Kernel { kWarpMma, kTcgen05, kFma, kRun };
Kernel kernel_for(int k, int n)
{
    if (k > 32 && n <= 128) return kTcgen05;
    if (fits_block(k, n)) return kWarpMma;
    return fits_small(k, n) ? kFma : kRun;
}

template <typename T, int PL, int SCHEME>
int ortho_any(const Io<T> &io, int64_t blocks, int rows, int cols, int steps, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    if (blocks == 0) return MONARCH_OK;
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    switch (kernel_for(k, n)) {
        case kTcgen05:
            if (k > 64) return launch_tc<T, PL, 128, 128>(io, blocks, rows, cols, steps, ws, s);
            if (n > 64) return launch_tc<T, PL, 64, 128>(io, blocks, rows, cols, steps, ws, s);
            return launch_tc<T, PL, 64, 64>(io, blocks, rows, cols, steps, ws, s);
        case kWarpMma: return ortho_block<T, PL>(io, blocks, rows, cols, steps, s);
        case kFma:
            return launch_serialized_up_to((int)kSmallMax, ortho_small_kernel<T>, dim3((unsigned)blocks), kSmallThreads, (int)(small_floats(k, n) * 4), s, io, rows, cols, steps);
        default: return ortho_large<T, PL, SCHEME>(io, blocks, rows, cols, steps, dtype, ws, ws_bytes, s);
    }
}

}  // namespace
}  // namespace tc

// `least`: what a call needs, else what it runs best with
size_t ortho_workspace_bytes(int64_t blocks, int32_t rows, int32_t cols, int dtype, bool least)
{
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return tc::kernel_for(k, n) != tc::kRun ? (size_t)MONARCH_STATUS_BYTES : tc::large_layout(blocks, rows, cols, dtype, least ? 1 : tc::kMostParts).total;
}

int orthogonalize(const void *G, void *O, int64_t blocks, int32_t rows, int32_t cols, int32_t steps, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    if (dtype == MONARCH_F32) {
        const tc::Io<float> io = {G, nullptr, (float *)O, 0.0f, 0.0f, 0.0f, 0};
        return tc::ortho_any<float, 3, tc::kP3x3>(io, blocks, rows, cols, steps, dtype, ws, ws_bytes, s);
    }
    const tc::Io<__nv_bfloat16> io = {G, nullptr, (__nv_bfloat16 *)O, 0.0f, 0.0f, 0.0f, 0};
    return tc::ortho_any<__nv_bfloat16, 2, tc::kP2x2>(io, blocks, rows, cols, steps, dtype, ws, ws_bytes, s);
}

int muon_step(void *W, const float *dW, float *V, int64_t blocks, int32_t rows, int32_t cols, float keep, float step, float beta, int nesterov,
              int32_t steps, int dtype, void *ws, size_t ws_bytes, cudaStream_t s)
{
    if (dtype == MONARCH_F32) {
        const tc::Io<float> io = {dW, V, (float *)W, keep, step, beta, nesterov};
        return tc::ortho_any<float, 3, tc::kP3x3>(io, blocks, rows, cols, steps, dtype, ws, ws_bytes, s);
    }
    const tc::Io<__nv_bfloat16> io = {dW, V, (__nv_bfloat16 *)W, keep, step, beta, nesterov};
    return tc::ortho_any<__nv_bfloat16, 2, tc::kP2x2>(io, blocks, rows, cols, steps, dtype, ws, ws_bytes, s);
}

}  // namespace monarch
