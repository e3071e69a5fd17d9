// Matrix products on CTA pairs (tcgen05, cta_group::2) whose operands are held as one, two or three bf16 PLANES: a value is
// hi + lo (+ lo2), each plane the bf16 rounding of what the ones before it leave: off by at most 2^-8, 2^-16 or 2^-24 of the
// value.  A product of two such operands is a few plane products added up in the same fp32 accumulator:
//   kP1    hi hi                                        operands that are bf16 themselves
//   kP2x1  hi hi + lo hi                                first operand in two planes, second one bf16
//   kP3x1  the same with three planes of the first
//   kP2x2  hi hi + hi lo + lo hi                        both in two planes (left out: lo lo, at most 2^-16 of the product)
//   kP3x3  the six with at most two orders of lo        fp32 operands (left out: 2^-23 of the product), hi hi last
// A tf32 product would keep 11 bits and fp32 FMA runs at a 25th of this rate.
//
//   C[m][n] = sum_k A(m, k) B(n, k)       A, B stored [rows][K] (K-major) or [K][rows] (MN-major), each with its own flag
//
// Persistent kernel on clusters of two CTAs, output tiles of 256 rows and tn = 256 columns (192 or 128 where that fills the pairs
// better: pg_tile): CTA r of a pair owns 128 rows of A and loads tn / 2 of the rows of B; one MMA instruction of 256 x tn x 16 runs
// on both SMs.  Shared memory is a ring of 16 KB operand tiles
// (128 x 64, 128-byte swizzle), loaded in the order in which the plane products use them, so that a tile of a plane is loaded
// once per K chunk however many products it enters.  Two accumulators of 256 columns in tensor memory alternate.
//   warps 0-7  epilogue: warp w reads rows 32 (w % 4) .. of column half w / 4
//   warp 8     lane 0: TMA loads;  warp 9  lane 0 of the even CTA: MMAs
// Every wait is bounded (tc_common.cuh).
#pragma once

#include "mma_tiles.cuh"

namespace monarch {
namespace tc {

enum PlaneScheme { kP1 = 0, kP2x1 = 1, kP2x2 = 2, kP3x3 = 3, kP3x1 = 4 };

constexpr int kPgTile = 256, kPgChunk = 64;
constexpr int kPgSlotBytes = 128 * kPgChunk * 2, kPgMaxSlots = 13;
constexpr int kPgThreads = 320, kPgEpiWarps = 8;
constexpr int kPgStageBytes = 32 * 32 * 2;      // an epilogue warp's piece of a bf16 result
// slots beside `stage` such pieces per epilogue warp
__host__ __device__ constexpr int pg_slots(int stage) { return kPgMaxSlots - stage * kPgEpiWarps * kPgStageBytes / kPgSlotBytes; }
__host__ __device__ constexpr int pg_smem(int stage) { return pg_slots(stage) * kPgSlotBytes + stage * kPgEpiWarps * kPgStageBytes + 1024; }

// loads per K chunk: bit 2 = operand B, bits 0-1 = plane
__host__ __device__ constexpr int pg_loads(int s) { return s == kP1 ? 2 : s == kP2x1 ? 3 : s == kP2x2 || s == kP3x1 ? 4 : 6; }
__host__ __device__ constexpr int pg_load(int s, int l)
{
    constexpr int kB = 4;
    constexpr int t[5][6] = {{0, kB, 0, 0, 0, 0}, {kB, 0, 1, 0, 0, 0}, {0, kB, kB + 1, 1, 0, 0}, {0, kB + 2, kB + 1, 1, kB, 2}, {kB, 0, 1, 2, 0, 0}};
    return t[s][l];
}
// products that become possible with load l: (load of A) | (load of B) << 4, up to two; 0xff: none
__host__ __device__ constexpr int pg_mma(int s, int l, int i)
{
    constexpr int none = 0xff;
    constexpr int t[5][6][2] = {{{none, none}, {0x10, none}, {none, none}, {none, none}, {none, none}, {none, none}},
                                {{none, none}, {0x01, none}, {0x02, none}, {none, none}, {none, none}, {none, none}},
                                {{none, none}, {0x10, none}, {0x20, none}, {0x13, none}, {none, none}, {none, none}},
                                {{none, none}, {0x10, none}, {0x20, none}, {0x23, none}, {0x43, none}, {0x45, 0x40}},
                                {{none, none}, {0x01, none}, {0x02, none}, {0x03, none}, {none, none}, {none, none}}};
    return t[s][l][i];
}
// loads whose last use is among the products of load l (bit mask)
__host__ __device__ constexpr int pg_done(int s, int l)
{
    constexpr int t[5][6] = {{0, 3, 0, 0, 0, 0}, {0, 2, 5, 0, 0, 0}, {0, 0, 5, 10, 0, 0}, {0, 2, 0, 4, 8, 49}, {0, 2, 4, 9, 0, 0}};
    return t[s][l];
}

// The tensor cores add to an fp32 accumulator without rounding to nearest: sums of mixed signs shrink by some 2^-25 per step of 16
// products (measured: a sum over 8192 tokens of two planes, 1024 steps, was 1.9e-5 off; 3e-5 over 1500 steps).  Where the result is
// float32, a run in tensor memory ends after this many K chunks and the epilogue warps add the runs up in registers, while the
// MMAs go on in the other accumulator.  With all six plane products a run is one chunk, hi hi last: the 20 steps before it lose of
// sums that are 2^-8 as large, four of the whole (orthogonalised update in fp32, hi hi first and runs of two chunks: 1.9e-5 off).
__host__ __device__ constexpr int pg_seg(int s) { return s == kP1 ? 16 : s == kP2x1 ? 8 : s == kP2x2 || s == kP3x1 ? 5 : 1; }

struct PlaneGemm {
    unsigned *status;
    const int *count;          // device: rows that take part (token rows), or null
    int count_is_k;            // count bounds K (else M)
    int row0, rows;            // rows of M: row0 .. row0 + rows (rows clipped by *count - row0)
    int cols, tn;              // columns of N; columns of a tile: 256, 128 or, K-major B only, 192
    int kdim;                  // contraction length (clipped by *count)
    int a_k0, b_k0;            // first K coordinate of the operands
    int b_n0;                  // first N coordinate of B
    int splits;                // parts of K, each a product of its own
    int *splits_out;           // device: null, or `splits` is the most there may be, the kernel chooses (pg_cost) and says so here
    const int *splits_in;      // device: null, or the number of parts
    int n_fastest;             // neighbouring pairs take neighbouring column tiles (else row tiles)
    int seg;                   // K chunks per accumulation in tensor memory (kernels with PROMOTE)
    int half;                  // the operands' 16-bit values are fp16
};

struct PgTile {
    int z, row, col;           // part of K; this thread's row; first of this warp's columns (a half of the tile)
    int half;                  // which half tile of the columns that is
    int zero;                  // nothing was accumulated
};

constexpr int kPgPairs = 74;       // CTA pairs of a B200: what sizes are chosen for (launches ask the device)

// Time of `tiles` output tiles in `s` parts of K, in K chunks: rounds of the pairs over the parts; a part costs some 6 chunks more
__host__ __device__ constexpr long long pg_cost(long long tiles, int kchunks, int s)
{
    return (tiles * s + kPgPairs - 1) / kPgPairs * ((kchunks + s - 1) / s + 6);
}
// Columns of a tile: the width that takes the pairs the fewest column rounds; narrower tiles reload A more often (a tenth, a fifth)
inline int pg_tile(long long mtiles, int cols, bool any)
{
    auto cost = [&](int tn, int slow) { return (mtiles * ((cols + tn - 1) / tn) + kPgPairs - 1) / kPgPairs * tn * slow; };
    int best = 256;
    if (any && cost(192, 11) < cost(best, 10)) best = 192;
    if (cost(128, 12) < cost(best, best == 192 ? 11 : 10)) best = 128;
    return best;
}

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *m, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(m), "r"(bar & 0xFEFFFFFFu), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// 32 consecutive columns of this thread's lane, waited for
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&f)[32])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(f);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
    // the wait names the registers, so that nothing that reads them can move before it
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27])
                 :
                 : "memory");
    asm volatile("" : "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}

// 16 columns of this thread's lane, requested; tmem_ready names the registers so that nothing that reads them moves before it
__device__ __forceinline__ void tmem_ask16(uint32_t taddr, float (&f)[16]) { tmem_ld16(taddr, reinterpret_cast<uint32_t (&)[16]>(f)); }
__device__ __forceinline__ void tmem_ready(float (&f)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]), "+f"(f[8]), "+f"(f[9]),
                   "+f"(f[10]), "+f"(f[11]), "+f"(f[12]), "+f"(f[13]), "+f"(f[14]), "+f"(f[15])
                 :
                 : "memory");
}

// one lane of a converged warp; unlike lane == 0 it leaves the operands of what follows in uniform registers
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Results leave through shared memory, N pieces of 2 KB per epilogue warp.  A thread has a row of 32 columns: stored from registers,
// each instruction would touch 32 rows of 16 or 32 bytes.
//   bf16 planes  32 x 32 pieces (64-byte swizzle) that TMA writes, all planes of a chunk behind one proxy fence (a fence per piece
//                took 0.5 us each); lane 0 sends and waits
//   float32      32 x 32 tiles of two pieces (128-byte swizzle) that TMA writes or adds to what is there, where rows allow it; else, and
//                where rows go to places of their own, a tile read back a row at a time, lane = column
template <int N> struct PgStage {
    const CUtensorMap *map;
    uint32_t base;
    int lane, turn;
    __device__ __forceinline__ uint32_t piece(int i) const { return base + i * kPgStageBytes; }
    // the pieces sent have been read, but for those of the last PENDING groups
    template <int PENDING = 0> __device__ __forceinline__ void begin() const
    {
        if (lane == 0) tma_store_wait_read<PENDING>();
        __syncwarp();
    }
    // 16 packed words: this lane's row of 32 values
    __device__ __forceinline__ void row(int i, const uint32_t (&w)[16]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece(i) + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)), "r"(w[4 * j]),
                         "r"(w[4 * j + 1]), "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                         : "memory");
    }
    // piece `to` = piece `from` transposed, 8 x 8 blocks at a time (after a __syncwarp)
    __device__ __forceinline__ void transpose(int from, int to) const
    {
        const int i = lane, r = lane & 7, blk = lane >> 3;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m[4];
            ldm4t(m, piece(from) + i * 64 + ((j ^ ((i >> 1) & 3)) << 4));                         // blocks (0 .. 3, j)
            const int o = 8 * j + r;
            stm4(piece(to) + o * 64 + ((blk ^ ((o >> 1) & 3)) << 4), m);                          // blocks (j, 0 .. 3)
        }
    }
    // everything written is visible to TMA; then lane 0 sends pieces and closes the group
    __device__ __forceinline__ void ready() const
    {
        fence_proxy_async_smem();
        __syncwarp();
    }
    __device__ __forceinline__ void send(int i, int x, int y, int z) const
    {
        if (lane == 0) tma_store_3d(map, piece(i), x, y, z);
    }
    __device__ __forceinline__ void close() const
    {
        if (lane == 0) tma_store_commit();
    }
    // a float32 tile, the other one of two each time: this lane's row of 32 values, to (x, y, z) of the map or added to what is there; N >= 4
    __device__ __forceinline__ void tile(const float (&v)[32], int x, int y, int z, bool add)
    {
        static_assert(N >= 4 || N == 0, "two tiles");
        const uint32_t buf = base + turn * 4096;
        turn ^= 1;
        if (lane == 0) tma_store_wait_read<1>();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "f"(v[4 * j]), "f"(v[4 * j + 1]),
                         "f"(v[4 * j + 2]), "f"(v[4 * j + 3])
                         : "memory");
        ready();
        if (lane == 0) {
            if (add)
                asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(buf), "r"(x), "r"(y),
                             "r"(z)
                             : "memory");
            else
                tma_store_3d(map, buf, x, y, z);
            tma_store_commit();
        }
    }
    // f(row, value of column `lane` in that row, old(row)) for 32 rows, eight `old` at a time before the first of their `f`; N >= 2
    template <class G, class F> __device__ __forceinline__ void rows(const float (&v)[32], G old, F f) const
    {
        static_assert(N * kPgStageBytes >= 32 * 32 * 4, "a tile of floats");
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; ++j) asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + (lane * 32 + (j ^ lane)) * 4), "f"(v[j]) : "memory");
        __syncwarp();
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += 8) {
            float w[8], x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = old(r0 + k);
#pragma unroll
            for (int k = 0; k < 8; ++k) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[k]) : "r"(base + ((r0 + k) * 32 + (lane ^ (r0 + k))) * 4) : "memory");
#pragma unroll
            for (int k = 0; k < 8; ++k) f(r0 + k, x[k], w[k]);
        }
    }
};

struct PgBars {
    uint64_t full[kPgMaxSlots], empty[kPgMaxSlots];                           // full: used in the even CTA only
    uint64_t acc_full[2], acc_empty[2];
};

// A wait whose common case is one instruction, the rest out of line: these kernels are often launched for one tile per pair, and
// what they have not executed before has to be fetched first.
static __device__ __noinline__ bool pg_wait_on(uint32_t bar, uint32_t parity, unsigned *status, volatile int *dead, unsigned code)
{
    return mbar_wait<true>(bar, parity, status, dead, code);
}
__device__ __forceinline__ bool pg_wait(uint32_t bar, uint32_t parity, unsigned *status, volatile int *dead, unsigned code)
{
    return mbar_try_wait_cluster_acquire(bar, parity) || pg_wait_on(bar, parity, status, dead, code);
}
// The same by a whole warp, which goes on or gives up together: what follows takes all lanes
__device__ __forceinline__ bool pg_wait_warp(uint32_t bar, uint32_t parity, unsigned *status, volatile int *dead, unsigned code)
{
    return __all_sync(~0u, pg_wait(bar, parity, status, dead, code));
}

// Epi: struct with  begin(const Epi::Args &, const PgTile &) (a tile ahead: loads),  start(args, tile),  chunk(args, tile, c, float (&v)[32], stage)  for c = 0, 32, .. < tn / 2,
// end(args, tile); kStage: pieces in `stage`, its warp's PgStage (0: none).  PROMOTE: at most p.seg chunks are accumulated in tensor memory, sums of those in fp32 registers.
template <int AMN, int BMN, int SCHEME, bool PROMOTE, class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPgThreads, 1)
plane_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_c,
                  const PlaneGemm p, const typename Epi::Args args)
{
    constexpr int kPgSlots = pg_slots(Epi::kStage);
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) PgBars bars;
    __shared__ uint32_t tmem_base_s;
    __shared__ int dead_s;

    const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // the same in all lanes, for the compiler too
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
    volatile int *dead = &dead_s;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPgSlots; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 1);                      // the even CTA's expect_tx arrival
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&bars.acc_full[a]), 1);
            mbar_init(smem_u32(&bars.acc_empty[a]), 2 * kPgEpiWarps);   // epilogue warps of both CTAs
        }
        fence_mbar_init();
        dead_s = 0;
        tma_prefetch_desc(&tm_a);
        tma_prefetch_desc(&tm_b);
    }
    if (warp == 0) {
        tmem_alloc_pair(smem_u32(&tmem_base_s), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive_release();                                           // both CTAs' barriers exist before any remote arrive
    cluster_wait_acquire();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(~0u, tmem_base_s, 0);
    depend_launch();
    depend_wait();

    int rows = p.rows, kdim = p.kdim;
    if (p.count != nullptr) {
        const int n = *p.count;
        if (p.count_is_k) kdim = min(kdim, n);
        else rows = max(0, min(rows, n - p.row0));
    }
    const int tn = p.tn;
    const int mtiles = (rows + kPgTile - 1) / kPgTile, ntiles = (p.cols + tn - 1) / tn;
    const int kchunks = (kdim + kPgChunk - 1) / kPgChunk;
    const int plane_tiles = mtiles * ntiles;
    int splits = p.splits_in != nullptr ? *p.splits_in : p.splits;
    if (p.splits_out != nullptr) {
        // the cheapest number of parts; every warp finds the same one
        long long best = 0x7fffffffffffffffLL;
        for (int s = lane + 1; s <= p.splits; s += 32) best = min(best, pg_cost(plane_tiles, kchunks, s) << 10 | s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(~0u, best, o));
        splits = (int)(best & 1023);
        if (blockIdx.x == 0 && threadIdx.x == 0) *p.splits_out = splits;
    }
    const int per_split = (kchunks + splits - 1) / splits;
    const int total = plane_tiles * splits;                               // below 2^31 (launch_plane_gemm)
    const uint32_t full0 = smem_u32(bars.full), empty0 = smem_u32(bars.empty);
    const uint32_t accf0 = smem_u32(bars.acc_full), acce0 = smem_u32(bars.acc_empty);
    constexpr int kLoads = pg_loads(SCHEME);
    const int seg = PROMOTE ? p.seg : 0x7fffffff;

    struct At {
        int split, mt, nt, c0, c1;
    };
    auto locate = [&](int tile) {
        At a;
        a.split = splits > 1 ? tile / plane_tiles : 0;
        const int t = tile - a.split * plane_tiles;
        const int q = t / (p.n_fastest ? ntiles : mtiles), r = t - q * (p.n_fastest ? ntiles : mtiles);
        a.mt = p.n_fastest ? q : r;
        a.nt = p.n_fastest ? r : q;
        a.c0 = min(a.split * per_split, kchunks);
        a.c1 = min(a.c0 + per_split, kchunks);
        return a;
    };

    if (warp == 8) {
        // ------------------------------------------------------------ loader (both CTAs)
        if (elect_one()) {
            uint32_t slot = 0, phase = 1;
            bool ok = true;
            for (int tile = pair; ok && tile < total; tile += npairs) {
                const At at = locate(tile);
                const int m0 = p.row0 + at.mt * kPgTile + (int)rank * 128, n0 = p.b_n0 + at.nt * tn + (int)rank * (tn / 2);
                for (int c = at.c0; ok && c < at.c1; ++c) {
                    const int ka = p.a_k0 + c * kPgChunk, kb = p.b_k0 + c * kPgChunk;
#pragma unroll
                    for (int l = 0; l < kLoads; ++l) {
                        if (!pg_wait(empty0 + slot * 8, phase, p.status, dead, kErrSlotWait)) { ok = false; break; }
                        const uint32_t dst = ring0 + slot * kPgSlotBytes, full = full0 + slot * 8;
                        constexpr int tag[6] = {pg_load(SCHEME, 0), pg_load(SCHEME, 1), pg_load(SCHEME, 2), pg_load(SCHEME, 3),
                                                pg_load(SCHEME, 4), pg_load(SCHEME, 5)};
                        const int plane = tag[l] & 3;
                        // the even CTA announces the bytes of both halves; either CTA's may land first
                        if (rank == 0) mbar_expect_tx(full, (tag[l] & 4) ? tn * (kPgChunk * 2) : 2 * kPgSlotBytes);
                        if (tag[l] & 4) {
                            const int z = plane;
                            if constexpr (BMN) {
                                tma_load_3d_pair(dst, &tm_b, n0, kb, z, full);
                                if (tn == 256) tma_load_3d_pair(dst + 8192, &tm_b, n0 + 64, kb, z, full);
                            } else {
                                tma_load_3d_pair(dst, &tm_b, kb, n0, z, full);
                            }
                        } else {
                            const int z = plane;
                            if constexpr (AMN) {
                                tma_load_3d_pair(dst, &tm_a, m0, ka, z, full);
                                tma_load_3d_pair(dst + 8192, &tm_a, m0 + 64, ka, z, full);
                            } else {
                                tma_load_3d_pair(dst, &tm_a, ka, m0, z, full);
                            }
                        }
                        if (++slot == kPgSlots) { slot = 0; phase ^= 1; }
                    }
                }
            }
        }
    } else if (warp == 9) {
        if (rank == 0 && elect_one()) {
            // ------------------------------------------------------------ even CTA: MMA issuer for the pair
            const uint32_t idesc = make_idesc_bf16(256, tn, AMN, BMN) & (p.half ? ~((1u << 7) | (1u << 10)) : ~0u);     // formats of A and B: 1 bf16, 0 fp16
            constexpr uint32_t astep = AMN ? 128 : 2, bstep = BMN ? 128 : 2;
            const uint64_t adesc = AMN ? make_smem_desc(0, 8192, 1024, kSwizzle128) : make_smem_desc(0, 16, 1024, kSwizzle128);
            const uint64_t bdesc = BMN ? make_smem_desc(0, 8192, 1024, kSwizzle128) : make_smem_desc(0, 16, 1024, kSwizzle128);
            uint32_t slot = 0, phase = 0, it = 0;
            bool ok = true;
            for (int tile = pair; ok && tile < total; tile += npairs) {
                const At at = locate(tile);
                for (int c0 = at.c0; ok && c0 < at.c1; c0 = (at.c1 - c0 > seg) ? c0 + seg : at.c1, ++it) {
                    const int c1 = (at.c1 - c0 > seg) ? c0 + seg : at.c1;
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
                            if (++slot == kPgSlots) { slot = 0; phase ^= 1; }
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
        const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * (tn / 2));
        uint32_t it = 0;
        bool ok = true;
        PgStage<(Epi::kStage > 0 ? Epi::kStage : 1)> stage = {&tm_c, ring0 + kPgSlots * kPgSlotBytes + warp * Epi::kStage * kPgStageBytes, lane, 0};
        auto place = [&](const At &at) {
            PgTile t;
            t.z = at.split;
            t.half = at.nt * 2 + (warp >> 2);
            t.row = p.row0 + at.mt * kPgTile + (int)rank * 128 + (warp & 3) * 32 + lane;
            t.col = at.nt * tn + (warp >> 2) * (tn / 2);
            t.zero = at.c0 >= at.c1;
            return t;
        };
        // what a tile's rows bring along is asked for a tile ahead
        At at_next = locate(min(pair, max(total - 1, 0)));
        PgTile t_next = place(at_next);
        Epi e_next;
        if (pair < total) e_next.begin(args, t_next);
        for (int tile = pair; ok && tile < total; tile += npairs) {
            const At at = at_next;
            const PgTile t = t_next;
            Epi e = e_next;
            if (tile + npairs < total) {
                at_next = locate(tile + npairs);
                t_next = place(at_next);
                e_next.begin(args, t_next);
            }
            e.start(args, t);
            if constexpr (!PROMOTE) {
                uint32_t buf = it & 1;
                if (!t.zero) {
                    if (!pg_wait_warp(accf0 + buf * 8, (it >> 1) & 1, p.status, dead, kErrMmaWait)) { ok = false; break; }
                    tc_fence_after();
                    ++it;
                }
#pragma unroll 1
                for (int h = 0; h * 64 < tn; ++h) {
                    float v[32];
                    if (!t.zero) {
                        tmem_ld32(lane_base + buf * 256 + h * 32, v);
                        if ((h + 1) * 64 >= tn) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_remote(acce_leader + buf * 8);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                    }
                    e.chunk(args, t, h * 32, v, stage);
                }
            } else {
                float acc[4][32];
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[h][i] = 0.0f;
                for (int c0 = at.c0; c0 < at.c1; c0 = (at.c1 - c0 > seg) ? c0 + seg : at.c1, ++it) {
                    const uint32_t buf = it & 1;
                    if (!pg_wait_warp(accf0 + buf * 8, (it >> 1) & 1, p.status, dead, kErrMmaWait)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        if (h * 64 >= tn) break;
#pragma unroll
                        for (int g = 0; g < 32; g += 16) {                    // 16 at a time: registers
                            float v[16];
                            tmem_ask16(lane_base + buf * 256 + h * 32 + g, v);
                            tmem_ready(v);
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[h][g + i] += v[i];
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(acce_leader + buf * 8);
                }
                if (!ok) break;
                // one copy of the conversion, the columns moved up to it: a launch of one tile per pair runs this code once, and most
                // of the time of four copies went into fetching them (2 us for 32 columns)
#pragma unroll 1
                for (int h = 0; h * 64 < tn; ++h) {
                    e.chunk(args, t, h * 32, acc[0], stage);
#pragma unroll
                    for (int i = 0; i < 32; ++i) { acc[0][i] = acc[1][i]; acc[1][i] = acc[2][i]; acc[2][i] = acc[3][i]; }
                }
            }
            e.end(args, t);
        }
        if (Epi::kStage > 0 && lane == 0) tma_store_wait_all<0>();
    }

    // the even CTA's barriers receive arrivals from the odd CTA until it is done: leave together.  After a wait that ran out no load,
    // which lands here, and no MMA, which reads here and writes tensor memory, may outlive this CTA, whichever warp gave up
    tc_fence_before();
    __syncthreads();
    let_copies_land(dead);
    cluster_arrive_release();
    cluster_wait_acquire();
    if (warp == 0) tmem_dealloc_pair(tmem_base, 512);
}

// A stack of `z` matrices [rows][cols] (bf16, rows `ld` elements apart, matrices `zstride` elements apart) as an operand.
// K-major: boxes of 64 columns x 128 rows (`box_rows`: tn / 2 for the second operand); MN-major: 64 columns x 64 rows, two side by
// side or, tn = 128, one.
inline int plane_map(CUtensorMap *m, const void *base, int mn_major, int64_t rows, int64_t cols, int64_t ld, int64_t zstride, int64_t z, int box_rows = 128)
{
    const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)z};
    const uint64_t strides[2] = {(uint64_t)ld * 2, (uint64_t)zstride * 2};
    const uint32_t box[3] = {64, mn_major ? 64u : (uint32_t)box_rows, 1};
    return encode_tmap_nd(m, base, 2, 3, dims, strides, box, 128);
}

// as the target of PgStage pieces
inline int plane_target(CUtensorMap *m, const void *base, int64_t rows, int64_t cols, int64_t ld, int64_t zstride, int64_t z)
{
    const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)z};
    const uint64_t strides[2] = {(uint64_t)ld * 2, (uint64_t)zstride * 2};
    const uint32_t box[3] = {32, 32, 1};
    return encode_tmap_nd(m, base, 2, 3, dims, strides, box, 64);
}

// as the target of PgStage::tile (cols a multiple of 4)
inline int tile_target(CUtensorMap *m, const void *base, int64_t rows, int64_t cols, int64_t zstride, int64_t z)
{
    const uint64_t dims[3] = {(uint64_t)cols, (uint64_t)rows, (uint64_t)z};
    const uint64_t strides[2] = {(uint64_t)cols * 4, (uint64_t)zstride * 4};
    const uint32_t box[3] = {32, 32, 1};
    return encode_tmap_nd(m, base, 4, 3, dims, strides, box, 128);
}

// tm_c: the target of an epilogue that has a stage (any map for the others)
template <int AMN, int BMN, int SCHEME, bool PROMOTE, class Epi>
int launch_plane_gemm(const CUtensorMap &tm_a, const CUtensorMap &tm_b, const CUtensorMap &tm_c, const PlaneGemm &p, const typename Epi::Args &args, cudaStream_t s)
{
    constexpr int kPgSmem = pg_smem(Epi::kStage);
    const auto kern = plane_gemm_kernel<AMN, BMN, SCHEME, PROMOTE, Epi>;
    static PerDeviceCache cache;
    int pairs = cache.get();
    if (pairs < 0) {
        MONARCH_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kPgSmem));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2, 1, 1);
        cfg.blockDim = dim3(kPgThreads, 1, 1);
        cfg.dynamicSmemBytes = kPgSmem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        MONARCH_CUDA_TRY(cudaOccupancyMaxActiveClusters(&pairs, kern, &cfg));
        cache.set(pairs);
    }
    if (pairs < 1) return MONARCH_ERR_CUDA;
    const long long mt = (p.rows + kPgTile - 1) / kPgTile;
    const long long total = mt * ((p.cols + p.tn - 1) / p.tn) * p.splits;
    if (total <= 0) return MONARCH_OK;
    if (total > 0x7ffffff0) return MONARCH_ERR_UNSUPPORTED;
    const int grid = 2 * (int)(total < pairs ? total : pairs);
    return launch_serialized(kern, dim3((unsigned)grid), kPgThreads, kPgSmem, s, tm_a, tm_b, tm_c, p, args);
}

}  // namespace tc
}  // namespace monarch
